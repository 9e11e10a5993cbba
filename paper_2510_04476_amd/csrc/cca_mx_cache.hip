// The latent cache in 4 bits: rows stored, read back, and evicted by accumulated attention weight (include/cca.h).
#include "cca_mx.h"

namespace cca {

namespace {

constexpr int TOK = 64;  // tokens of a workgroup

// ---------------------------------------------------------------------------
// Store: one workgroup per (64 tokens, head, sequence) and K or V.  A lane takes 8 numbers (16 or 32 bytes), four lanes a group:
// its largest magnitude over them by two lane exchanges, then 4 conversions of two numbers each.  Bound by what it moves (read 2
// or 4 bytes a number, write 17 / 32).  The scale bytes of a token lie T bytes apart, those of neighbouring tokens
// side by side: they go through LDS so that a wavefront stores them along the tokens.
// ---------------------------------------------------------------------------
struct StoreArgs {
  int n, Hk, dh, T, max_row;
  long long tiles;  // B * 2 H_k * ceil(n / 64): K's heads of a sequence, then V's

  const int *rows, *counts, *pos;
  int *row_pos;
  float *weight;
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const mx_u4 w = *reinterpret_cast<const mx_u4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = mx_lo(w[i]), x[2 * i + 1] = mx_hi(w[i]);
  } else {
    const mx_f4 a = *reinterpret_cast<const mx_f4 *>(p), b = *reinterpret_cast<const mx_f4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
}

// The scale of a lane's group (4 lanes x 8 numbers)
__device__ __forceinline__ uint32_t group_scale(const float (&x)[8]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = mx_max_abs(a, x[i]);
  a = mx_max_abs(a, mx_dpp<0xB1>(a));  // quad_perm [1,0,3,2]
  a = mx_max_abs(a, mx_dpp<0x4E>(a));  // quad_perm [2,3,0,1]
  return mx_scale_of(a);
}

template <typename T>
__global__ __launch_bounds__(256) void mx_store_kernel(StoreArgs a, const T *__restrict__ k, const T *__restrict__ v,
                                                      unsigned char *__restrict__ k_codes, unsigned char *__restrict__ k_scales,
                                                      unsigned char *__restrict__ v_codes, unsigned char *__restrict__ v_scales) {
  __shared__ unsigned char sc[8][TOK];  // (d_h / 32 <= 8 groups)
  const int tid = threadIdx.x, per = (a.n + TOK - 1) / TOK;
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, __syncthreads()) {
    const int t0 = (int)(tile % per) * TOK, hv = (int)(tile / per % (2 * a.Hk)), h = hv % a.Hk, b = (int)(tile / per / (2 * a.Hk));
    const bool is_v = hv >= a.Hk;
    const int row0 = mx_clamp(a.rows[b], 0, a.max_row), live = min(mx_clamp(a.counts ? a.counts[b] : a.n, 0, a.n), a.T - row0);
    const int nt = min(TOK, live - t0);
    if (nt <= 0) continue;
    const T *src = (is_v ? v : k) + ((long long)b * a.n * a.Hk + h) * a.dh;
    const long long head = (long long)b * a.Hk + h;
    unsigned char *codes = (is_v ? v_codes : k_codes) + (head * a.T + row0) * (a.dh / 2);
    const int lpr = a.dh / 8;  // lanes of a row
    for (int i = tid; i < nt * lpr; i += 256) {  // (a multiple of 4 lanes: a group's lanes are together)
      const int t = i / lpr, c = i % lpr;
      float x[8];
      load8(src + (long long)(t0 + t) * a.Hk * a.dh + c * 8, x);
      const uint32_t s = group_scale(x);
      *reinterpret_cast<uint32_t *>(codes + (long long)(t0 + t) * (a.dh / 2) + c * 4) = mx_codes(x, s);
      if ((c & 3) == 0) sc[c >> 2][t] = (unsigned char)s;
    }
    __syncthreads();
    unsigned char *scales = (is_v ? v_scales : k_scales) + head * (a.dh / 32) * a.T + row0 + t0;
    for (int i = tid; i < a.dh / 32 * TOK; i += 256)
      if (i % TOK < nt) scales[(long long)(i / TOK) * a.T + i % TOK] = sc[i / TOK][i % TOK];
    if (!is_v && tid < nt) {
      const long long at = head * a.T + row0 + t0 + tid;
      if (a.row_pos) a.row_pos[at] = (a.pos ? a.pos[b] : row0) + t0 + tid;
      if (a.weight) a.weight[at] = 0.f;
    }
  }
}

// Read back: the same workgroups the other way round
template <typename T>
__global__ __launch_bounds__(256) void mx_rows_kernel(StoreArgs a, T *__restrict__ k, T *__restrict__ v,
                                                     const unsigned char *__restrict__ k_codes, const unsigned char *__restrict__ k_scales,
                                                     const unsigned char *__restrict__ v_codes, const unsigned char *__restrict__ v_scales) {
  __shared__ unsigned char sc[8][TOK];
  const int tid = threadIdx.x, per = (a.n + TOK - 1) / TOK;
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, __syncthreads()) {
    const int t0 = (int)(tile % per) * TOK, hv = (int)(tile / per % (2 * a.Hk)), h = hv % a.Hk, b = (int)(tile / per / (2 * a.Hk));
    const bool is_v = hv >= a.Hk;
    const int row0 = a.rows ? mx_clamp(a.rows[b], 0, a.max_row) : 0, live = min(mx_clamp(a.counts ? a.counts[b] : a.n, 0, a.n), a.T - row0);
    const int nt = min(TOK, a.n - t0), nl = live - t0;  // tokens of this workgroup; those of them that are rows
    const long long head = (long long)b * a.Hk + h;
    const unsigned char *codes = (is_v ? v_codes : k_codes) + (head * a.T + row0) * (a.dh / 2);
    const unsigned char *scales = (is_v ? v_scales : k_scales) + head * (a.dh / 32) * a.T + row0 + t0;
    for (int i = tid; i < a.dh / 32 * TOK; i += 256)
      if (i % TOK < nl) sc[i / TOK][i % TOK] = scales[(long long)(i / TOK) * a.T + i % TOK];
    __syncthreads();
    T *dst = (is_v ? v : k) + ((long long)b * a.n * a.Hk + h) * a.dh;
    const int lpr = a.dh / 8;
    for (int i = tid; i < nt * lpr; i += 256) {
      const int t = i / lpr, c = i % lpr;
      mx_u4 w = {0, 0, 0, 0};
      if (t < nl) {
        const uint32_t code = *reinterpret_cast<const uint32_t *>(codes + (long long)(t0 + t) * (a.dh / 2) + c * 4);
        w = __builtin_bit_cast(mx_u4, mx_eight(code, (uint32_t)sc[c >> 2][t] << 23));
      }
      T *to = dst + (long long)(t0 + t) * a.Hk * a.dh + c * 8;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<mx_u4 *>(to) = w;
      } else {
        *reinterpret_cast<mx_f4 *>(to) = mx_f4{mx_lo(w[0]), mx_hi(w[0]), mx_lo(w[1]), mx_hi(w[1])};
        *reinterpret_cast<mx_f4 *>(to + 4) = mx_f4{mx_lo(w[2]), mx_hi(w[2]), mx_lo(w[3]), mx_hi(w[3])};
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Eviction, first launch: one workgroup per (sequence, head) picks the rows that stay.  A row's rank as an unsigned key: recent
// rows 0xffffffff, else the weight's bits turned so that they order as the numbers do, NaN 0.  The key of the last row that stays is
// found digit by digit (11 + 11 + 10 bits): a histogram in LDS of the rows that agree with the digits so far.  Rows
// above it stay, and of those that equal it the first.  One ordered sum over the rows then numbers the holes below `budget`
// and the kept rows beyond it.
// Out: kept rows in row order (`list`, budget entries, those from hole 0's counterpart on are the movers) and holes; counts.
// ---------------------------------------------------------------------------
constexpr int SEL = 1024, DIGIT = 11;
struct EvictArgs {
  long long heads;  // B * H_k
  int Hk, T, dh, max_len, budget, recent;
  const int *len;
  const float *weight;
  const int *pos;
  float *weight_out;  // weight_out, pos_out: as the inputs (in place) or elsewhere
  int *pos_out, *len_out;
  int *holes, *movers, *counts;  // (B * Hk, half), (B * Hk, half), (B * Hk, 2): number of moves, new length
  int half;                      // min(budget, T - budget): the most moves
};

__device__ __forceinline__ uint32_t rank_key(float w, int pos, int newest, int recent) {
  if ((long long)pos > (long long)newest - recent) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 counts as 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int block_max(int v, int *red) {
  for (int off = 32; off > 0; off >>= 1) v = max(v, __shfl_xor(v, off));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < SEL / 64; ++w) v = max(v, red[w]);
  __syncthreads();
  return v;
}

__global__ __launch_bounds__(SEL) void mx_select_kernel(EvictArgs a) {
  __shared__ int hist[1 << DIGIT];
  __shared__ int red[SEL / 64][2];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (long long head = blockIdx.x; head < a.heads; head += gridDim.x, __syncthreads()) {
  const int n = mx_clamp(a.len[head / a.Hk], 0, a.max_len);
  const float *w = a.weight + head * a.T;
  const int *p = a.pos + head * a.T;
  const bool apart = a.weight_out != a.weight || a.pos_out != a.pos;
  int *counts = a.counts + head * 2;
  if (n <= a.budget) {
    if (tid == 0) counts[0] = 0, counts[1] = n;
    if (apart)
      for (int i = tid; i < n; i += SEL) a.weight_out[head * a.T + i] = w[i], a.pos_out[head * a.T + i] = p[i];
    continue;
  }
  int newest = INT32_MIN;
  for (int i = tid; i < n; i += SEL) newest = max(newest, p[i]);
  newest = block_max(newest, &red[0][0]);
  // the budget-th largest key
  uint32_t prefix = 0, mask = 0;
  int want = a.budget;  // how many of the rows that agree with the prefix are still to be taken
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < (1 << DIGIT); i += SEL) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += SEL) {
      const uint32_t key = rank_key(w[i], p[i], newest, a.recent);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1u)], 1);
    }
    __syncthreads();
    // from the top: thread t holds two neighbouring bins; the first bin at which the sum reaches `want`
    const int hi = (1 << DIGIT) - 1 - 2 * tid, c1 = hist[hi], c0 = hist[hi - 1];
    int sum = c1 + c0;
    for (int off = 1; off < 64; off <<= 1) {
      const int up = __shfl_up(sum, off);
      if (lane >= off) sum += up;
    }
    if (lane == 63) red[wave][0] = sum;
    __syncthreads();
    int before = 0;
    for (int x = 0; x < wave; ++x) before += red[x][0];
    before += sum - (c1 + c0);
    if (before < want && before + c1 >= want) found[0] = hi, found[1] = before;
    else if (before + c1 < want && before + c1 + c0 >= want) found[0] = hi - 1, found[1] = before + c1;
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    mask |= ((1u << bits) - 1u) << shift;
    want -= found[1];
    __syncthreads();
  }
  // `want` rows of key `prefix` stay, the first ones.  Thread t takes rows t * per ...: rows above the key and rows that equal it
  // before its own, by one sum over the workgroup.
  const int per = (n + SEL - 1) / SEL, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  int above = 0, equal = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t key = rank_key(w[i], p[i], newest, a.recent);
    above += key > prefix;
    equal += key == prefix;
  }
  int sa = above, se = equal;
  for (int off = 1; off < 64; off <<= 1) {
    const int ua = __shfl_up(sa, off), ue = __shfl_up(se, off);
    if (lane >= off) sa += ua, se += ue;
  }
  if (lane == 63) red[wave][0] = sa, red[wave][1] = se;
  __syncthreads();
  for (int x = 0; x < wave; ++x) sa += red[x][0], se += red[x][1];
  sa -= above;
  se -= equal;
  int *holes = a.holes + head * a.half, *movers = a.movers + head * a.half;
  for (int i = i0; i < i1; ++i) {
    const float wi = w[i];
    const int pi = p[i];
    const uint32_t key = rank_key(wi, pi, newest, a.recent);
    const int kept = sa + min(se, want);  // rows before i that stay
    const bool keep = key > prefix || (key == prefix && se < want);
    if (i < a.budget) {
      if (!keep) holes[i - kept] = i;
      else if (apart) a.weight_out[head * a.T + i] = wi, a.pos_out[head * a.T + i] = pi;
    } else if (keep) {
      movers[a.budget - 1 - kept] = i;  // counted from the last kept row: the list is filled backwards
    }
    sa += key > prefix;
    se += key == prefix;
    if (i == a.budget - 1) counts[0] = a.budget - (kept + (keep ? 1 : 0)), counts[1] = a.budget;
  }
  }
}

// Second launch: hole h gets row movers[moves - 1 - h].  Sources lie at or beyond `budget`, targets below: no order is needed.  A
// workgroup takes 32 moves of a head: a wavefront the codes of 8, then a thread a scale byte, a weight, a position.
constexpr int MOVES = 32;
__global__ __launch_bounds__(256) void mx_move_kernel(EvictArgs a, unsigned char *__restrict__ k_codes, unsigned char *__restrict__ k_scales,
                                                     unsigned char *__restrict__ v_codes, unsigned char *__restrict__ v_scales) {
  const int tid = threadIdx.x, per = a.half > MOVES ? (a.half + MOVES - 1) / MOVES : 1;
  for (long long tile = blockIdx.x; tile < a.heads * per; tile += gridDim.x) {
  const long long head = tile / per;
  const int moves = a.counts[head * 2], m0 = (int)(tile % per) * MOVES;
  if (m0 == 0 && tid == 0 && head % a.Hk == 0) a.len_out[head / a.Hk] = a.counts[head * 2 + 1];
  if (m0 >= moves) continue;
  const int nm = min(MOVES, moves - m0), words = a.dh / 8, groups = a.dh / 32;
  const int *holes = a.holes + head * a.half + m0, *movers = a.movers + head * a.half + (moves - 1 - m0);
  const long long base = head * a.T;
  for (int i = tid; i < nm * words * 2; i += 256) {
    const int m = i / (2 * words), c = i % (2 * words);
    uint32_t *codes = reinterpret_cast<uint32_t *>(c < words ? k_codes : v_codes);
    const int x = c < words ? c : c - words;
    codes[(base + holes[m]) * words + x] = codes[(base + movers[-m]) * words + x];
  }
  for (int i = tid; i < nm * groups * 2; i += 256) {
    const int m = i % nm, g = i / nm;
    unsigned char *scales = (g < groups ? k_scales : v_scales) + (head * groups + (g < groups ? g : g - groups)) * a.T;
    scales[holes[m]] = scales[movers[-m]];
  }
  if (tid < nm) {
    const long long from = base + movers[-tid], to = base + holes[tid];
    a.weight_out[to] = a.weight[from];
    a.pos_out[to] = a.pos[from];
  }
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
constexpr long long MAX_GRID = 1 << 20;  // workgroups of a launch; they take the rest in turn
long long store_tiles(const Dims &d, int n) { return (long long)d.B * 2 * d.Hk * ((n + TOK - 1) / TOK); }

}  // namespace

hipError_t mx_store(const Dims &d, const cca_mx_cache &c, const void *k, const void *v, int n, const int *rows, int max_row,
                    const int *counts, const int *pos, hipStream_t s) {
  const StoreArgs a{n, d.Hk, d.dh, d.T, max_row, store_tiles(d, n), rows, counts, pos, reinterpret_cast<int *>(c.pos), c.weight};
  const unsigned grid = (unsigned)(a.tiles < MAX_GRID ? a.tiles : MAX_GRID);
  auto p = [](void *x) { return static_cast<unsigned char *>(x); };
  if (d.bf16) mx_store_kernel<bf16_t><<<grid, 256, 0, s>>>(a, (const bf16_t *)k, (const bf16_t *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  else mx_store_kernel<float><<<grid, 256, 0, s>>>(a, (const float *)k, (const float *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  return hipGetLastError();
}

hipError_t mx_rows(const Dims &d, const cca_mx_cache &c, void *k, void *v, int n, const int *first, const int *counts, hipStream_t s) {
  const StoreArgs a{n, d.Hk, d.dh, d.T, d.T, store_tiles(d, n), first, counts, nullptr, nullptr, nullptr};
  const unsigned grid = (unsigned)(a.tiles < MAX_GRID ? a.tiles : MAX_GRID);
  auto p = [](void *x) { return static_cast<const unsigned char *>(x); };
  if (d.bf16) mx_rows_kernel<bf16_t><<<grid, 256, 0, s>>>(a, (bf16_t *)k, (bf16_t *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  else mx_rows_kernel<float><<<grid, 256, 0, s>>>(a, (float *)k, (float *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  return hipGetLastError();
}

// The plan of an eviction: holes, movers, counts.  A budget leaves at most T / 2 moves.
size_t mx_evict_scratch_bytes(const Dims &d) {
  const size_t heads = (size_t)d.B * d.Hk;
  return 2 * align256(heads * ((size_t)d.T / 2) * sizeof(int)) + align256(heads * 2 * sizeof(int));
}

hipError_t mx_evict(const Dims &d, const cca_mx_cache &c, int *len, int max_len, int budget, int recent, float *weight_out, int *pos_out,
                    int *len_out, void *workspace, hipStream_t s) {
  const size_t heads = (size_t)d.B * d.Hk;
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  const size_t list = align256(heads * ((size_t)d.T / 2) * sizeof(int));
  const int half = budget < max_len - budget ? budget : max_len - budget;  // (max_len <= T: at most T / 2)
  EvictArgs a{(long long)heads, d.Hk, d.T, d.dh, max_len, budget, recent, len, c.weight, reinterpret_cast<const int *>(c.pos),
              weight_out ? weight_out : c.weight, pos_out ? pos_out : reinterpret_cast<int *>(c.pos), len_out ? len_out : len,
              reinterpret_cast<int *>(ws), reinterpret_cast<int *>(ws + list), reinterpret_cast<int *>(ws + 2 * list), half > 0 ? half : 0};
  mx_select_kernel<<<(unsigned)(a.heads < MAX_GRID ? a.heads : MAX_GRID), SEL, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long tiles = a.heads * (a.half > MOVES ? (a.half + MOVES - 1) / MOVES : 1);
  auto p = [](void *x) { return static_cast<unsigned char *>(x); };
  mx_move_kernel<<<(unsigned)(tiles < MAX_GRID ? tiles : MAX_GRID), 256, 0, s>>>(a, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  return hipGetLastError();
}

}  // namespace cca
