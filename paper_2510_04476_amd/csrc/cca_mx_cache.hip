// The latent cache in 4 bits: rows stored, read back, and evicted by accumulated attention weight (include/cca.h).
#include <type_traits>

#include "cca_mx.h"

namespace cca {

namespace {

constexpr int TOK = 64;  // tokens of a workgroup

// ---------------------------------------------------------------------------
// Store: one workgroup per (64 tokens, head, sequence) and K or V.  A lane takes 8 numbers (16 or 32 bytes), four lanes a group:
// its largest magnitude over them by two lane exchanges, then 4 conversions of two numbers each.  Bound by what it moves (read 2
// or 4 bytes a number, write 17 / 32).  The scale bytes of a token lie T bytes apart, those of neighbouring tokens
// side by side: they go through LDS so that a wavefront stores them along the tokens.  1 x 16384 tokens, 2 heads of 128, bf16: 6.5 us, 3.3
// TB/s; 32 x 1 token: 3.5 us, a launch and one latency.
// ---------------------------------------------------------------------------
struct StoreArgs {
  int n, Hk, T;
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

// Where a workgroup's 64 tokens lie
struct Tile {
  int t0, b, row0, live;  // first token; sequence; its first row and how many of its n tokens are rows
  long long head;
  bool is_v;
};
__device__ __forceinline__ Tile tile_of(const StoreArgs &a, long long tile) {
  const int per = (a.n + TOK - 1) / TOK;
  Tile t;
  const int hv = (int)(tile / per % (2 * a.Hk));
  t.t0 = (int)(tile % per) * TOK;
  t.b = (int)(tile / per / (2 * a.Hk));
  t.is_v = hv >= a.Hk;
  t.head = (long long)t.b * a.Hk + hv % a.Hk;
  t.row0 = a.rows ? mx_clamp(a.rows[t.b], 0, a.T) : 0;
  t.live = min(mx_clamp(a.counts ? a.counts[t.b] : a.n, 0, a.n), a.T - t.row0);
  return t;
}

// (16-byte pieces of the 64 tokens: N32 = d_h / 32 to a thread, all requested before the first is used)
template <typename T, int N32>
__global__ __launch_bounds__(256) void mx_store_kernel(StoreArgs a, const T *__restrict__ k, const T *__restrict__ v,
                                                      unsigned char *__restrict__ k_codes, unsigned char *__restrict__ k_scales,
                                                      unsigned char *__restrict__ v_codes, unsigned char *__restrict__ v_scales) {
  constexpr int DH = 32 * N32, LPR = DH / 8;
  __shared__ unsigned char sc[N32][TOK];
  const int tid = threadIdx.x;
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, __syncthreads()) {
    const Tile t = tile_of(a, tile);
    const int nt = min(TOK, t.live - t.t0), h = (int)(t.head % a.Hk);
    if (nt <= 0) continue;
    const T *src = (t.is_v ? v : k) + (((long long)t.b * a.n + t.t0) * a.Hk + h) * DH;
    unsigned char *codes = (t.is_v ? v_codes : k_codes) + (t.head * a.T + t.row0 + t.t0) * (DH / 2);
    float x[N32][8];
#pragma unroll
    for (int u = 0; u < N32; ++u) {
      const int i = u * 256 + tid, tok = min(i / LPR, nt - 1), c = i % LPR;  // tokens past the last repeat it; nobody stores them
      load8(src + (long long)tok * a.Hk * DH + c * 8, x[u]);
    }
#pragma unroll
    for (int u = 0; u < N32; ++u) {
      const int i = u * 256 + tid, tok = i / LPR, c = i % LPR;
      const uint32_t s = group_scale(x[u]);  // (four lanes of one token)
      if (tok >= nt) continue;
      *reinterpret_cast<uint32_t *>(codes + tok * (DH / 2) + c * 4) = mx_codes(x[u], s);
      if ((c & 3) == 0) sc[c >> 2][tok] = (unsigned char)s;
    }
    __syncthreads();
    unsigned char *scales = (t.is_v ? v_scales : k_scales) + t.head * N32 * a.T + t.row0 + t.t0;
#pragma unroll
    for (int i = tid; i < N32 * TOK; i += 256)
      if (i % TOK < nt) scales[(long long)(i / TOK) * a.T + i % TOK] = sc[i / TOK][i % TOK];
    if (!t.is_v && tid < nt) {
      const long long at = t.head * a.T + t.row0 + t.t0 + tid;
      if (a.row_pos) a.row_pos[at] = (a.pos ? a.pos[t.b] : t.row0) + t.t0 + tid;
      if (a.weight) a.weight[at] = 0.f;
    }
  }
}

// Read back: the same workgroups the other way round.  1 x 16384 tokens, 2 heads of 128, bf16: 6.3 us; 16 x 4096: 14.6 us, 5.8 TB/s.
template <typename T, int N32>
__global__ __launch_bounds__(256) void mx_rows_kernel(StoreArgs a, T *__restrict__ k, T *__restrict__ v,
                                                     const unsigned char *__restrict__ k_codes, const unsigned char *__restrict__ k_scales,
                                                     const unsigned char *__restrict__ v_codes, const unsigned char *__restrict__ v_scales) {
  constexpr int DH = 32 * N32, LPR = DH / 8;
  __shared__ unsigned char sc[N32][TOK];
  const int tid = threadIdx.x;
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, __syncthreads()) {
    const Tile t = tile_of(a, tile);
    const int nt = min(TOK, a.n - t.t0), nl = t.live - t.t0, h = (int)(t.head % a.Hk);  // tokens of this workgroup; those of them that are rows
    uint32_t code[N32];
    if (nl > 0) {
      const unsigned char *codes = (t.is_v ? v_codes : k_codes) + (t.head * a.T + t.row0 + t.t0) * (DH / 2);
      const unsigned char *scales = (t.is_v ? v_scales : k_scales) + t.head * N32 * a.T + t.row0 + t.t0;
#pragma unroll
      for (int u = 0; u < N32; ++u) {
        const int i = u * 256 + tid;
        code[u] = *reinterpret_cast<const uint32_t *>(codes + min(i / LPR, nl - 1) * (DH / 2) + i % LPR * 4);
      }
#pragma unroll
      for (int i = tid; i < N32 * TOK; i += 256) sc[i / TOK][i % TOK] = scales[(long long)(i / TOK) * a.T + min(i % TOK, nl - 1)];
    }
    __syncthreads();
    T *dst = (t.is_v ? v : k) + (((long long)t.b * a.n + t.t0) * a.Hk + h) * DH;
#pragma unroll
    for (int u = 0; u < N32; ++u) {
      const int i = u * 256 + tid, tok = i / LPR, c = i % LPR;
      if (tok >= nt) continue;
      mx_u4 w = {0, 0, 0, 0};
      if (tok < nl) w = __builtin_bit_cast(mx_u4, mx_eight(code[u], (uint32_t)sc[c >> 2][tok] << 23));
      T *to = dst + (long long)tok * a.Hk * DH + c * 8;
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
// found digit by digit (11 + 11 + 10 bits): a histogram in LDS of the rows that agree with the digits so far, two copies side by
// side (neighbouring lanes hold similar weights: one copy has them queue for the same words).  Rows above that key stay, and of
// those that equal it the first.  Then each wavefront counts both kinds in its own stretch of rows and, behind one sum over the
// wavefronts, numbers the holes below `budget` and the kept rows beyond it.
// HELD: the keys lie in LDS, so that weights and positions are read once; longer heads are read again by every pass.
// Bound by one workgroup's chain - three digits with three barriers each, a pass before and two behind - and, on long heads, by its vector
// instructions: 256 rows 8.8 us, 1024 9.1, 4608 12.5, 16000 16.3, 32000 21.8, 60000 (read again) 52.7.
// ---------------------------------------------------------------------------
constexpr int SEL = 1024, DIGIT = 11, COPIES = 2;
constexpr int HELD_ROWS = 32768;  // 128 KB of keys beside 16 KB of histogram
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
typedef int mx_i4 __attribute__((ext_vector_type(4)));

// (no position exceeds the newest one: their difference fits 32 bits)
__device__ __forceinline__ uint32_t rank_key(float w, int pos, int newest, int recent) {
  const uint32_t u = __float_as_uint(w + 0.f), k = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);  // -0 counts as 0
  return (uint32_t)newest - (uint32_t)pos < (uint32_t)recent ? 0xffffffffu : w != w ? 0u : k;
}
// Sum over the lanes up to this one: shifts inside each row of 16 lanes, then the rows' last sums handed on
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8 (zero from before the row)
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31 into rows 2 and 3
  return x;
}
template <bool HELD>
__global__ __launch_bounds__(SEL) void mx_select_kernel(EvictArgs a) {
  extern __shared__ __attribute__((aligned(16))) int sel_lds[];
  int *const hist = sel_lds;                                                        // [bin][copy]
  uint32_t *const keys = reinterpret_cast<uint32_t *>(sel_lds + (COPIES << DIGIT));  // HELD: of every row
  __shared__ int red[SEL / 64][2], found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (long long head = blockIdx.x; head < a.heads; head += gridDim.x, __syncthreads()) {
    const float *const w = a.weight + head * a.T;
    const int *const p = a.pos + head * a.T;
    const bool apart = a.weight_out != a.weight || a.pos_out != a.pos;
    float *const wo = a.weight_out + head * a.T;
    int *const po = a.pos_out + head * a.T;
    const int n = mx_clamp(a.len[head / a.Hk], 0, a.max_len);
    if (tid == 0) a.counts[head * 2 + 1] = min(n, a.budget);
    if (n <= a.budget) {
      if (tid == 0) a.counts[head * 2] = 0;
      if (apart)
        for (int i = tid; i < n; i += SEL) wo[i] = w[i], po[i] = p[i];
      continue;
    }
    // Rows four at a time, several groups requested together; the capacity is a multiple of 32, so a group that begins below n is inside it.
    // Lanes past the end repeat the last group.  (Loops stay rolled: a launch runs them a few times, and code that it has to fetch first
    // costs more than the iterations.  With the rows of 8 iterations unrolled into registers: 4608 and 30011 rows 17.6 and 38.6 us.)
    const int last = (n - 1) & ~3;
    auto request = [&](const auto *from, int r0, auto (&to)[4]) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 4; ++u) to[u] = *reinterpret_cast<const std::remove_reference_t<decltype(to[0])> *>(from + min(r0 + 4 * SEL * u, last));
    };
    mx_f4 wv[4];
    if constexpr (HELD) request(w, 4 * tid, wv);  // the first weights beside the positions, which wait in LDS
    int newest = INT32_MIN;
#pragma unroll 1
    for (int r0 = 4 * tid; r0 < n; r0 += 32 * SEL) {
      mx_i4 pv[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) pv[u] = *reinterpret_cast<const mx_i4 *>(p + min(r0 + 4 * SEL * u, last));
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int row = r0 + 4 * SEL * u;
        if (HELD && row < n) *reinterpret_cast<mx_i4 *>(keys + row) = pv[u];
#pragma unroll
        for (int e = 0; e < 4; ++e) newest = row + e < n ? max(newest, pv[u][e]) : newest;
      }
    }
    for (int off = 32; off > 0; off >>= 1) newest = max(newest, __shfl_xor(newest, off));
    if (lane == 0) red[wave][0] = newest;
    for (int i = tid; i < (COPIES << DIGIT) / 4; i += SEL) reinterpret_cast<mx_i4 *>(hist)[i] = mx_i4{0, 0, 0, 0};
    __syncthreads();
#pragma unroll
    for (int x = 0; x < SEL / 64; ++x) newest = max(newest, red[x][0]);
    // keys of rows `row` ... `row` + 3; those from n on have the lowest, and are the last of it: they never stay
    auto keys_of = [&](int row, mx_f4 wv, mx_i4 pv) __attribute__((always_inline)) {
      mx_u4 k;
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = rank_key(wv[e], pv[e], newest, a.recent);
      if (row + 4 > n) {
#pragma unroll
        for (int e = 1; e < 4; ++e) k[e] = row + e < n ? k[e] : 0u;
      }
      return k;
    };
    uint32_t prefix = 0, mask = 0;
    int want = a.budget;  // how many of the rows that agree with the prefix are still to be taken
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t bins = pass == 2 ? 1023u : 2047u;
      auto count = [&](uint32_t k) __attribute__((always_inline)) {
        if ((k & mask) == prefix) atomicAdd(&hist[((k >> shift) & bins) * COPIES + (lane & (COPIES - 1))], 1);
      };
      if (HELD && pass > 0) {
#pragma unroll 1
        for (int r = 4 * tid; r < n; r += 4 * SEL) {
          const mx_u4 k = *reinterpret_cast<const mx_u4 *>(keys + r);
#pragma unroll
          for (int e = 0; e < 4; ++e) count(k[e]);
        }
      } else {
#pragma unroll 1
        for (int r0 = 4 * tid; r0 < n; r0 += 16 * SEL) {
          mx_f4 next[4];
          mx_i4 pv[4];
          if constexpr (HELD) {
            request(w, r0 + 16 * SEL, next);
          } else {
            request(w, r0, wv);
            request(p, r0, pv);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int row = r0 + 4 * SEL * u;
            if (row >= n) continue;
            if constexpr (HELD) pv[u] = *reinterpret_cast<const mx_i4 *>(keys + row);
            const mx_u4 k = keys_of(row, wv[u], pv[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) count(k[e]);
            if constexpr (HELD) *reinterpret_cast<mx_u4 *>(keys + row) = k;
          }
          if constexpr (HELD)
#pragma unroll
            for (int u = 0; u < 4; ++u) wv[u] = next[u];
        }
      }
      __syncthreads();
      // from the top: thread t holds two neighbouring bins, which it clears; the first bin at which the sum reaches `want`
      const int hi = (1 << DIGIT) - 1 - 2 * tid;
      int c[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        int2 *const h = reinterpret_cast<int2 *>(hist) + (hi - x);
        const int2 v = *h;
        *h = make_int2(0, 0);
        c[x] = v.x + v.y;
      }
      const int sum = wave_scan(c[0] + c[1]);
      if (lane == 63) red[wave][1] = sum;
      __syncthreads();
      int before = sum - c[0] - c[1];
#pragma unroll
      for (int x = 0; x < SEL / 64; ++x) before += x < wave ? red[x][1] : 0;
      if (before < want && before + c[0] >= want) found[0] = hi, found[1] = before, found[2] = c[0];
      else if (before + c[0] < want && before + c[0] + c[1] >= want) found[0] = hi - 1, found[1] = before + c[0], found[2] = c[1];
      __syncthreads();
      prefix |= (uint32_t)found[0] << shift;
      mask |= bins << shift;
      want -= found[1];
      // (`found` and `red` are written again behind the next pass's barriers)
    }
    // Rows above `thr` stay.  With more rows of key `prefix` than `want`, of those the first; else they count as above.  (All n > budget rows
    // cannot be above: without ties prefix > 0.)
    const bool ties = found[2] > want;
    const uint32_t thr = ties ? prefix : prefix - 1;
    // A wavefront's stretch: whole lines of 256 rows
    const int stretch = ((n + SEL / 64 - 1) / (SEL / 64) + 255) / 256 * 256, r0 = wave * stretch, r1 = min(n, r0 + stretch);
    auto keys_at = [&](int row) __attribute__((always_inline)) {
      if (row >= n) return mx_u4{0u, 0u, 0u, 0u};
      if constexpr (HELD) return *reinterpret_cast<const mx_u4 *>(keys + row);
      else return keys_of(row, *reinterpret_cast<const mx_f4 *>(w + row), *reinterpret_cast<const mx_i4 *>(p + row));
    };
    int above = 0, equal = 0;
#pragma unroll 1
    for (int r = r0; r < r1; r += 256) {
      const mx_u4 k = keys_at(r + 4 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        above += __popcll(__ballot(k[e] > thr));
        if (ties) equal += __popcll(__ballot(k[e] == prefix));
      }
    }
    if (lane == 0) red[wave][0] = above, red[wave][1] = equal;
    __syncthreads();
    above = equal = 0;  // before this wavefront's rows
#pragma unroll
    for (int x = 0; x < SEL / 64; ++x) above += x < wave ? red[x][0] : 0, equal += x < wave ? red[x][1] : 0;
    int *const holes = a.holes + head * a.half, *const movers = a.movers + head * a.half;  // (movers: counted from the last kept row, filled backwards)
#pragma unroll 1
    for (int r = r0; r < r1; r += 256) {
      const int row = r + 4 * lane;
      const mx_u4 k = keys_at(row);
      int mine = 0;  // above | equal << 16
#pragma unroll
      for (int e = 0; e < 4; ++e) mine += k[e] > thr ? 1 : 0;
      if (ties) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += k[e] == prefix ? 1 << 16 : 0;
      }
      const int upto = wave_scan(mine), all = __builtin_amdgcn_readlane(upto, 63);
      int sa = above + ((upto - mine) & 0xffff), se = equal + ((upto - mine) >> 16);  // rows before this lane's
      above += all & 0xffff;
      equal += all >> 16;
      if (!ties && r >= a.budget) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k[e] > thr) movers[(uint32_t)(a.budget - 1 - sa++)] = row + e;
      } else if (!ties && r + 256 < a.budget) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (k[e] <= thr) holes[(uint32_t)(row + e - sa)] = row + e;
          else ++sa;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = row + e, kept = sa + min(se, want);  // rows before i that stay
          const bool is_above = k[e] > thr, is_equal = ties && k[e] == prefix, keep = is_above || (is_equal && se < want);
          if (i < a.budget) {
            if (!keep) holes[i - kept] = i;
          } else if (keep && i < n) {
            movers[a.budget - 1 - kept] = i;
          }
          if (i == a.budget - 1) a.counts[head * 2] = a.budget - (kept + (keep ? 1 : 0));
          sa += is_above;
          se += is_equal;
        }
      }
    }
    // Elsewhere the rows below `budget` go as they are, the holes too: the second launch fills those.  (In a loop of its own: with these loads
    // in the one above, each of its turns waited for the last one's stores, which took 9 of 24 us on 32000 rows.)
    if (apart) {
#pragma unroll 4
      for (int row = 4 * tid; row < a.budget; row += 4 * SEL) {
        const mx_f4 wv = *reinterpret_cast<const mx_f4 *>(w + row);
        const mx_i4 pv = *reinterpret_cast<const mx_i4 *>(p + row);
        if (row + 4 <= a.budget) {
          *reinterpret_cast<mx_f4 *>(wo + row) = wv;
          *reinterpret_cast<mx_i4 *>(po + row) = pv;
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (row + e < a.budget) wo[row + e] = wv[e], po[row + e] = pv[e];
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Second launch: hole m gets row movers[moves - 1 - m].  Sources lie at or beyond `budget`, targets below: no order is needed.  A
// workgroup takes 32 moves of a head: a word of codes, then a scale byte, a weight and a position to a thread in turn.  (Moved by the
// workgroup that picked them, 512 of dh = 128 and 3300 of 64 took 8 and 31 us more; this launch takes 4.5 and 5.8.)
// ---------------------------------------------------------------------------
struct Cache {
  unsigned char *k_codes, *k_scales, *v_codes, *v_scales;
};
constexpr int PART = 32;
__global__ __launch_bounds__(256) void mx_move_kernel(EvictArgs a, Cache c) {
  const int tid = threadIdx.x, per = a.half > PART ? (a.half + PART - 1) / PART : 1;
  const int words = a.dh / 8, groups = a.dh / 32;  // words of a row's codes; scale bytes
  __shared__ int from[PART], to[PART];
  for (long long tile = blockIdx.x; tile < a.heads * per; tile += gridDim.x, __syncthreads()) {
    const long long head = tile / per, base = head * a.T;
    const int moves = a.counts[head * 2], m0 = (int)(tile % per) * PART, nm = min(PART, moves - m0);
    if (m0 == 0 && tid == 0 && head % a.Hk == 0) a.len_out[head / a.Hk] = a.counts[head * 2 + 1];
    if (nm <= 0) continue;
    if (tid < nm) {
      const int f = a.movers[head * a.half + moves - 1 - m0 - tid], t = a.holes[head * a.half + m0 + tid];
      from[tid] = f, to[tid] = t;
      a.weight_out[base + t] = a.weight[base + f];
      a.pos_out[base + t] = a.pos[base + f];
    }
    __syncthreads();
    // eight threads to a row's codes of K and of V each
    const int m = tid >> 3;
    if (m < nm) {
      const long long f = (base + from[m]) * words, t = (base + to[m]) * words;
#pragma unroll 4
      for (int x = tid & 7; x < words; x += 8) {
        const uint32_t k = reinterpret_cast<const uint32_t *>(c.k_codes)[f + x], v = reinterpret_cast<const uint32_t *>(c.v_codes)[f + x];
        reinterpret_cast<uint32_t *>(c.k_codes)[t + x] = k;
        reinterpret_cast<uint32_t *>(c.v_codes)[t + x] = v;
      }
      // and to its scale bytes, T bytes apart
      if ((tid & 7) < groups) {
        const long long at = (head * groups + (tid & 7)) * a.T;
        const unsigned char k = c.k_scales[at + from[m]], v = c.v_scales[at + from[m]];
        c.k_scales[at + to[m]] = k;
        c.v_scales[at + to[m]] = v;
      }
    }
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
constexpr long long MAX_GRID = 1 << 20;  // workgroups of a launch; they take the rest in turn
long long store_tiles(const Dims &d, int n) { return (long long)d.B * 2 * d.Hk * ((n + TOK - 1) / TOK); }

}  // namespace

// f(integral constant of d_h / 32)
template <typename F>
static hipError_t by_width(int dh, F f) {
  switch (dh / 32) {
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    case 5: f(std::integral_constant<int, 5>{}); break;
    case 6: f(std::integral_constant<int, 6>{}); break;
    case 7: f(std::integral_constant<int, 7>{}); break;
    default: f(std::integral_constant<int, 8>{}); break;
  }
  return hipGetLastError();
}

hipError_t mx_store(const Dims &d, const cca_mx_cache &c, const void *k, const void *v, int n, const int *rows, const int *counts,
                    const int *pos, hipStream_t s) {
  const StoreArgs a{n, d.Hk, d.T, store_tiles(d, n), rows, counts, pos, reinterpret_cast<int *>(c.pos), c.weight};
  const unsigned grid = (unsigned)(a.tiles < MAX_GRID ? a.tiles : MAX_GRID);
  auto p = [](void *x) { return static_cast<unsigned char *>(x); };
  return by_width(d.dh, [&](auto w) {
    constexpr int N32 = decltype(w)::value;
    if (d.bf16) mx_store_kernel<bf16_t, N32><<<grid, 256, 0, s>>>(a, (const bf16_t *)k, (const bf16_t *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
    else mx_store_kernel<float, N32><<<grid, 256, 0, s>>>(a, (const float *)k, (const float *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  });
}

hipError_t mx_rows(const Dims &d, const cca_mx_cache &c, void *k, void *v, int n, const int *first, const int *counts, hipStream_t s) {
  const StoreArgs a{n, d.Hk, d.T, store_tiles(d, n), first, counts, nullptr, nullptr, nullptr};
  const unsigned grid = (unsigned)(a.tiles < MAX_GRID ? a.tiles : MAX_GRID);
  auto p = [](void *x) { return static_cast<const unsigned char *>(x); };
  return by_width(d.dh, [&](auto w) {
    constexpr int N32 = decltype(w)::value;
    if (d.bf16) mx_rows_kernel<bf16_t, N32><<<grid, 256, 0, s>>>(a, (bf16_t *)k, (bf16_t *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
    else mx_rows_kernel<float, N32><<<grid, 256, 0, s>>>(a, (float *)k, (float *)v, p(c.k_codes), p(c.k_scales), p(c.v_codes), p(c.v_scales));
  });
}

// The plan of an eviction: holes, movers (a budget leaves at most T / 2 moves), counts.
size_t mx_evict_scratch_bytes(const Dims &d) {
  const size_t heads = (size_t)d.B * d.Hk;
  return 2 * align256(heads * ((size_t)d.T / 2) * sizeof(int)) + align256(heads * 2 * sizeof(int));
}

hipError_t mx_evict(const Dims &d, const cca_mx_cache &cache, int *len, int max_len, int budget, int recent, float *weight_out, int *pos_out,
                    int *len_out, void *workspace, hipStream_t s) {
  const size_t heads = (size_t)d.B * d.Hk, list = align256(heads * ((size_t)d.T / 2) * sizeof(int));
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  auto ints = [](unsigned char *p) { return reinterpret_cast<int *>(p); };
  auto bytes = [](void *p) { return static_cast<unsigned char *>(p); };
  int *const pos = reinterpret_cast<int *>(cache.pos);
  const int most = budget < max_len - budget ? budget : max_len - budget;  // (max_len <= T: at most T / 2)
  const EvictArgs a{(long long)heads, d.Hk, d.T, d.dh, max_len, budget, recent, len, cache.weight, pos, weight_out ? weight_out : cache.weight,
                    pos_out ? pos_out : pos, len_out ? len_out : len, ints(ws), ints(ws + list), ints(ws + 2 * list), most > 0 ? most : 0};
  const unsigned grid = (unsigned)(a.heads < MAX_GRID ? a.heads : MAX_GRID);
  constexpr size_t HIST = (size_t)(COPIES << DIGIT) * 4;
  hipError_t e;
  if (max_len <= HELD_ROWS) {
    if ((e = raise_lds_limit<mx_select_kernel<true>>(HIST + (size_t)HELD_ROWS * 4)) != hipSuccess) return e;
    mx_select_kernel<true><<<grid, SEL, HIST + (size_t)(max_len + 3) / 4 * 16, s>>>(a);
  } else {
    mx_select_kernel<false><<<grid, SEL, HIST, s>>>(a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const long long tiles = a.heads * (a.half > PART ? (a.half + PART - 1) / PART : 1);
  mx_move_kernel<<<(unsigned)(tiles < MAX_GRID ? tiles : MAX_GRID), 256, 0, s>>>(
      a, Cache{bytes(cache.k_codes), bytes(cache.k_scales), bytes(cache.v_codes), bytes(cache.v_scales)});
  return hipGetLastError();
}

}  // namespace cca
