// Projections with 4-bit weights, for the few rows of a decode step: y (M, N) = x (M, K) W, and the quantisation of W.
#include "cca_mx.h"

namespace cca {

namespace {

constexpr int WAVES = 8;

struct ProjArgs {
  const unsigned char *codes, *scales;  // (N, K/2), (N, K/32)
  const void *x;
  void *y;
  RowDest dest;
  int M, K, N;
};

// x (8 numbers of a row from `at`) as TERMS parts in bf16
template <typename T, int TERMS>
__device__ __forceinline__ void load_x(const T *p, bool on, mx_bf8 (&f)[TERMS]) {
  if constexpr (TERMS == 1) {
    mx_u4 w = *reinterpret_cast<const mx_u4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = on ? w[i] : 0u;
    f[0] = __builtin_bit_cast(mx_bf8, w);
  } else {
    const mx_f4 a = *reinterpret_cast<const mx_f4 *>(p), b = *reinterpret_cast<const mx_f4 *>(p + 4);
    float r[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = on ? r[i] : 0.f;
#pragma unroll
    for (int u = 0; u < TERMS; ++u) {
      mx_u4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t wi = mx_pack(r[2 * i], r[2 * i + 1]);
        w[i] = wi;
        r[2 * i] -= mx_lo(wi), r[2 * i + 1] -= mx_hi(wi);
      }
      f[u] = __builtin_bit_cast(mx_bf8, w);
    }
  }
}

// ---------------------------------------------------------------------------
// Workgroup = 16 columns x 16 MT rows, its eight wavefronts share K.  Lane (m, j) takes 32 numbers of column m (16 bytes, one
// scale) per 128 of K; four products of 16 x 16 x 32.
// ---------------------------------------------------------------------------
template <typename T, typename TO, int MT>
__global__ __launch_bounds__(WAVES * 64) void mx_project_kernel(ProjArgs a) {
  constexpr int TERMS = sizeof(T) == 4 ? 3 : 1;
  __shared__ float red[WAVES][MT][16][17];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, j = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT, col = min(n0 + m, a.N - 1), groups = a.K / 32;
  const unsigned char *codes = a.codes + (long long)col * (a.K / 2), *scales = a.scales + (long long)col * groups;
  const T *x = static_cast<const T *>(a.x);
  mx_f4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = mx_f4{0.f, 0.f, 0.f, 0.f};
  const int steps = (groups + 3) / 4, per = (steps + WAVES - 1) / WAVES, s1 = min(steps, (wave + 1) * per);
  for (int st = wave * per; st < s1; ++st) {
    const int g = st * 4 + j, gc = min(g, groups - 1);
    const bool on = g < groups;
    const mx_u4 w = *reinterpret_cast<const mx_u4 *>(codes + gc * 16);
    const uint32_t sc = on ? (uint32_t)scales[gc] << 23 : 0u;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const mx_bf8 wf = mx_eight(w[s], sc);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        mx_bf8 xf[TERMS];
        load_x<T, TERMS>(x + (long long)min(m0 + 16 * t + m, a.M - 1) * a.K + gc * 32 + 8 * s, on, xf);
#pragma unroll
        for (int u = 0; u < TERMS; ++u) acc[t] = mx_mfma(wf, xf[u], acc[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave][t][m][4 * j + i] = acc[t][i];
  __syncthreads();
  for (int i = tid; i < MT * 256; i += WAVES * 64) {
    const int t = i / 256, r = i / 16 % 16, c = i % 16;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += red[w][t][r][c];
    const int row = m0 + 16 * t + r;
    if (row < a.M && n0 + c < a.N) store_f(static_cast<TO *>(a.y) + a.dest.at(row, a.N) + n0 + c, sum);
  }
}

// W (K, N) -> codes, scales: a thread per (column, group), columns along the threads
template <typename T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ w, int K, int N, unsigned char *__restrict__ codes,
                                                         unsigned char *__restrict__ scales) {
  const int n = blockIdx.x * 256 + threadIdx.x, g = blockIdx.y;
  if (n >= N) return;
  const T *p = w + (long long)g * 32 * N + n;
  float x[4][8], amax = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    x[i / 8][i % 8] = load_f(p + (long long)i * N);
    amax = mx_max_abs(amax, x[i / 8][i % 8]);
  }
  const uint32_t s = mx_scale_of(amax);
  mx_u4 c;
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = mx_codes(x[i], s);
  *reinterpret_cast<mx_u4 *>(codes + (long long)n * (K / 2) + g * 16) = c;
  scales[(long long)n * (K / 32) + g] = (unsigned char)s;
}

template <typename T, typename TO>
hipError_t launch(const ProjArgs &a, hipStream_t s) {
  const unsigned cols = (a.N + 15) / 16;
  if (a.M <= 16) mx_project_kernel<T, TO, 1><<<dim3(cols, 1), WAVES * 64, 0, s>>>(a);
  else mx_project_kernel<T, TO, 2><<<dim3(cols, (a.M + 31) / 32), WAVES * 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t mx_project(bool bf16, const void *x, const cca_mx_weight &w, void *y, bool y_f32, const RowDest &dest, int M, int K, int N,
                      hipStream_t s) {
  const ProjArgs a{static_cast<const unsigned char *>(w.codes), static_cast<const unsigned char *>(w.scales), x, y, dest, M, K, N};
  if (!bf16) return launch<float, float>(a, s);
  return y_f32 ? launch<bf16_t, float>(a, s) : launch<bf16_t, bf16_t>(a, s);
}

hipError_t mx_quantize(bool bf16, const void *w, int K, int N, void *codes, void *scales, hipStream_t s) {
  const dim3 grid((N + 255) / 256, K / 32);
  if (bf16) mx_quantize_kernel<bf16_t><<<grid, 256, 0, s>>>((const bf16_t *)w, K, N, (unsigned char *)codes, (unsigned char *)scales);
  else mx_quantize_kernel<float><<<grid, 256, 0, s>>>((const float *)w, K, N, (unsigned char *)codes, (unsigned char *)scales);
  return hipGetLastError();
}

}  // namespace cca
