// The residual's addition and the root-mean-square norm in front of a sublayer's projections, with results in 32, 16 or 8 bits.
#include <math.h>

#include "mdbf_rows.h"

namespace mdbf {

constexpr int kNormMaxChannels = 65536;
// Results beyond this are stored past the caches: 8192 rows of 4096 bf16 channels with the new stream (134 MB) 39.0 us instead of 41.1, 16384 75.5 instead of
// 94.3, with a read of y behind them 52.3 and 52.0, 99.6 and 112.6; of 256 rows (4 MB) 4.2 and 4.3, 7.0 and 7.0.  (Between 8 and 32 MB it would gain
// too, 16 MB 5.1 us instead of 7.3: the border is that of the attention block's results.)
constexpr int64_t kNormStreamBytes = 32ll << 20;

struct NormArgs {
  const void *x, *res;
  const float* weight;
  void *res_out, *y, *scales;
  int64_t ldx, ldr, ldro, ldy, lds, t0;           // t0: the launch's first row
  int32_t T, n, yd, group;
  float eps;
};

// Sum resp. largest over the lanes of a row: a wave, or all of the workgroup's waves.
template <int WAVES>
__device__ __forceinline__ double row_sum(double v, double* part) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  if (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += part[w];
  }
  return v;
}
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* part) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  if (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = max(v, part[w]);
  }
  return v;
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

template <bool STREAM>
__device__ __forceinline__ void store_codes8(void* base, int64_t at, int count, const float (&x)[8]) {
  typedef U32x2 __attribute__((aligned(1))) U32x2u;
  const U32x2 v = {codes4(x[0], x[1], x[2], x[3]), codes4(x[4], x[5], x[6], x[7])};
  MDBF_GLOBAL uint8_t* p = (MDBF_GLOBAL uint8_t*)base + at;
  if (count >= 8) {
    if (STREAM) __builtin_nontemporal_store(v, (MDBF_GLOBAL U32x2u*)p);
    else *(MDBF_GLOBAL U32x2u*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = (uint8_t)(v[i / 4] >> (8 * (i % 4)));
  }
}

// h = x + residual, y = h / sqrt(mean h^2 + eps) * w: rows are read once and stay in registers, eight channels a lane and piece, WAVES waves
// a row (workgroups of four waves where a row takes one).  (Beyond 16384 channels sixteen waves have eight pieces and 128 registers each: with a residual 24
// to 51 of them lie in scratch memory.)  The squares are exact in fp64 and so in effect is their sum, whatever its
// order: what is rounded to 8 bits afterwards, and the scales, do not go by the shape of the launch; beside the loads that costs nothing.
// Bound by HBM where it is large: 8192 rows of 4096 bf16 channels with residual into e4m3 with a scale byte per 32 (236 MB) 37.8 us, 6.2
// TB/s, more than a copy's 4.9 because more is read than written; 64 rows are the latency of a launch, its loads and one meeting of the
// waves, 4.2 us.  HD: the stream's type, -1 without residual.
template <int XD, int HD, int WAVES, int VPT, bool STREAM>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void norm_kernel(NormArgs a) {
  constexpr int HT = HD < 0 ? XD : HD, ROWS = WAVES >= 4 ? 1 : 4 / WAVES, LANES = WAVES * 64;
  __shared__ double sums[WAVES];
  __shared__ uint32_t tops[WAVES];
  const int lane = threadIdx.x & (LANES - 1);
  const int64_t t = a.t0 + (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / LANES : 0);
  if (t >= a.T) return;                     // (rows of one wave only: no barrier follows there)

  Raw8<XD> rx[VPT];
  Raw8<HT> rr[VPT];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int c = (v * LANES + lane) * 8;
    if (c < a.n) {
      load_raw8<XD>(a.x, t * a.ldx + c, a.n - c, rx[v]);
      if (HD >= 0) load_raw8<HT>(a.res, t * a.ldr + c, a.n - c, rr[v]);
    }
  }
  float h[VPT][8];
  double sum = 0;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int c = (v * LANES + lane) * 8;
    if (c < a.n) {
      to_float8<XD>(rx[v], h[v]);
      if (HD >= 0) {
        float r[8];
        to_float8<HT>(rr[v], r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] += r[i];
        if (a.res_out) store_float8<HT, STREAM>(a.res_out, t * a.ldro + c, a.n - c, h[v]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)h[v][i], (double)h[v][i], sum);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = 0.0f;
    }
  }
  sum = row_sum<WAVES>(sum, sums);
  const float r = (float)(1.0 / sqrt(sum / a.n + (double)a.eps));

  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int c = (v * LANES + lane) * 8;
    if (c >= a.n) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[v][i] *= r;
    if (a.weight) {
      Raw8<MDBF_F32> rw;
      float w[8];
      load_raw8<MDBF_F32>(a.weight, c, a.n - c, rw);
      to_float8<MDBF_F32>(rw, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] *= w[i];
    }
    if (a.yd == MDBF_E4M3) {               // a NaN's bits are the largest
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, h[v][i]) & 0x7fffffffu);
    }
  }
  if (a.yd == MDBF_E4M3 && a.group == 0) {
    top = row_max<WAVES>(top, tops);
    const bool bad = top >= 0x7f800000u;
    float scale = __builtin_bit_cast(float, top) / 448.0f;
    if (scale == 0.0f) scale = 1.0f;
    if (bad) scale = __builtin_nanf("");
    if (lane == 0) ((MDBF_GLOBAL float*)a.scales)[t * a.lds] = scale;
    if (scale < 0x1p-126f) {                // of few bits: y may be more than 464 of it, for which the conversion has NaN instead of 448
      const float most = 448.0f * scale;
#pragma unroll
      for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = fminf(fmaxf(h[v][i], -most), most);
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = (v * LANES + lane) * 8;
      if (c >= a.n) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] /= scale;
      store_codes8<STREAM>(a.y, t * a.ldy + c, a.n - c, h[v]);
    }
  } else if (a.yd == MDBF_E4M3) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = (v * LANES + lane) * 8;     // (the four lanes of a block are past the row's end together or hold zeros)
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, h[v][i]) & 0x7fffffffu);
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      if (c >= a.n) continue;
      // 448 = 1.75 * 2^8
      const int byte = m >= 0x7f800000u ? 255 : min(max((int)(m >> 23) - 8 + ((m & 0x7fffffu) > 0x600000u), 1), 254);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = byte == 255 ? __builtin_nanf("") : __builtin_ldexpf(h[v][i], 127 - byte);
      if ((lane & 3) == 0) ((MDBF_GLOBAL uint8_t*)a.scales)[t * a.lds + c / 32] = (uint8_t)byte;
      store_codes8<STREAM>(a.y, t * a.ldy + c, a.n - c, h[v]);
    }
  } else {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = (v * LANES + lane) * 8;
      if (c >= a.n) continue;
      if (a.yd == MDBF_F32) store_float8<MDBF_F32, STREAM>(a.y, t * a.ldy + c, a.n - c, h[v]);
      else if (a.yd == MDBF_F16) store_float8<MDBF_F16, STREAM>(a.y, t * a.ldy + c, a.n - c, h[v]);
      else store_float8<MDBF_BF16, STREAM>(a.y, t * a.ldy + c, a.n - c, h[v]);
    }
  }
}

template <int XD, int HD, int WAVES, int VPT>
static void launch_norm_w(const NormArgs& all, bool stream, hipStream_t s) {
  constexpr int ROWS = WAVES >= 4 ? 1 : 4 / WAVES;
  const int64_t groups = (all.T + (int64_t)ROWS - 1) / ROWS, most = (1ll << 31) / (WAVES * 64 * ROWS);
  for (int64_t g0 = 0; g0 < groups; g0 += most) {   // (a launch has less than 2^32 threads: beyond, their number wraps without an error)
    NormArgs a = all;
    a.t0 = g0 * ROWS;
    const dim3 grid((unsigned)(groups - g0 < most ? groups - g0 : most)), block(WAVES * 64 * ROWS);
    if (stream) norm_kernel<XD, HD, WAVES, VPT, true><<<grid, block, 0, s>>>(a);
    else norm_kernel<XD, HD, WAVES, VPT, false><<<grid, block, 0, s>>>(a);
  }
}

// Waves and pieces by the width: few rows want many waves, whose loads are on their way together, and many rows few, whose meetings cost less; one choice
// serves both within some per cent.  us of 64 rows, and of 16 million channels in all (bf16, with residual):
//   512   1 x 1 2.9, 21.0; 4 x 1 2.8, 27.5                       11008   16 x 2 4.5, 23.3; 8 x 4 4.8, 22.7; 4 x 8 6.4, 24.9
//   2048  4 x 1 3.0, 21.3; 1 x 4 4.7, 19.6; 8 x 1 3.0, 21.3      16384   16 x 2 5.3, 22.1; 8 x 4 5.6, 21.8; 4 x 8 7.6, 21.2
//   4096  4 x 2 3.7, 21.1; 8 x 1 3.3, 21.6; 16 x 1 3.4, 24.3     32768   16 x 8 8.0, 23.9; 16 x 4 7.6, 24.6; 65536   16 x 8 13.8, 22.8
template <int XD, int HD>
static void launch_norm_h(const NormArgs& a, bool stream, hipStream_t s) {
  if (a.n <= 512) launch_norm_w<XD, HD, 1, 1>(a, stream, s);
  else if (a.n <= 2048) launch_norm_w<XD, HD, 4, 1>(a, stream, s);
  else if (a.n <= 4096) launch_norm_w<XD, HD, 4, 2>(a, stream, s);
  else if (a.n <= 16384) launch_norm_w<XD, HD, 16, 2>(a, stream, s);
  else launch_norm_w<XD, HD, 16, 8>(a, stream, s);
}

template <int XD>
static void launch_norm_x(int hd, const NormArgs& a, bool stream, hipStream_t s) {
  if (hd < 0) launch_norm_h<XD, -1>(a, stream, s);
  else if (hd == MDBF_F32) launch_norm_h<XD, MDBF_F32>(a, stream, s);
  else launch_norm_h<XD, XD>(a, stream, s);
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_add_norm(const mdbf_norm_t* desc, const void* x_dev, int64_t ldx, const void* residual_dev, int64_t ldr,
                  const float* weight_dev, int T, void* residual_out_dev, int64_t ldro, void* y_dev, int64_t ldy,
                  void* scales_dev, int64_t lds, void* stream) {
  if (!desc) return MDBF_EINVAL;
  const int n = desc->n;
  const bool eight = desc->y_dtype == MDBF_E4M3;
  if (!row_dtype(desc->x_dtype) || (!row_dtype(desc->y_dtype) && !eight)) return MDBF_EDTYPE;
  if ((residual_dev || residual_out_dev) && !row_dtype(desc->h_dtype)) return MDBF_EDTYPE;
  if (n < 1 || T < 1 || !x_dev || !y_dev || ldx < n || ldy < n || !(desc->eps >= 0.0f)) return MDBF_EINVAL;
  if ((residual_dev && ldr < n) || (residual_out_dev && (!residual_dev || ldro < n))) return MDBF_EINVAL;
  if (eight ? !scales_dev || lds < (desc->scale_group ? (n + 31) / 32 : 1) : scales_dev || desc->scale_group) return MDBF_EINVAL;
  if (n > kNormMaxChannels || (desc->scale_group != 0 && desc->scale_group != 32)) return MDBF_EUNSUPPORTED;
  if (residual_dev && desc->h_dtype != desc->x_dtype && desc->h_dtype != MDBF_F32) return MDBF_EUNSUPPORTED;
  const void* ptrs[] = {x_dev, residual_dev, weight_dev, residual_out_dev, y_dev, scales_dev};
  for (const void* p : ptrs)
    if (!ptr_aligned(p, 16)) return MDBF_EALIGN;
  const NormArgs a = {x_dev, residual_dev, weight_dev, residual_out_dev, y_dev, scales_dev, ldx, ldr, ldro, ldy, lds, 0,
                      T, n, desc->y_dtype, desc->scale_group, desc->eps};
  const int64_t written = (int64_t)T * n * ((eight ? 1 : dtype_size(desc->y_dtype)) + (residual_out_dev ? dtype_size(desc->h_dtype) : 0));
  const bool nt = written > kNormStreamBytes;
  const int hd = residual_dev ? desc->h_dtype : -1;
  if (desc->x_dtype == MDBF_F16) launch_norm_x<MDBF_F16>(hd, a, nt, (hipStream_t)stream);
  else if (desc->x_dtype == MDBF_BF16) launch_norm_x<MDBF_BF16>(hd, a, nt, (hipStream_t)stream);
  else launch_norm_x<MDBF_F32>(hd, a, nt, (hipStream_t)stream);
  return hip_fail((int)hipGetLastError());
}

}  // extern "C"
