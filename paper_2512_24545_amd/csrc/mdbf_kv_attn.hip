// Attention over the 4-bit cache in pages (format and layout: include/mdbf.h).
//
// For a query row (a new token's head) and the tokens j that it sees:  z_j = scale q . k_j,  out = sum_j e^(z_j - m) v_j /
// sum_j e^(z_j - m), in one pass over the cache with a running maximum m and sum.  The query heads that share a kv head
// are rows of one product, so a page is read once for all of them.
//
// On the matrix cores the scores are K Q^T (tokens x rows) and the results V^T P^T (channels x rows): a lane holds one
// query row throughout, the scores' registers are the second product's operand as they lie, and maxima and sums need two
// exchanges between lanes.  Codes become fp16 or bf16 numbers, exactly, with their block's scale by the conversion
// instruction: keys in the registers that feed the product, values on their way into LDS, where transposing reads take them.
#include <math.h>

#include <algorithm>

#include "mdbf_kv.h"

namespace mdbf {

typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 F16x8 __attribute__((ext_vector_type(8)));
typedef short S16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
  const uint8_t* cache;
  const int32_t *table, *cu, *lengths;
  const void* q;
  void* out;
  int64_t table_ld, ldq, ldo;
  int32_t table_width, T, pages, kv_heads, group, page_shift, causal, window, row_tiles;
  float scale;                 // of the scores, times log2(e)
  uint8_t wide_q, wide_o;
};

template <int DT>
__device__ __forceinline__ F32x4 mma16(U32x4 a, U32x4 b, F32x4 c) {
  if (DT == MDBF_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b), c, 0, 0, 0);
}
// eight codes times their scale
template <int DT>
__device__ __forceinline__ U32x4 numbers(uint32_t codes, float unit) {
  if (DT == MDBF_F16)
    return U32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 3))};
  return U32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3))};
}
template <int DT>
__device__ __forceinline__ uint32_t round2(float a, float b) {
  const F32x2 v = {a, b};
  if (DT == MDBF_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, F16x2));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, Bf16x2));
}
__device__ __forceinline__ float unit_of(uint32_t scale_byte) { return __builtin_bit_cast(float, scale_byte << 23); }

// a wave's LDS operations execute in order: this keeps the compiler from moving them across
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A request's part of the step: its first row, its new tokens and its length, cut to what the buffers hold.
struct Request {
  int start, fresh, len;
};
__device__ __forceinline__ Request request_of(const AttnArgs& a, int b) {
  Request r;
  r.start = min(max(a.cu[b], 0), a.T);
  r.fresh = (int)min(max((int64_t)a.cu[b + 1] - r.start, (int64_t)0), (int64_t)(a.T - r.start));
  r.len = (int)min((int64_t)max(a.lengths[b], 0), min((int64_t)a.table_width << a.page_shift, (int64_t)0x7fffff00));
  return r;
}
// the tokens lo <= j < hi that new token i sees
struct Sees {
  int lo, hi;
};
__device__ __forceinline__ Sees sees(const AttnArgs& a, const Request& r, int i) {
  const int pos = r.len - r.fresh + i;
  if (!a.causal) return {0, r.len};
  return {a.window ? max(pos - a.window + 1, 0) : 0, max(pos + 1, 0)};
}

constexpr int kTile = 32;        // tokens per step of a wave
constexpr int kWaves = 4;

// One kv head, 16 query rows; the tokens' tiles are dealt out to the four waves, which meet at the end.
template <int D, int DT>
__global__ __launch_bounds__(64 * kWaves) void attn_few_kernel(AttnArgs a) {
  constexpr int KW = D / 32;                  // dwords of codes per lane and key tile = matrix steps over the channels
  constexpr int KS = D <= 128 ? 1 : D / 128;  // scales among them
  constexpr int VU = D / 64;                  // 16-byte units of values per lane and tile
  constexpr int VROW = D * 2 + 32;            // bytes of a token's values in LDS
  constexpr int CT = D / 16;                  // channel tiles
  constexpr int OROW = D + 4;                 // floats of a row of results in LDS
  static_assert(kTile * VROW >= 16 * OROW * 4, "the results fit the values' place");
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves][kTile * VROW];
  __shared__ float stat[kWaves][2][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
  uint32_t idx = blockIdx.x;
  const int rt0 = idx % a.row_tiles;
  idx /= a.row_tiles;
  const int head = idx % a.kv_heads, b = idx / a.kv_heads;
  const Request rq = request_of(a, b);
  const int64_t rows = (int64_t)rq.fresh * a.group;
  const int P = 1 << a.page_shift;
  const int64_t head_bytes = kv_head_bytes(P, D);
  const MDBF_GLOBAL int32_t* table = (const MDBF_GLOBAL int32_t*)a.table + b * a.table_ld;
  const MDBF_GLOBAL uint8_t* cache = (const MDBF_GLOBAL uint8_t*)a.cache;
  unsigned char* vals = lds[wave];

  for (int64_t rt = rt0; rt * 16 < rows; rt += a.row_tiles) {
    const int64_t R = rt * 16 + r;
    const bool valid = R < rows;
    const int i = valid ? (int)(R / a.group) : 0, g = valid ? (int)(R % a.group) : 0;
    Sees me = sees(a, rq, i);
    if (!valid) me.hi = me.lo = 0;
    // of the first and the last row: what any row sees, and what all rows see
    const Sees s0 = sees(a, rq, (int)(rt * 16 / a.group)), s1 = sees(a, rq, (int)(min(rt * 16 + 15, rows - 1) / a.group));
    const int tmin = s0.lo, tmax = s1.hi, all_lo = s1.lo, all_hi = s0.hi;

    U32x4 qf[KW];
    const int64_t q_at = (int64_t)(rq.start + i) * a.ldq + (int64_t)(head * a.group + g) * D + h * (D / 4);
#pragma unroll
    for (int s = 0; s < KW; ++s) {
      qf[s] = U32x4{0, 0, 0, 0};
      if (valid) {
        const MDBF_GLOBAL uint16_t* p = (const MDBF_GLOBAL uint16_t*)a.q + q_at + 8 * s;
        if (a.wide_q) {
          qf[s] = *(const MDBF_GLOBAL U32x4*)p;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) qf[s][j] = (uint32_t)p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
        }
      }
    }

    float m = -INFINITY, l = 0;
    F32x4 acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = F32x4{0, 0, 0, 0};

    for (int t0 = (tmin & ~(kTile - 1)) + wave * kTile; t0 < tmax; t0 += kWaves * kTile) {
      // the tile's two halves of 16 tokens lie in one page each; pages behind the last are not looked up
      uint32_t kc[2][KW], ks[2][KS];
      U32x4 vc[VU];
      uint32_t vs[VU];
      int64_t base[2];
      int off[2];
      bool there[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int tok = t0 + 16 * f;
        const int page = table[min(tok, rq.len - 1) >> a.page_shift];
        there[f] = (uint32_t)page < (uint32_t)a.pages;
        base[f] = ((int64_t)(there[f] ? page : 0) * a.kv_heads + head) * head_bytes;
        off[f] = tok & (P - 1);
        const MDBF_GLOBAL uint32_t* kp = (const MDBF_GLOBAL uint32_t*)(cache + base[f] + (int64_t)(off[f] + r) * (D / 2) + h * (D / 8));
#pragma unroll
        for (int s = 0; s < KW; ++s) kc[f][s] = kp[s];
        const MDBF_GLOBAL uint8_t* sp = cache + base[f] + (int64_t)P * D + (off[f] + r) * (D / 32);
#pragma unroll
        for (int s = 0; s < KS; ++s) ks[f][s] = there[f] ? sp[D == 64 ? h >> 1 : h * KS + s] : kKvNanScale;
      }
#pragma unroll
      for (int n = 0; n < VU; ++n) {
        const int f = D == 64 ? lane >> 5 : n / (VU / 2 ? VU / 2 : 1);
        const int unit = D == 64 ? lane & 31 : (n % (VU / 2 ? VU / 2 : 1)) * 64 + lane;
        const int64_t at = (f ? base[1] : base[0]);
        const int o = f ? off[1] : off[0];
        vc[n] = *(const MDBF_GLOBAL U32x4*)(cache + at + (int64_t)P * (D / 2) + o * (D / 2) + unit * 16);
        vs[n] = (f ? there[1] : there[0]) ? cache[at + (int64_t)P * (D + D / 32) + o * (D / 32) + unit] : kKvNanScale;
      }

      // scores: a lane holds those of its row with tokens 4 h + 0 .. 3 of each half
      float z[2][4];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        F32x4 s4 = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KW; ++s) s4 = mma16<DT>(numbers<DT>(kc[f][s], unit_of(ks[f][KS == 1 ? 0 : s / 4])), qf[s], s4);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[f][j] = s4[j] * a.scale;
      }
      const bool inside = t0 >= all_lo && t0 + kTile <= all_hi;     // every row sees every token
      if (!inside) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int tok = t0 + 16 * f + 4 * h + j;
            if (tok < me.lo || tok >= me.hi) z[f][j] = -INFINITY;
          }
      }
      float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top), use = mn == -INFINITY ? 0.0f : mn;
      const float alpha = __builtin_amdgcn_exp2f(m - use);
      m = mn;
      float p[2][4], sum = 0;
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[f][j] = __builtin_amdgcn_exp2f(z[f][j] - use);
          sum += p[f][j];
        }
      l = l * alpha + sum;
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c] *= alpha;
      }
      const U32x4 pf = {round2<DT>(p[0][0], p[0][1]), round2<DT>(p[0][2], p[0][3]), round2<DT>(p[1][0], p[1][1]), round2<DT>(p[1][2], p[1][3])};

      // values that no row sees are zeros; NaN among the others goes to the rows that see it, not through the product, where a
      // zero weight would bring it to all rows
#pragma unroll
      for (int n = 0; n < VU; ++n) {
        const int f = D == 64 ? lane >> 5 : n / (VU / 2 ? VU / 2 : 1);
        const int unit = D == 64 ? lane & 31 : (n % (VU / 2 ? VU / 2 : 1)) * 64 + lane;
        const int row = 16 * f + unit / (D / 32), tok = t0 + row;
        if (!inside && (tok < tmin || tok >= tmax)) {
          vc[n] = U32x4{0, 0, 0, 0};
          vs[n] = 127;
        }
        uint64_t bad = __ballot(vs[n] == kKvNanScale);
        if (bad) {
          if (vs[n] == kKvNanScale) {
            vc[n] = U32x4{0, 0, 0, 0};
            vs[n] = 127;
          }
          for (; bad; bad &= bad - 1) {
            const int from = __builtin_ctzll(bad);
            const int bu = D == 64 ? from & 31 : (n % (VU / 2 ? VU / 2 : 1)) * 64 + from, bf = D == 64 ? from >> 5 : f;
            const int bt = t0 + 16 * bf + bu / (D / 32), bg = bu % (D / 32);
#pragma unroll
            for (int c = 0; c < CT; ++c)
              if (c / 2 == bg && bt >= me.lo && bt < me.hi) acc[c] = F32x4{NAN, NAN, NAN, NAN};
          }
        }
        const float unit_f = unit_of(vs[n]);
        unsigned char* to = vals + row * VROW + (unit % (D / 32)) * 64;
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<U32x4*>(to + w * 16) = numbers<DT>(vc[n][w], unit_f);
      }
      wave_lds_order();
      // a lane's channel of tokens 4 h + 0 .. 3 of each half: the order of the scores' registers
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const unsigned char* from = vals + (4 * h + (r >> 2)) * VROW + c * 32 + (r & 3) * 8;
        const U32x2 v0 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)from));
        const U32x2 v1 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)(from + 16 * VROW)));
        acc[c] = mma16<DT>(U32x4{v0[0], v0[1], v1[0], v1[1]}, pf, acc[c]);
      }
      wave_lds_order();
    }

    // the waves meet
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (h == 0) {
      stat[wave][0][r] = m;
      stat[wave][1][r] = l;
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<F32x4*>(vals + (r * OROW + c * 16 + h * 4) * 4) = acc[c];
    __syncthreads();
    {
      constexpr int N = D / 16;      // channels per thread
      const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
      const int64_t Ro = rt * 16 + row;
      if (Ro < rows) {
        const int io = (int)(Ro / a.group), go = (int)(Ro % a.group);
        const Sees so = sees(a, rq, io);
        float top = stat[0][0][row];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, stat[w][0][row]);
        if (top == -INFINITY) top = 0.0f;
        float sum = 0, o[N];
#pragma unroll
        for (int c = 0; c < N; ++c) o[c] = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(stat[w][0][row] - top);
          sum += f * stat[w][1][row];
          const float* from = reinterpret_cast<const float*>(lds[w]) + row * OROW + part * N;
#pragma unroll
          for (int c = 0; c < N; ++c) o[c] += f * from[c];
        }
        const float inv = 1.0f / sum;
        uint32_t w2[N / 2];
#pragma unroll
        for (int c = 0; c < N / 2; ++c) w2[c] = so.hi > so.lo ? round2<DT>(o[2 * c] * inv, o[2 * c + 1] * inv) : 0u;
        MDBF_GLOBAL uint16_t* to = (MDBF_GLOBAL uint16_t*)a.out + (int64_t)(rq.start + io) * a.ldo + (int64_t)(head * a.group + go) * D + part * N;
        if (a.wide_o) {
#pragma unroll
          for (int c = 0; c < N / 4; ++c) ((MDBF_GLOBAL U32x2*)to)[c] = U32x2{w2[2 * c], w2[2 * c + 1]};
        } else {
#pragma unroll
          for (int c = 0; c < N / 2; ++c) {
            to[2 * c] = (uint16_t)w2[c];
            to[2 * c + 1] = (uint16_t)(w2[c] >> 16);
          }
        }
      }
    }
    __syncthreads();
  }
}

static int check_attn(const mdbf_kv_t* kv, const mdbf_attn_t* at, int requests, int T) {
  int st = check_kv(kv);
  if (st) return st;
  if (!at || requests < 1 || T < 1) return MDBF_EINVAL;
  if (at->q_heads <= 0 || at->q_heads % kv->kv_heads || at->window < 0 || at->max_fresh < 1 || at->max_length < 1 || !isfinite(at->scale))
    return MDBF_EINVAL;
  if (at->window && !(at->flags & MDBF_ATTN_CAUSAL)) return MDBF_EINVAL;
  if ((at->flags & ~MDBF_ATTN_CAUSAL) || at->q_heads > (1 << 16)) return MDBF_EUNSUPPORTED;
  return MDBF_OK;
}

template <int DT>
static void launch_few(int d, unsigned grid, const AttnArgs& a, hipStream_t s) {
  if (d == 64) attn_few_kernel<64, DT><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (d == 128) attn_few_kernel<128, DT><<<grid, 64 * kWaves, 0, s>>>(a);
  else attn_few_kernel<256, DT><<<grid, 64 * kWaves, 0, s>>>(a);
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_kv_attention_workspace_bytes(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T, size_t* bytes_out) {
  if (!bytes_out) return MDBF_EINVAL;
  int st = check_attn(kv, attn, requests, T);
  if (st) return st;
  *bytes_out = 0;
  return MDBF_OK;
}

int mdbf_kv_attention(const mdbf_kv_t* kv, const mdbf_attn_t* attn, const void* cache_dev, size_t cache_bytes,
                      const int32_t* table_dev, int64_t table_ld, int table_width, const int32_t* cu_dev,
                      const int32_t* lengths_dev, int requests, const void* q_dev, int64_t ldq, int T, void* out_dev,
                      int64_t ldo, void* workspace_dev, size_t workspace_bytes, void* stream) {
  int st = check_attn(kv, attn, requests, T);
  if (st) return st;
  if ((st = check_kv_cache(kv, cache_dev, cache_bytes))) return st;
  const int64_t row = (int64_t)attn->q_heads * kv->head_dim;
  if (!table_dev || !cu_dev || !lengths_dev || !q_dev || !out_dev || table_width < 1 || table_ld < table_width || ldq < row || ldo < row)
    return MDBF_EINVAL;
  const void *wide[] = {q_dev, out_dev, workspace_dev}, *ints[] = {table_dev, cu_dev, lengths_dev};
  for (const void* p : wide)
    if (!kv_aligned(p, 16)) return MDBF_EALIGN;
  for (const void* p : ints)
    if (!kv_aligned(p, 4)) return MDBF_EALIGN;
  (void)workspace_bytes;
  AttnArgs a = {};
  a.cache = (const uint8_t*)cache_dev, a.table = table_dev, a.cu = cu_dev, a.lengths = lengths_dev, a.q = q_dev, a.out = out_dev;
  a.table_ld = table_ld, a.ldq = ldq, a.ldo = ldo, a.table_width = table_width, a.T = T, a.pages = kv->pages;
  a.kv_heads = kv->kv_heads, a.group = attn->q_heads / kv->kv_heads, a.page_shift = kv_page_shift(kv->page_size);
  a.causal = attn->flags & MDBF_ATTN_CAUSAL, a.window = attn->window;
  a.scale = (float)(attn->scale * 1.4426950408889634);
  a.wide_q = ldq % 8 == 0, a.wide_o = ldo % 4 == 0;
  const int64_t most = std::min<int64_t>(attn->max_fresh, T);
  a.row_tiles = (int32_t)std::min<int64_t>((most * a.group + 15) / 16, 1 << 16);
  const int64_t grid = (int64_t)requests * a.kv_heads * a.row_tiles;
  if (grid > 0x7fffffff) return MDBF_EUNSUPPORTED;
  if (kv->dtype == MDBF_F16) launch_few<MDBF_F16>(kv->head_dim, (unsigned)grid, a, (hipStream_t)stream);
  else launch_few<MDBF_BF16>(kv->head_dim, (unsigned)grid, a, (hipStream_t)stream);
  return hip_fail((int)hipGetLastError());
}

}  // extern "C"
