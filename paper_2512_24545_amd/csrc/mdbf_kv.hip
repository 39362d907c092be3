// Around the attention over the 4-bit cache: block tables and slot maps, norm and rotation of queries and keys, and
// tokens into the cache and out of it.  Format and layout of the cache are described in include/mdbf.h.
#include <math.h>

#include <algorithm>

#include "mdbf_kv.h"

namespace mdbf {

// ---- block tables and slot maps -------------------------------------------------------------------------
// A prefix sum over the requests, then one entry per new token; a workgroup goes through the requests 1024 at a time,
// one per thread, twice: sums and checks first (nothing is written before the step is known to fit), then the scan (up to 1024
// the first one's results are still there), whose prefixes stay in LDS for the tokens and the new pages, which find their
// request by bisection.  Long steps leave the tokens to a second launch that bisects cu, in LDS where that has room.  All
// latency: the kernel takes 5.1 us for 64 requests with a token each, 7.4 and 6.5 for 500 prompts of 250000 tokens (3 MB, 0.6 us at
// the rate of a copy): dependent loads, a scan (a second one and more from 1025 requests on) and its barriers.
constexpr int kSlotThreads = 1024;
constexpr int kSlotOneLaunch = 8192;      // new tokens up to which the first launch writes the slots too
constexpr int kSlotTokens = 1024;         // tokens per workgroup of the second launch

struct SlotArgs {
  const int32_t *cached, *fresh, *free_pages, *taken;
  int32_t *table, *lengths, *cu, *positions, *taken_out, *status;
  int64_t* slots;
  int64_t table_ld;
  int32_t requests, page_shift, table_width, free_count, T, tokens_here;
};

// inclusive sum over the workgroup's threads of two values at once; `total` receives the sums of all
__device__ __forceinline__ void scan_pair(int64_t& a, int64_t& b, int64_t (&total)[2], int64_t (*waves)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t ua = __shfl_up(a, o), ub = __shfl_up(b, o);
    if (lane >= o) {
      a += ua;
      b += ub;
    }
  }
  __syncthreads();          // the last use of `waves` is over
  if (lane == 63) {
    waves[wave][0] = a;
    waves[wave][1] = b;
  }
  __syncthreads();
  int64_t before_a = 0, before_b = 0;
  total[0] = total[1] = 0;
  for (int w = 0; w < kSlotThreads / 64; ++w) {
    if (w == wave) {
      before_a = total[0];
      before_b = total[1];
    }
    total[0] += waves[w][0];
    total[1] += waves[w][1];
  }
  a += before_a;
  b += before_b;
}

// the last i with start[i] <= t, start[0] <= t
template <class P>
__device__ __forceinline__ int last_at_most(P start, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = lo + ((hi - lo) >> 1);
    if (start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(SlotArgs a) {
  __shared__ int64_t waves[kSlotThreads / 64][2];
  __shared__ int32_t tok_start[kSlotThreads], page_start[kSlotThreads], had[kSlotThreads], held[kSlotThreads];
  const int tid = threadIdx.x, P = 1 << a.page_shift;
  const int taken = a.taken[0];

  int64_t tokens = 0, pages = 0;
  int status = 0;
  for (int64_t r = tid; r < a.requests; r += kSlotThreads) {
    const int64_t c = a.cached[r], f = a.fresh[r];
    if (c < 0 || f < 0 || c + f > 0x7fffffff) {
      status |= MDBF_KV_BAD_LENGTH;
    } else {
      const int64_t after = (c + f + P - 1) >> a.page_shift;
      if (after > a.table_width) status |= MDBF_KV_BAD_WIDTH;
      tokens += f;
      pages += after - ((c + P - 1) >> a.page_shift);
    }
  }
  int64_t total[2];
  scan_pair(tokens, pages, total, waves);
  const bool one_round = a.requests <= kSlotThreads;      // tokens, pages: the sums up to and with this thread's request
  __shared__ int flags;
  if (tid == 0) flags = 0;
  __syncthreads();
  if (__any(status) && status) atomicOr(&flags, status);
  __syncthreads();
  status = flags;
  if (total[0] > a.T) status |= MDBF_KV_BAD_TOKENS;
  if (taken < 0 || taken + total[1] > a.free_count) status |= MDBF_KV_NO_PAGES;
  if (tid == 0) {
    a.status[0] = status;
    a.taken_out[0] = status ? taken : taken + (int)total[1];
  }
  const int real = status ? 0 : (int)total[0];
  if (a.tokens_here)
    for (int64_t t = real + tid; t < a.T; t += kSlotThreads) {
      a.slots[t] = -1;
      a.positions[t] = -1;
    }
  if (status) {
    for (int64_t r = tid; r < a.requests; r += kSlotThreads) {
      a.lengths[r] = max(a.cached[r], 0);
      a.cu[r] = 0;
    }
    if (tid == 0) a.cu[a.requests] = 0;
    return;
  }

  int tok0 = 0, page0 = taken;              // of the requests before this pass
  for (int64_t r0 = 0; r0 < a.requests; r0 += kSlotThreads) {
    const int64_t r = r0 + tid;
    const int n = (int)min((int64_t)kSlotThreads, a.requests - r0);
    const int c = tid < n ? a.cached[r] : 0, f = tid < n ? a.fresh[r] : 0;
    const int before = (int)(((int64_t)c + P - 1) >> a.page_shift), after = (int)(((int64_t)c + f + P - 1) >> a.page_shift);
    int64_t t = f, p = after - before;
    if (one_round) t = tokens, p = pages;
    else scan_pair(t, p, total, waves);
    const int first = tok0 + (int)t - f, page = page0 + (int)p - (after - before);
    tok_start[tid] = first;
    page_start[tid] = page;
    had[tid] = c;
    held[tid] = before;
    if (tid < n) {
      a.lengths[r] = c + f;
      a.cu[r] = first;
    }
    __syncthreads();
    for (int64_t j = tid; j < total[1]; j += kSlotThreads) {
      const int i = (int)j;
      const int q = last_at_most(page_start, n, page0 + i);
      a.table[(r0 + q) * a.table_ld + held[q] + (page0 + i - page_start[q])] = a.free_pages[page0 + i];
    }
    if (a.tokens_here)
      for (int i = tid; i < (int)total[0]; i += kSlotThreads) {
        const int q = last_at_most(tok_start, n, tok0 + i);
        const int pos = had[q] + (tok0 + i - tok_start[q]), at = pos >> a.page_shift;
        // (entries that this launch makes are taken from the free list itself)
        const int pg = at < held[q] ? a.table[(r0 + q) * a.table_ld + at] : a.free_pages[page_start[q] + at - held[q]];
        a.slots[tok0 + i] = ((int64_t)pg << a.page_shift) + (pos & (P - 1));
        a.positions[tok0 + i] = pos;
      }
    tok0 += (int)total[0];
    page0 += (int)total[1];
    __syncthreads();
  }
  if (tid == 0) a.cu[a.requests] = tok0;
}

// the tokens of a long step, from cu and the tables that slots_kernel left
constexpr int kSlotLds = 4096;            // requests whose cu a workgroup copies
__global__ __launch_bounds__(256) void slots_tokens_kernel(SlotArgs a) {
  __shared__ int32_t starts[kSlotLds];
  const int P = 1 << a.page_shift, real = a.cu[a.requests];
  const bool here = a.requests <= kSlotLds;
  if (here) {
    for (int r = threadIdx.x; r < a.requests; r += 256) starts[r] = a.cu[r];
    __syncthreads();
  }
  for (int64_t t = (int64_t)blockIdx.x * kSlotTokens + threadIdx.x, end = min((int64_t)a.T, ((int64_t)blockIdx.x + 1) * kSlotTokens);
       t < end; t += 256) {
    int64_t slot = -1;
    int pos = -1;
    if (t < real) {
      const int r = here ? last_at_most(starts, a.requests, (int)t) : last_at_most(a.cu, a.requests, (int)t);
      pos = a.cached[r] + ((int)t - (here ? starts[r] : a.cu[r]));
      slot = ((int64_t)a.table[r * a.table_ld + (pos >> a.page_shift)] << a.page_shift) + (pos & (P - 1));
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
  }
}

// ---- tokens in and out ----------------------------------------------------------------------------------
// Eight channels per lane, head_dim / 8 lanes per head: 16 bytes of a 16-bit type, one dword of codes, a block's scale in
// four lanes.  A wave takes one token and walks over its heads, so what goes with the position is loaded once.

template <int DT>
__device__ __forceinline__ void load8(const void* base, int64_t at, bool wide, float (&x)[8]) {
  if (!wide) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = load_as_float(base, at + i, DT);
  } else if (DT == MDBF_F32) {
    const MDBF_GLOBAL F32x4* p = (const MDBF_GLOBAL F32x4*)((const MDBF_GLOBAL float*)base + at);
    const F32x4 a = __builtin_nontemporal_load(p), b = __builtin_nontemporal_load(p + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  } else {
    const U32x4 v = __builtin_nontemporal_load((const MDBF_GLOBAL U32x4*)((const MDBF_GLOBAL uint16_t*)base + at));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = v[i];      // (the bit cast of a vector's element itself would take element 0)
      if (DT == MDBF_F16) {
        const F16x2 h = __builtin_bit_cast(F16x2, w);
        x[2 * i] = (float)h[0];
        x[2 * i + 1] = (float)h[1];
      } else {
        x[2 * i] = __builtin_bit_cast(float, w << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
      }
    }
  }
}

// two values rounded to nearest in the 16-bit type
template <int DT>
__device__ __forceinline__ uint32_t round_pair(float a, float b) {
  const F32x2 v = {a, b};
  if (DT == MDBF_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, F16x2));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, Bf16x2));
}

// STREAM: the results of the call are more than the caches should hold for a reader (a template's argument: of two stores to one
// place the compiler makes one, without the hint)
template <int DT, bool STREAM>
__device__ __forceinline__ void store8(void* base, int64_t at, bool wide, const float (&x)[8]) {
  if (!wide) {
#pragma unroll
    for (int i = 0; i < 8; ++i) store_from_float(base, at + i, DT, x[i]);
  } else if (DT == MDBF_F32) {
    MDBF_GLOBAL F32x4* p = (MDBF_GLOBAL F32x4*)((MDBF_GLOBAL float*)base + at);
    const F32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
    if (STREAM) {
      __builtin_nontemporal_store(a, p);
      __builtin_nontemporal_store(b, p + 1);
    } else {
      p[0] = a;
      p[1] = b;
    }
  } else {
    U32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = round_pair<DT>(x[2 * i], x[2 * i + 1]);
    MDBF_GLOBAL U32x4* p = (MDBF_GLOBAL U32x4*)((MDBF_GLOBAL uint16_t*)base + at);
    if (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
  }
}

// x rounded to the type
template <int DT>
__device__ __forceinline__ void round8(float (&x)[8]) {
  if (DT == MDBF_F32) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = round_pair<DT>(x[2 * i], x[2 * i + 1]);
    if (DT == MDBF_F16) {
      const F16x2 h = __builtin_bit_cast(F16x2, v);
      x[2 * i] = (float)h[0];
      x[2 * i + 1] = (float)h[1];
    } else {
      x[2 * i] = __builtin_bit_cast(float, v << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, v & 0xffff0000u);
    }
  }
}

// The scale byte of a block from its largest magnitude's bits, and eight codes by the conversion instruction (nearest, ties to
// the even code, beyond 6 saturated).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top, int kv_dt) {
  const uint32_t e = top >> 23;
  if (e == 255) return kKvNanScale;
  const int b = (int)e - 2 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)min(max(b, (int)kKvScaleMin[kv_dt]), (int)kKvScaleMax[kv_dt]);
}
__device__ __forceinline__ void quantise8(const float (&x)[8], int kv_dt, uint32_t& codes, uint32_t& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);   // a NaN's bits are the largest
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  scale = scale_byte(top, kv_dt);
  const float unit = __builtin_bit_cast(float, scale << 23);
  codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], unit, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], unit, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], unit, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], unit, 3);
}
__device__ __forceinline__ void store_codes(uint8_t* cache, const KvPlace& at, int e, uint32_t codes, uint32_t scale) {
  *(MDBF_GLOBAL uint32_t*)((MDBF_GLOBAL uint8_t*)cache + at.codes + e * 4) = codes;
  if ((e & 3) == 0) ((MDBF_GLOBAL uint8_t*)cache)[at.scales + (e >> 2)] = (uint8_t)scale;
}

struct QkvArgs {
  const void *q, *k, *v;
  const float *qw, *kw, *rope;
  const int32_t* positions;
  void *q_out, *k_out;
  uint8_t* cache;
  const int64_t* slots;
  int64_t ldq, ldk, ldv, ldqo, ldko, slot_count;
  int32_t T, q_heads, kv_heads, rot, rope_rows, page_shift, kv_dt, units, units_per_wave, interleaved;
  float eps;
  uint8_t wide_q, wide_k, wide_v, wide_qo, wide_ko, stream;
};

// Rows in, rows out and codes out, each once: x / sqrt(mean x^2 + eps) * w, then pairs (p, q) -> (p c - q s, q c + p s), in fp32 and
// rounded once, at the store; keys that go into the cache are first rounded to the outputs' type, as by a program that stored them in
// between; values go in as they come.  D / 8 lanes hold a head, eight channels each: the sum of squares is a few exchanges among them, a rotated
// pair lies in one lane or in two of the same head, and the lanes' cosines and sines serve all heads of a token.  Bound by HBM where
// it is large: 8192 tokens of 64 heads of 128 (273 MB) 54 us, the keys and values of 32 heads into the cache and back (340 MB) 69 us,
// 4.9 to 5.1 TB/s, what a copy reaches; 64 tokens of 40 heads are the latency of a launch and its loads, 4.1 us.
// Units of a token: query heads, key heads and, where the cache is written, value heads.
template <int XD, int YD, int D, bool STREAM>
__global__ __launch_bounds__(256) void qkv_kernel(QkvArgs a) {
  constexpr int L = D / 8, PER = 64 / L;
  const int lane = threadIdx.x & 63, e = lane & (L - 1), sub = lane / L;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const int u0 = blockIdx.y * a.units_per_wave, u1 = min(u0 + a.units_per_wave, a.units);

  // the lane's cosines and sines; those of padding and of channels that stay are not used
  const int pos = a.rot ? a.positions[t] : 0;
  const bool padding = pos < 0;
  const int half = a.rot >> 1, c0 = e * 8;
  const bool turned = c0 < a.rot;
  float cs[8], sn[8];
  int partner = lane;
  if (turned && !padding) {
    const float* row = a.rope + (int64_t)min(pos, a.rope_rows - 1) * a.rot;
    if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cs[i] = ((const MDBF_GLOBAL float*)row)[c0 / 2 + i];
        sn[i] = ((const MDBF_GLOBAL float*)row)[half + c0 / 2 + i];
      }
    } else {
      const int p = c0 < half ? c0 : c0 - half;
      partner = c0 < half ? lane + half / 8 : lane - half / 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        cs[i] = ((const MDBF_GLOBAL float*)row)[p + i];
        sn[i] = ((const MDBF_GLOBAL float*)row)[half + p + i];
        if (c0 < half) sn[i] = -sn[i];
      }
    }
    if (pos >= a.rope_rows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = __builtin_nanf("");
    }
  }
  const int64_t slot = a.cache ? a.slots[t] : -1;
  const bool caches = !padding && slot >= 0 && slot < a.slot_count;

  for (int u = u0 + sub; u < u1; u += PER) {     // (a unit's lanes stay together: shuffles do not leave it)
    const int kind = u < a.q_heads ? 0 : u < a.q_heads + a.kv_heads ? 1 : 2;
    const int h = kind == 0 ? u : kind == 1 ? u - a.q_heads : u - a.q_heads - a.kv_heads;
    float x[8];
    if (kind == 0) load8<XD>(a.q, t * a.ldq + (int64_t)h * D + c0, a.wide_q, x);
    else if (kind == 1) load8<XD>(a.k, t * a.ldk + (int64_t)h * D + c0, a.wide_k, x);
    else load8<XD>(a.v, t * a.ldv + (int64_t)h * D + c0, a.wide_v, x);
    if (kind < 2) {
      const float* w = kind ? a.kw : a.qw;
      if (w) {
        float ss = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
        for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
        const float r = 1.0f / sqrtf(ss / D + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * ((const MDBF_GLOBAL float*)w)[c0 + i];
      }
      if (a.rot) {
        if (a.interleaved) {
          if (turned) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = x[2 * i], q = x[2 * i + 1];
              x[2 * i] = p * cs[i] - q * sn[i];
              x[2 * i + 1] = q * cs[i] + p * sn[i];
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float other = __shfl(x[i], partner);
            if (turned) x[i] = x[i] * cs[i] + other * sn[i];
          }
        }
      }
      if (padding) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
      }
      if (kind == 0) store8<YD, STREAM>(a.q_out, t * a.ldqo + (int64_t)h * D + c0, a.wide_qo, x);
      else if (a.k_out) store8<YD, STREAM>(a.k_out, t * a.ldko + (int64_t)h * D + c0, a.wide_ko, x);
      if (kind == 1) round8<YD>(x);
    }
    if (kind && caches) {
      uint32_t codes, scale;
      quantise8(x, a.kv_dt, codes, scale);
      store_codes(a.cache, kv_place(slot, h, kind - 1, a.kv_heads, a.page_shift, D), e, codes, scale);
    }
  }
}

struct ReadArgs {
  const uint8_t* cache;
  const int64_t* slots;
  void *k, *v;
  int64_t ldk, ldv, slot_count;
  int32_t T, kv_heads, page_shift;
  uint32_t scale_max;
  uint8_t wide_k, wide_v, stream;
};

template <int YD, int D, bool STREAM>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
  constexpr int L = D / 8, PER = 64 / L;
  const int lane = threadIdx.x & 63, e = lane & (L - 1), sub = lane / L;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const int64_t slot = a.slots[t];
  const bool there = slot >= 0 && slot < a.slot_count;
  for (int u = sub; u < 2 * a.kv_heads; u += PER) {
    const int value = u >= a.kv_heads, h = value ? u - a.kv_heads : u;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (there) {
      const KvPlace at = kv_place(slot, h, value, a.kv_heads, a.page_shift, D);
      const uint32_t codes = *(const MDBF_GLOBAL uint32_t*)((const MDBF_GLOBAL uint8_t*)a.cache + at.codes + e * 4);
      const uint32_t scale = ((const MDBF_GLOBAL uint8_t*)a.cache)[at.scales + (e >> 2)];
      const float unit = __builtin_bit_cast(float, (scale > a.scale_max ? kKvNanScale : scale) << 23);
      const F32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1),
                  p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
      x[0] = p0[0], x[1] = p0[1], x[2] = p1[0], x[3] = p1[1], x[4] = p2[0], x[5] = p2[1], x[6] = p3[0], x[7] = p3[1];
    }
    store8<YD, STREAM>(value ? a.v : a.k, t * (value ? a.ldv : a.ldk) + (int64_t)h * D + e * 8, value ? a.wide_v : a.wide_k, x);
  }
}

// ---- checks ---------------------------------------------------------------------------------------------
static bool valid_dtype(int d) { return d == MDBF_F16 || d == MDBF_BF16 || d == MDBF_F32; }
static bool valid_head_dim(int d) { return d == 64 || d == 128 || d == 256; }

int check_kv(const mdbf_kv_t* kv) {
  if (!kv) return MDBF_EINVAL;
  if (kv->pages <= 0 || kv->kv_heads <= 0 || kv->head_dim <= 0 || kv->page_size <= 0) return MDBF_EINVAL;
  if (kv->dtype != MDBF_F16 && kv->dtype != MDBF_BF16) return MDBF_EDTYPE;
  const int P = kv->page_size;
  if (!valid_head_dim(kv->head_dim) || P < 16 || P > 256 || (P & (P - 1)) || kv->kv_heads > (1 << 16)) return MDBF_EUNSUPPORTED;
  return MDBF_OK;
}

int check_kv_cache(const mdbf_kv_t* kv, const void* cache, size_t cache_bytes) {
  int st = check_kv(kv);
  if (st) return st;
  if (!cache) return MDBF_EINVAL;
  if (!kv_aligned(cache, 16)) return MDBF_EALIGN;
  if (cache_bytes / (size_t)kv_page_bytes(*kv) < (size_t)kv->pages) return MDBF_EWORKSPACE;
  return MDBF_OK;
}

// Results beyond this are written past the caches: 8192 tokens of 64 heads (134 MB) 57.9 -> 53.4 us, their keys and values back
// out of the cache 80.6 -> 68.6 us together with the append's loads.
constexpr int64_t kStreamBytes = 32 << 20;
static bool wide_rows(int64_t ld, int dt) { return ld * dtype_size(dt) % 16 == 0; }

template <int XD, int YD, bool STREAM>
static void launch_qkv_s(int d, dim3 grid, const QkvArgs& a, hipStream_t s) {
  if (d == 64) qkv_kernel<XD, YD, 64, STREAM><<<grid, 256, 0, s>>>(a);
  else if (d == 128) qkv_kernel<XD, YD, 128, STREAM><<<grid, 256, 0, s>>>(a);
  else qkv_kernel<XD, YD, 256, STREAM><<<grid, 256, 0, s>>>(a);
}
template <int XD, int YD>
static void launch_qkv_d(int d, dim3 grid, const QkvArgs& a, hipStream_t s) {
  if (a.stream) launch_qkv_s<XD, YD, true>(d, grid, a, s);
  else launch_qkv_s<XD, YD, false>(d, grid, a, s);
}
template <int XD>
static void launch_qkv_x(int yd, int d, dim3 grid, const QkvArgs& a, hipStream_t s) {
  if (yd == MDBF_F16) launch_qkv_d<XD, MDBF_F16>(d, grid, a, s);
  else if (yd == MDBF_BF16) launch_qkv_d<XD, MDBF_BF16>(d, grid, a, s);
  else launch_qkv_d<XD, MDBF_F32>(d, grid, a, s);
}
static int launch_qkv(int xd, int yd, int d, QkvArgs& a, hipStream_t s) {
  const int per = 64 / (d / 8);
  // a wave per token where there are tokens enough for the device, else the heads of a token on several waves
  const int64_t waves = 4096;
  int parts = (int)std::min<int64_t>((a.units + per - 1) / per, std::max<int64_t>(1, waves / a.T));
  a.units_per_wave = ((a.units + parts - 1) / parts + per - 1) / per * per;
  parts = (a.units + a.units_per_wave - 1) / a.units_per_wave;
  const dim3 grid((unsigned)(((int64_t)a.T + 3) / 4), (unsigned)parts);
  if (xd == MDBF_F16) launch_qkv_x<MDBF_F16>(yd, d, grid, a, s);
  else if (xd == MDBF_BF16) launch_qkv_x<MDBF_BF16>(yd, d, grid, a, s);
  else launch_qkv_x<MDBF_F32>(yd, d, grid, a, s);
  return (int)hipGetLastError();
}

template <int YD, bool STREAM>
static void launch_read_s(int d, const ReadArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.T + 3) / 4));
  if (d == 64) read_kernel<YD, 64, STREAM><<<grid, 256, 0, s>>>(a);
  else if (d == 128) read_kernel<YD, 128, STREAM><<<grid, 256, 0, s>>>(a);
  else read_kernel<YD, 256, STREAM><<<grid, 256, 0, s>>>(a);
}
template <int YD>
static void launch_read_d(int d, const ReadArgs& a, hipStream_t s) {
  if (a.stream) launch_read_s<YD, true>(d, a, s);
  else launch_read_s<YD, false>(d, a, s);
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_kv_page_bytes(const mdbf_kv_t* kv, size_t* bytes_out) {
  if (!bytes_out) return MDBF_EINVAL;
  int st = check_kv(kv);
  if (st) return st;
  *bytes_out = (size_t)kv_page_bytes(*kv);
  return MDBF_OK;
}

int mdbf_kv_slots(int requests, int page_size, const int32_t* cached_dev, const int32_t* fresh_dev, int32_t* table_dev,
                  int64_t table_ld, int table_width, const int32_t* free_dev, int free_count, const int32_t* taken_dev,
                  int T, int32_t* lengths_dev, int32_t* cu_dev, int64_t* slots_dev, int32_t* positions_dev,
                  int32_t* taken_out_dev, int32_t* status_dev, void* stream) {
  if (requests < 1 || T < 1 || table_width < 1 || table_ld < table_width || free_count < 0) return MDBF_EINVAL;
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return MDBF_EUNSUPPORTED;
  const void* ptrs[] = {cached_dev, fresh_dev, table_dev, taken_dev, lengths_dev, cu_dev, slots_dev, positions_dev, taken_out_dev, status_dev};
  for (const void* p : ptrs) {
    if (!p) return MDBF_EINVAL;
    if (!kv_aligned(p, p == slots_dev ? 8 : 4)) return MDBF_EALIGN;
  }
  if (free_count && !free_dev) return MDBF_EINVAL;
  if (!kv_aligned(free_dev, 4)) return MDBF_EALIGN;
  SlotArgs a;
  a.cached = cached_dev, a.fresh = fresh_dev, a.free_pages = free_dev, a.taken = taken_dev;
  a.table = table_dev, a.lengths = lengths_dev, a.cu = cu_dev, a.positions = positions_dev;
  a.taken_out = taken_out_dev, a.status = status_dev, a.slots = slots_dev, a.table_ld = table_ld;
  a.requests = requests, a.page_shift = kv_page_shift(page_size), a.table_width = table_width;
  a.free_count = free_count, a.T = T, a.tokens_here = T <= kSlotOneLaunch;
  slots_kernel<<<1, kSlotThreads, 0, (hipStream_t)stream>>>(a);
  int e = (int)hipGetLastError();
  if (e == 0 && !a.tokens_here) {
    slots_tokens_kernel<<<(unsigned)(((int64_t)T + kSlotTokens - 1) / kSlotTokens), 256, 0, (hipStream_t)stream>>>(a);
    e = (int)hipGetLastError();
  }
  return hip_fail(e);
}

int mdbf_kv_append(const mdbf_kv_t* kv, void* cache_dev, size_t cache_bytes, const void* k_dev, int64_t ldk,
                   const void* v_dev, int64_t ldv, int x_dtype, const int64_t* slots_dev, int T, void* stream) {
  int st = check_kv_cache(kv, cache_dev, cache_bytes);
  if (st) return st;
  if (!valid_dtype(x_dtype)) return MDBF_EDTYPE;
  const int64_t row = (int64_t)kv->kv_heads * kv->head_dim;
  if (!k_dev || !v_dev || !slots_dev || T < 1 || ldk < row || ldv < row) return MDBF_EINVAL;
  if (!kv_aligned(k_dev, 16) || !kv_aligned(v_dev, 16) || !kv_aligned(slots_dev, 8)) return MDBF_EALIGN;
  QkvArgs a = {};
  a.k = k_dev, a.v = v_dev, a.cache = (uint8_t*)cache_dev, a.slots = slots_dev;
  a.ldk = ldk, a.ldv = ldv, a.slot_count = (int64_t)kv->pages * kv->page_size;
  a.T = T, a.kv_heads = kv->kv_heads, a.page_shift = kv_page_shift(kv->page_size), a.kv_dt = kv->dtype;
  a.units = 2 * kv->kv_heads;
  a.wide_k = wide_rows(ldk, x_dtype), a.wide_v = wide_rows(ldv, x_dtype);
  return hip_fail(launch_qkv(x_dtype, MDBF_F32, kv->head_dim, a, (hipStream_t)stream));
}

int mdbf_kv_read(const mdbf_kv_t* kv, const void* cache_dev, size_t cache_bytes, const int64_t* slots_dev, int T,
                 void* k_dev, int64_t ldk, void* v_dev, int64_t ldv, int y_dtype, void* stream) {
  int st = check_kv_cache(kv, cache_dev, cache_bytes);
  if (st) return st;
  if (!valid_dtype(y_dtype)) return MDBF_EDTYPE;
  const int64_t row = (int64_t)kv->kv_heads * kv->head_dim;
  if (!k_dev || !v_dev || !slots_dev || T < 1 || ldk < row || ldv < row) return MDBF_EINVAL;
  if (!kv_aligned(k_dev, 16) || !kv_aligned(v_dev, 16) || !kv_aligned(slots_dev, 8)) return MDBF_EALIGN;
  ReadArgs a;
  a.cache = (const uint8_t*)cache_dev, a.slots = slots_dev, a.k = k_dev, a.v = v_dev, a.ldk = ldk, a.ldv = ldv;
  a.slot_count = (int64_t)kv->pages * kv->page_size, a.T = T, a.kv_heads = kv->kv_heads;
  a.page_shift = kv_page_shift(kv->page_size), a.scale_max = kKvScaleMax[kv->dtype];
  a.wide_k = wide_rows(ldk, y_dtype), a.wide_v = wide_rows(ldv, y_dtype);
  a.stream = 2 * (int64_t)T * row * dtype_size(y_dtype) > kStreamBytes;
  if (y_dtype == MDBF_F16) launch_read_d<MDBF_F16>(kv->head_dim, a, (hipStream_t)stream);
  else if (y_dtype == MDBF_BF16) launch_read_d<MDBF_BF16>(kv->head_dim, a, (hipStream_t)stream);
  else launch_read_d<MDBF_F32>(kv->head_dim, a, (hipStream_t)stream);
  return hip_fail((int)hipGetLastError());
}

int mdbf_qk_norm_rope(const mdbf_rope_t* desc, const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk,
                      const float* q_weight_dev, const float* k_weight_dev, const float* rope_dev,
                      const int32_t* positions_dev, int T, void* q_out_dev, int64_t ldqo, void* k_out_dev, int64_t ldko,
                      const mdbf_kv_t* kv, void* cache_dev, size_t cache_bytes, const void* v_dev, int64_t ldv,
                      const int64_t* slots_dev, void* stream) {
  if (!desc) return MDBF_EINVAL;
  const int d = desc->head_dim;
  if (desc->q_heads <= 0 || desc->kv_heads <= 0 || d <= 0 || desc->rot_dim < 0 || desc->rot_dim > d) return MDBF_EINVAL;
  if (!valid_dtype(desc->x_dtype) || !valid_dtype(desc->y_dtype)) return MDBF_EDTYPE;
  if (!valid_head_dim(d) || desc->rot_dim % 16 || (desc->flags & ~MDBF_ROPE_INTERLEAVED) || desc->q_heads > (1 << 16) ||
      desc->kv_heads > (1 << 16))
    return MDBF_EUNSUPPORTED;
  const int64_t rowq = (int64_t)desc->q_heads * d, rowk = (int64_t)desc->kv_heads * d;
  if (!q_dev || !k_dev || !q_out_dev || T < 1 || ldq < rowq || ldk < rowk || ldqo < rowq) return MDBF_EINVAL;
  if ((k_out_dev && ldko < rowk) || (!k_out_dev && !kv) || !(desc->eps >= 0.0f)) return MDBF_EINVAL;
  if (desc->rot_dim && (!rope_dev || !positions_dev || desc->rope_rows < 1)) return MDBF_EINVAL;
  const void* ptrs[] = {q_dev, k_dev, q_weight_dev, k_weight_dev, rope_dev, q_out_dev, k_out_dev};
  for (const void* p : ptrs)
    if (!kv_aligned(p, 16)) return MDBF_EALIGN;
  if (!kv_aligned(positions_dev, 4)) return MDBF_EALIGN;
  QkvArgs a = {};
  if (kv) {
    int st = check_kv_cache(kv, cache_dev, cache_bytes);
    if (st) return st;
    if (kv->kv_heads != desc->kv_heads || kv->head_dim != d || !v_dev || !slots_dev || ldv < rowk) return MDBF_EINVAL;
    if (!kv_aligned(v_dev, 16) || !kv_aligned(slots_dev, 8)) return MDBF_EALIGN;
    a.v = v_dev, a.ldv = ldv, a.wide_v = wide_rows(ldv, desc->x_dtype);
    a.cache = (uint8_t*)cache_dev, a.slots = slots_dev, a.slot_count = (int64_t)kv->pages * kv->page_size;
    a.page_shift = kv_page_shift(kv->page_size), a.kv_dt = kv->dtype;
  }
  a.q = q_dev, a.k = k_dev, a.qw = q_weight_dev, a.kw = k_weight_dev, a.rope = rope_dev, a.positions = positions_dev;
  a.q_out = q_out_dev, a.k_out = k_out_dev, a.ldq = ldq, a.ldk = ldk, a.ldqo = ldqo, a.ldko = ldko;
  a.T = T, a.q_heads = desc->q_heads, a.kv_heads = desc->kv_heads, a.rot = desc->rot_dim, a.rope_rows = desc->rope_rows;
  a.units = desc->q_heads + desc->kv_heads * (kv ? 2 : 1);
  a.stream = (int64_t)T * (rowq + rowk) * dtype_size(desc->y_dtype) > kStreamBytes;
  a.interleaved = desc->flags & MDBF_ROPE_INTERLEAVED, a.eps = desc->eps;
  a.wide_q = wide_rows(ldq, desc->x_dtype), a.wide_k = wide_rows(ldk, desc->x_dtype);
  a.wide_qo = wide_rows(ldqo, desc->y_dtype), a.wide_ko = wide_rows(ldko, desc->y_dtype);
  return hip_fail(launch_qkv(desc->x_dtype, desc->y_dtype, d, a, (hipStream_t)stream));
}

}  // extern "C"
