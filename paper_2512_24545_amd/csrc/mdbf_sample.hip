// The next token of each row of logits: temperature, top-k, top-p, min-p, and the draw from a given number.
#include <math.h>

#include "mdbf_rows.h"

namespace mdbf {

constexpr int kSampleMaxVocab = 1 << 20;

struct SampleArgs {
  const void* logits;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  int64_t ld;
  int32_t T, vocab;
};

// Logits as whole numbers of the same order; NaN is -inf, -0 is 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (!(x == x)) x = -__builtin_inff();
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
constexpr uint32_t kKeyNone = 0x007fffffu;      // -inf

// a row's settings
struct RowSetting {
  double largest, per_degree, top_p, min_p, u;
  uint32_t top, top_k;
  bool greedy;
};
__device__ __forceinline__ RowSetting row_setting(const SampleArgs& a, int64_t t, uint32_t top) {
  RowSetting r;
  const float temperature = a.temperature ? a.temperature[t] : 1.0f;
  r.greedy = !(temperature > 0.0f);
  r.per_degree = 1.0 / (double)temperature;
  r.top = top;
  r.largest = (double)key_value(top);
  const int k = a.top_k ? a.top_k[t] : 0;
  r.top_k = k > 0 && k < a.vocab ? (uint32_t)k : 0;
  const float p = a.top_p ? a.top_p[t] : 1.0f, least = a.min_p ? a.min_p[t] : 0.0f, u = a.u[t];
  r.top_p = p < 1.0f ? (double)p : 1.0;        // (NaN: no bound)
  r.min_p = least > 0.0f ? (double)least : 0.0;
  r.u = u > 0.0f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0;
  return r;
}
// the weight of a logit
__device__ __forceinline__ double weight(const RowSetting& r, uint32_t key) {
  if (key == r.top) return 1.0;
  if (key <= kKeyNone || r.top == 0xff800000u) return 0.0;
  return exp(((double)key_value(key) - r.largest) * r.per_degree);
}

template <int DT>
__device__ __forceinline__ uint32_t key_at(const SampleArgs& a, int64_t t, int i) {
  return order_key(load_as_float(a.logits, t * a.ld + i, DT));
}

constexpr int kPickThreads = 1024;
constexpr double kUnit = 0x1p43;                // weights as whole numbers: their sums do not go by the order of the additions

struct PickShared {
  uint32_t count[256];
  unsigned long long mass[256];
  unsigned long long sum[kPickThreads / 64];
  uint32_t top[kPickThreads / 64];
  uint32_t digit, count_before;
  unsigned long long mass_before;
};

// The place in the order of keys at which the number of tokens reaches `count`, or else their mass reaches `mass` (or goes beyond it).  Four
// digits of eight bits, the largest first.
struct Place {
  uint32_t key, ties, before;                   // of equal keys there are `ties`; tokens and mass in front of them
  unsigned long long mass_before;
};
template <int DT>
__device__ Place descend(const SampleArgs& a, int64_t t, const RowSetting& r, PickShared& s, uint32_t count, double mass, bool beyond) {
  const int tid = threadIdx.x, lane = tid & 63;
  Place at = {0, 0, 0, 0};
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) s.count[tid] = 0, s.mass[tid] = 0;
    __syncthreads();
    for (int i = tid; i < a.vocab; i += kPickThreads) {
      const uint32_t k = key_at<DT>(a, t, i);
      if (shift < 24 && ((k ^ at.key) >> (shift + 8))) continue;
      atomicAdd(&s.count[(k >> shift) & 255], 1u);
      const unsigned long long w = (unsigned long long)(weight(r, k) * kUnit);
      if (w) atomicAdd(&s.mass[(k >> shift) & 255], w);
    }
    __syncthreads();
    if (tid < 64) {
      uint32_t c = 0;
      unsigned long long m = 0;
      for (int q = 0; q < 4; ++q) c += s.count[255 - lane * 4 - q], m += s.mass[255 - lane * 4 - q];
      uint32_t c_to = c;
      unsigned long long m_to = m;
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t uc = __shfl_up(c_to, o);
        const unsigned long long um = __shfl_up(m_to, o);
        if (lane >= o) c_to += uc, m_to += um;
      }
      c_to += at.before, m_to += at.mass_before;
      const bool here = c && (count ? c_to >= count : beyond ? (double)m_to > mass : (double)m_to >= mass);
      const unsigned long long hit = __ballot(here), any = __ballot(c != 0);
      const int who = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(any);
      if (lane == who) {
        uint32_t cb = c_to - c;
        unsigned long long mb = m_to - m;
        for (int q = 0; q < 4; ++q) {
          const uint32_t b = 255 - lane * 4 - q, cc = s.count[b];
          if (!cc) continue;
          s.digit = b, s.count_before = cb, s.mass_before = mb;
          const double m2 = (double)(mb + s.mass[b]);
          if (count ? cb + cc >= count : beyond ? m2 > mass : m2 >= mass) break;
          cb += cc, mb += s.mass[b];
        }
      }
    }
    __syncthreads();
    at.key |= s.digit << shift;
    at.before = s.count_before, at.mass_before = s.mass_before;
    at.ties = s.count[s.digit];
  }
  return at;
}

// One workgroup a row, the row read again for every digit.
template <int DT>
__global__ __launch_bounds__(kPickThreads) void sample_kernel(SampleArgs a) {
  __shared__ PickShared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  uint32_t top = 0;
  for (int i = tid; i < a.vocab; i += kPickThreads) top = max(top, key_at<DT>(a, t, i));
  for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if (lane == 0) s.top[wave] = top;
  __syncthreads();
  for (int w = 0; w < kPickThreads / 64; ++w) top = max(top, s.top[w]);
  if (top <= kKeyNone) {
    if (tid == 0) {
      a.tokens[t] = -1;
      if (a.probs) a.probs[t] = 0.0f;
    }
    return;
  }
  const RowSetting r = row_setting(a, t, top);
  uint32_t key = top, tie = 0;
  double prob = 1.0;
  if (!r.greedy) {
    // what is kept is a first part of the order, and so is what each bound leaves: the least of their masses
    unsigned long long total = 0, likely = 0;
    for (int i = tid; i < a.vocab; i += kPickThreads) {
      const double x = weight(r, key_at<DT>(a, t, i));
      const unsigned long long w = (unsigned long long)(x * kUnit);
      total += w;
      if (x >= r.min_p) likely += w;
    }
    for (int q = 0; q < 2; ++q) {
      unsigned long long v = q ? likely : total;
      for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
      __syncthreads();
      if (lane == 0) s.sum[wave] = v;
      __syncthreads();
      v = 0;
      for (int w = 0; w < kPickThreads / 64; ++w) v += s.sum[w];
      (q ? likely : total) = v;
    }
    double kept = (double)total;
    if (r.top_k) {
      const Place p = descend<DT>(a, t, r, s, r.top_k, 0.0, false);
      kept = (double)p.mass_before + (double)(r.top_k - p.before) * (weight(r, p.key) * kUnit);
    }
    double least = kept;
    if (r.top_p < 1.0) {
      const double mass = r.top_p * kept;
      const Place p = descend<DT>(a, t, r, s, 0, mass, false);
      const double w = weight(r, p.key) * kUnit, b = (double)p.mass_before;
      double j = w > 0 ? ceil((mass - b) / w) : 1.0;
      j = fmin(fmax(j, 1.0), (double)p.ties);
      least = fmin(least, b + j * w);
    }
    if (r.min_p > 0.0) least = fmin(least, fmax((double)likely, kUnit));
    kept = least;
    const double mass = r.u * kept;
    const Place p = descend<DT>(a, t, r, s, 0, mass, true);
    const double w = weight(r, p.key) * kUnit, b = (double)p.mass_before;
    key = p.key;
    const double j = w > 0 ? floor((mass - b) / w) : 0.0;
    tie = (uint32_t)fmin(fmax(j, 0.0), (double)(p.ties - 1));
    prob = w / kept;
  }
  // the index of that one among equal logits
  __shared__ uint32_t found[kPickThreads / 64];
  uint32_t before = 0;
  for (int i0 = 0; i0 < a.vocab; i0 += kPickThreads) {
    const int i = i0 + tid;
    const bool eq = i < a.vocab && key_at<DT>(a, t, i) == key;
    const unsigned long long b = __ballot(eq);
    __syncthreads();
    if (lane == 0) found[wave] = __popcll(b);
    __syncthreads();
    uint32_t mine = before, all = before;
    for (int w = 0; w < kPickThreads / 64; ++w) {
      if (w < wave) mine += found[w];
      all += found[w];
    }
    if (eq && mine + __popcll(b & ((1ull << lane) - 1)) == tie) {
      a.tokens[t] = i;
      if (a.probs) a.probs[t] = (float)prob;
    }
    if (all > tie) break;
    before = all;
  }
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_sample_workspace_bytes(int T, int vocab, size_t* bytes_out) {
  if (T < 1 || vocab < 1 || !bytes_out) return MDBF_EINVAL;
  if (vocab > kSampleMaxVocab) return MDBF_EUNSUPPORTED;
  *bytes_out = 0;
  return MDBF_OK;
}

int mdbf_sample(const mdbf_sample_t* settings, const void* logits_dev, int64_t ld, int dtype, int T, int vocab, const float* u_dev,
                int32_t* tokens_dev, float* probs_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int st = mdbf_sample_workspace_bytes(T, vocab, &need);
  if (st) return st;
  if (!row_dtype(dtype)) return MDBF_EDTYPE;
  if (!settings || !logits_dev || !u_dev || !tokens_dev || ld < vocab || (need && !workspace_dev)) return MDBF_EINVAL;
  if (!ptr_aligned(logits_dev, 16) || !ptr_aligned(workspace_dev, 16)) return MDBF_EALIGN;
  const void* ptrs[] = {settings->temperature_dev, settings->top_k_dev, settings->top_p_dev, settings->min_p_dev, u_dev, tokens_dev, probs_dev};
  for (const void* p : ptrs)
    if (!ptr_aligned(p, 4)) return MDBF_EALIGN;
  if (workspace_bytes < need) return MDBF_EWORKSPACE;
  const SampleArgs a = {logits_dev, settings->temperature_dev, settings->top_p_dev, settings->min_p_dev, u_dev, settings->top_k_dev,
                        tokens_dev, probs_dev, ld, T, vocab};
  if (dtype == MDBF_F16) sample_kernel<MDBF_F16><<<T, kPickThreads, 0, (hipStream_t)stream>>>(a);
  else if (dtype == MDBF_BF16) sample_kernel<MDBF_BF16><<<T, kPickThreads, 0, (hipStream_t)stream>>>(a);
  else sample_kernel<MDBF_F32><<<T, kPickThreads, 0, (hipStream_t)stream>>>(a);
  return hip_fail((int)hipGetLastError());
}

}  // extern "C"
