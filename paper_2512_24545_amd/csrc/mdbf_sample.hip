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
  double largest, per_degree, grid, top_p, min_p, u;
  uint32_t top, top_k;
  bool greedy;
};
__device__ __forceinline__ RowSetting row_setting(const SampleArgs& a, int64_t t, uint32_t top) {
  RowSetting r;
  const float temperature = a.temperature ? a.temperature[t] : 1.0f;
  r.greedy = !(temperature > 0.0f);
  r.per_degree = 1.0 / (double)temperature;
  r.grid = 16 * 1.44269504088896340736 / (double)temperature;   // sixteenths of a factor of two per unit of the logits
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
  uint32_t found[kPickThreads / 64];
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
}// A row that nothing else serves: read again for every digit.
template <int DT>
__device__ void sample_digits(const SampleArgs& a, int64_t t, const RowSetting& r, PickShared& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t key = r.top, tie = 0;
  double prob = 1.0;
  {
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
  uint32_t before = 0;
  for (int i0 = 0; i0 < a.vocab; i0 += kPickThreads) {
    const int i = i0 + tid;
    const bool eq = i < a.vocab && key_at<DT>(a, t, i) == key;
    const unsigned long long b = __ballot(eq);
    __syncthreads();
    if (lane == 0) s.found[wave] = __popcll(b);
    __syncthreads();
    uint32_t mine = before, all = before;
    for (int w = 0; w < kPickThreads / 64; ++w) {
      if (w < wave) mine += s.found[w];
      all += s.found[w];
    }
    if (eq && mine + __popcll(b & ((1ull << lane) - 1)) == tie) {
      a.tokens[t] = i;
      if (a.probs) a.probs[t] = (float)prob;
    }
    if (all > tie) break;
    before = all;
  }
}

// ---- the two launches -----------------------------------------------------------------------------------
// With t = logit * 16 log2(e) / temperature a weight is 2^(t / 16) over the largest one's.  The first launch sorts the tokens of each part of a row into buckets
// of a sixteenth of a factor of two, floor(t), from the part's largest down, and sums there how many they are and their 2^(frac(t) / 16): one 64-bit whole
// number a bucket, whose additions in LDS have no order.  The buckets of all parts of a row lie on one grid, so the second launch, a workgroup a
// row, adds them up; prefix sums then tell in which bucket each bound and the drawn number lie.  Only the tokens of those few are looked
// at by themselves: parts that have some are read again, their tokens put in order, and the bounds applied exactly.  Tokens that equal the part's
// largest are counted apart, so that those that equal the row's largest, of weight 1, make up a bucket of an exact mass: where many are alike,
// bounds fall on borders between them.
constexpr int kBuckets = 768;                    // of a row: the largest, then 767 sixteenths, down to 2^-47 of it; less weighs nothing
constexpr int kPerOctave = 16;
constexpr int kFracBits = 39;                    // of 2^(frac / 16) - 1 < 0.0443: 16384 of them stay below 2^49, where the count begins
constexpr int kCountBit = 49;
constexpr int kList = 8192;                      // tokens that the second launch puts in order; rows that have more go by digits
constexpr int kPartThreads = 1024;
constexpr double kSlack = 1e-9;                  // by which sums of buckets and of tokens may differ, and more

struct PartHead {
  unsigned long long top;                        // key of the part's largest, ~its index: the largest with the lowest index is the largest number
  unsigned long long equal;                      // tokens that equal it
};

__device__ __forceinline__ double degrees(const RowSetting& r, float x) { return (double)x * r.grid; }

// 2^(x / 16) - 1 for x in [0, 1): the exponential's series, to 6e-14
__device__ __forceinline__ double sixteenth(double x) {
  constexpr double q = 0.69314718055994530942 / kPerOctave;
  constexpr double c1 = q, c2 = q * q / 2, c3 = q * q * q / 6, c4 = q * q * q * q / 24, c5 = q * q * q * q * q / 120, c6 = q * q * q * q * q * q / 720;
  return x * fma(x, fma(x, fma(x, fma(x, fma(x, c6, c5), c4), c3), c2), c1);
}

template <int DT, int EPT>
__global__ __launch_bounds__(kPartThreads) void sample_parts_kernel(SampleArgs a, PartHead* heads, unsigned long long* hists) {
  __shared__ unsigned long long hist[kBuckets];
  __shared__ unsigned long long tops[kPartThreads / 64];
  __shared__ uint32_t equal;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.y, part = t * gridDim.x + blockIdx.x;
  const int i0 = blockIdx.x * (kPartThreads * EPT);

  Raw8<DT> raw[EPT / 8];
#pragma unroll
  for (int p = 0; p < EPT / 8; ++p) {
    const int i = i0 + (p * kPartThreads + tid) * 8;
    if (i < a.vocab) load_raw8<DT>(a.logits, t * a.ld + i, a.vocab - i, raw[p]);
  }
  for (int o = tid; o < kBuckets; o += kPartThreads) hist[o] = 0;
  if (tid == 0) equal = 0;
  float v[EPT], best = -__builtin_inff();
  int at = 0x7fffffff;
#pragma unroll
  for (int p = 0; p < EPT / 8; ++p) {
    const int i = i0 + (p * kPartThreads + tid) * 8;
    float x[8];
    to_float8<DT>(raw[p], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = i + e < a.vocab && x[e] == x[e] ? x[e] : -__builtin_inff();
      v[p * 8 + e] = y;
      if (y > best) best = y, at = i + e;
    }
  }
  unsigned long long top = (unsigned long long)order_key(best) << 32 | (uint32_t)~at;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long u = __shfl_xor(top, o);
    if (u > top) top = u;
  }
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPartThreads / 64; ++w)
    if (tops[w] > top) top = tops[w];
  if (tid == 0) heads[part].top = top;
  const uint32_t key = (uint32_t)(top >> 32);
  const RowSetting r = row_setting(a, t, key);
  if (key <= kKeyNone || r.greedy) return;
  const float largest = key_value(key);
  const bool infinite = largest == __builtin_inff();    // then nothing else weighs
  const double base = floor(degrees(r, largest));
  uint32_t alike = 0;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const bool same = v[e] == largest;
    alike += (uint32_t)__popcll(__ballot(same));
    if (infinite || same) continue;
    const double d = degrees(r, v[e]), f = floor(d), down = base - f;
    if (down < kBuckets && v[e] > -__builtin_inff()) {
      // (the sum with 2^52 has the whole number in its last bits)
      const double g = fma(sixteenth(d - f), (double)(1ull << kFracBits), 0x1p52);
      atomicAdd(&hist[(int)down], __builtin_bit_cast(unsigned long long, g) - 0x4330000000000000ull + (1ull << kCountBit));
    }
  }
  if (lane == 0) atomicAdd(&equal, alike);
  __syncthreads();
  if (tid == 0) heads[part].equal = equal;
  for (int o = tid; o < kBuckets; o += kPartThreads) hists[part * kBuckets + o] = hist[o];
}

// What the second launch has in LDS.
constexpr int kRuns = 4;                         // runs of neighbouring buckets that are looked at
constexpr int kMaxParts = kSampleMaxVocab / (kPartThreads * 8);
struct RowShared {
  unsigned long long list[kList];                // ~key, index: the order of the tokens
  double before[kBuckets], seg_mass[kBuckets];   // mass in front of a bucket, and of the list in front of a bucket's first
  uint32_t count_before[kBuckets], seg_at[kBuckets];
  unsigned long long flags[kBuckets / 64];
  double sums[kPickThreads / 64];
  uint32_t counts[kPickThreads / 64];
  unsigned long long tops[kPickThreads / 64];
  unsigned long long part_extra[kMaxParts];      // of a part: its largest's bucket in the row (kBuckets: nothing there weighs), how many equal it, and
  int32_t part_top[kMaxParts];                   // their fractions
  uint32_t part_equal[kMaxParts], part_list[kMaxParts];
  double klo, khi, plo, phi, mlo, mhi, total;
  int k, p0, p1, m0, m1, u0, u1;
  float lower[kRuns], upper[kRuns];
  uint32_t n, parts, runs, dropped;
};

// what the wave wrote in LDS, or the workgroup, is there for all of it
template <int THREADS>
__device__ __forceinline__ void meet() {
  if (THREADS > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
  }
}

// The value of the last (or first) thread for which `here` holds, where it rises with the threads; else `none`.
template <int THREADS, bool FIRST>
__device__ __forceinline__ double end_of(bool here, double v, double none, double* part) {
  const unsigned long long b = __ballot(here);
  const int who = !b ? 0 : FIRST ? __builtin_ctzll(b) : 63 - __builtin_clzll(b);
  if (THREADS == 64) return b ? __shfl(v, who) : none;
  __syncthreads();
  if ((int)(threadIdx.x & 63) == who) part[threadIdx.x >> 6] = b ? v : none;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = FIRST ? fmin(v, part[w]) : fmax(v, part[w]);
  return v;
}

// Which buckets have to be looked at: those of the bounds and of the drawn number, the latter ones' ends by the least and the most that the bounds
// may leave.  k, p0 .., m0 .., u0 .. are set to no bound before.
__device__ __forceinline__ void choose_buckets(const RowSetting& r, RowShared& s, double before, double upto, uint32_t count_before, uint32_t count_to,
                                               double frac) {
  const int o = threadIdx.x;
  const bool in = o < kBuckets;
  if (in && r.top_k && count_before < r.top_k && count_to >= r.top_k) s.k = o, s.klo = before, s.khi = upto;
  if (r.min_p > 0.0 && in) {
    const double last = -floor(frac + kPerOctave * log2(r.min_p));      // the bucket of that weight, or its neighbour, is `last` + 1
    const int m0 = (int)fmin(fmax(last, 0.0), (double)kBuckets), m1 = (int)fmin(fmax(last + 2, 0.0), (double)(kBuckets - 1));
    if (m0 < kBuckets) {
      if (o == m0) s.m0 = o, s.mlo = before;
      if (o == m1) s.m1 = o, s.mhi = upto;
    }
  }
  __syncthreads();
  const double klo = fmin(s.klo, s.total), khi = fmin(s.khi, s.total);
  if (r.top_p < 1.0) {
    const double lo = r.top_p * klo * (1 - kSlack), hi = r.top_p * khi * (1 + kSlack);
    if (in && before < lo && upto >= lo) s.p0 = o, s.plo = before;
    if (in && before <= hi && upto > hi) s.p1 = o, s.phi = upto;
  }
  __syncthreads();
  const double ulo = r.u * fmin(klo, fmin(s.plo, s.mlo)) * (1 - kSlack), uhi = r.u * fmin(khi, fmin(s.phi, s.mhi)) * (1 + kSlack);
  if (in && before <= ulo && upto > ulo) s.u0 = o;
  if (in && before <= uhi && upto > uhi) s.u1 = o;
  __syncthreads();
  // (a bound that another one is sure to undercut needs none of its tokens)
  const bool least = s.mlo >= fmin(khi, s.phi), other = s.mhi <= fmin(klo, s.plo);
  const bool flag = in && ((!other && (o == s.k || (o >= s.p0 && o <= s.p1))) || (!least && o >= s.m0 && o <= s.m1) || (o >= s.u0 && o <= s.u1));
  const unsigned long long b = __ballot(flag);
  if (in && (o & 63) == 0) s.flags[o >> 6] = b;
  __syncthreads();
}
__device__ __forceinline__ bool flagged(const RowShared& s, int b) { return s.flags[b >> 6] >> (b & 63) & 1; }

// The list in order, bitonic: a wave sorts and merges 64 neighbours in registers, what is further apart meets in LDS.
__device__ __forceinline__ unsigned long long exchange(unsigned long long v, int x, int j, int k) {
  const unsigned long long u = __shfl_xor(v, j);
  return ((x & j) == 0) == ((x & k) == 0) ? (u < v ? u : v) : (u < v ? v : u);
}
template <int THREADS>
__device__ __forceinline__ void sort_list(RowShared& s, int n) {
  const int tid = threadIdx.x;
  if (THREADS == 64) {                          // so few that each counts those in front of it
    const unsigned long long v = tid < n ? s.list[tid] : ~0ull;
    int place = 0;
    for (int j = 0; j < n; ++j) place += __shfl(v, j) < v;
    meet<64>();
    if (v != ~0ull) s.list[place] = v;         // (those left out are alike)
    meet<64>();
    return;
  }
  int size = 64;
  while (size < n) size <<= 1;
  for (int x = tid; x < size; x += THREADS) {
    unsigned long long v = x < n ? s.list[x] : ~0ull;
#pragma unroll
    for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
      for (int j = k >> 1; j > 0; j >>= 1) v = exchange(v, x, j, k);
    s.list[x] = v;
  }
  for (int k = 128; k <= size; k <<= 1) {
    for (int j = k >> 1; j >= 64; j >>= 1) {
      meet<THREADS>();
      for (int i = tid; i < size / 2; i += THREADS) {
        const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x | j;
        const unsigned long long p = s.list[x], q = s.list[y];
        if ((p > q) == ((x & k) == 0)) s.list[x] = q, s.list[y] = p;
      }
    }
    meet<THREADS>();
    for (int x = tid; x < size; x += THREADS) {
      unsigned long long v = s.list[x];
#pragma unroll
      for (int j = 32; j > 0; j >>= 1) v = exchange(v, x, j, k);
      s.list[x] = v;
    }
  }
  meet<THREADS>();
}

// The bounds and the draw on the list, `taken` entries of which n count, by THREADS threads with up to PER tokens each.
template <int THREADS, int PER, class Bucket>
__device__ __forceinline__ void pick(const SampleArgs& a, int64_t t, const RowSetting& r, RowShared& s, int taken, int n, const Bucket& bucket_of) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  sort_list<THREADS>(s, taken);
  // each thread has a run of the list
  const int per = (n + THREADS - 1) / THREADS, x0 = min(tid * per, n), x1 = min(x0 + per, n);
  double w[PER], sum = 0;
  int bucket[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    if (x0 + q < x1) {
      const uint32_t k = ~(uint32_t)(s.list[x0 + q] >> 32);
      w[q] = weight(r, k);
      bucket[q] = bucket_of(key_value(k));
      sum += w[q];
    }
  }
  double run = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = __shfl_up(run, o);
    if (lane >= o) run += u;
  }
  if (THREADS > 64) {
    if (lane == 63) s.sums[wave] = run;
    __syncthreads();
  }
  run -= sum;
  if (THREADS > 64)
    for (int v = 0; v < wave; ++v) run += s.sums[v];
  double at[PER];                               // mass of the list in front of a token
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    if (x0 + q < x1) {
      at[q] = run;
      run += w[q];
      const int x = x0 + q, prev = x > 0 ? bucket_of(key_value(~(uint32_t)(s.list[x - 1] >> 32))) : -1;
      if (prev != bucket[q]) s.seg_mass[bucket[q]] = at[q], s.seg_at[bucket[q]] = x;
    }
  }
  meet<THREADS>();
#pragma unroll
  for (int q = 0; q < PER; ++q)
    if (x0 + q < x1) at[q] = s.before[bucket[q]] + (at[q] - s.seg_mass[bucket[q]]);
  const auto rank = [&](int q) { return s.count_before[bucket[q]] + (uint32_t)(x0 + q) - s.seg_at[bucket[q]]; };
  // what is kept is a first part of the order, and so is what each bound leaves: the least of their masses
  double kept = s.total;
  const bool least = s.mlo >= fmin(s.khi, fmin(s.phi, s.total)), other = s.mhi <= fmin(s.klo, fmin(s.plo, s.total));
  // (of a thread's tokens the last one that a bound leaves; `m` is none of them)
  const auto bound = [&](double m, auto holds) {
    bool some = false;
    double v = m;
#pragma unroll
    for (int q = 0; q < PER; ++q)
      if (x0 + q < x1 && holds(q)) some = true, v = fmax(v, at[q] + w[q]);
    return end_of<THREADS, false>(some, v, m, s.sums);
  };
  if (s.k >= 0 && !other) kept = bound(s.klo, [&](int q) { return bucket[q] == s.k && rank(q) < r.top_k; });
  if (r.top_p < 1.0 && !other) {
    const double mass = r.top_p * kept;
    kept = bound(s.plo, [&](int q) { return bucket[q] >= s.p0 && bucket[q] <= s.p1 && (at[q] < mass || rank(q) == 0); });
  }
  if (s.m1 >= 0 && !least)
    kept = fmin(kept, bound(s.mlo, [&](int q) { return bucket[q] >= s.m0 && bucket[q] <= s.m1 && (w[q] >= r.min_p || rank(q) == 0); }));
  const double drawn = r.u * kept;
  // the first that goes beyond it (or the last there is, if only the sums' rounding keeps that from it)
  constexpr double kNone = 1e9;
  double first = kNone, last = -1;
#pragma unroll
  for (int q = 0; q < PER; ++q)
    if (x0 + q < x1 && bucket[q] >= s.u0 && bucket[q] <= s.u1) {
      last = x0 + q;
      if (at[q] + w[q] > drawn) first = fmin(first, x0 + q);
    }
  first = end_of<THREADS, true>(first < kNone, first, kNone, s.sums);
  if (first == kNone) first = end_of<THREADS, false>(last >= 0, last, 0.0, s.sums);
  const int x = (int)first;
  if (x >= x0 && x < x1) {
    const unsigned long long it = s.list[x];
    a.tokens[t] = (int)(uint32_t)it;
    if (a.probs) a.probs[t] = (float)(weight(r, ~(uint32_t)(it >> 32)) / kept);
  }
}

template <int DT>
__global__ __launch_bounds__(kPickThreads) void sample_rows_kernel(SampleArgs a, const PartHead* heads, const unsigned long long* hists, int parts, int part_size) {
  extern __shared__ char shared[];
  RowShared& s = *(RowShared*)shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  unsigned long long top = 0;
  for (int c = tid; c < parts; c += kPickThreads) {
    const unsigned long long u = heads[t * parts + c].top;
    if (u > top) top = u;
  }
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long u = __shfl_xor(top, o);
    if (u > top) top = u;
  }
  if (lane == 0) s.tops[wave] = top;
  if (tid == 0) {
    s.n = s.parts = s.dropped = s.runs = 0;
    s.k = -1, s.p0 = s.m0 = s.u0 = 0, s.m1 = -1, s.u1 = kBuckets - 1;
    s.klo = s.khi = s.phi = s.mlo = s.mhi = INFINITY;
  }
  __syncthreads();
  for (int w = 0; w < kPickThreads / 64; ++w)
    if (s.tops[w] > top) top = s.tops[w];
  const uint32_t key = (uint32_t)(top >> 32);
  const RowSetting r = row_setting(a, t, key);
  if (key <= kKeyNone || r.greedy) {
    if (tid == 0) {
      a.tokens[t] = key <= kKeyNone ? -1 : (int)~(uint32_t)top;
      if (a.probs) a.probs[t] = key <= kKeyNone ? 0.0f : 1.0f;
    }
    return;
  }
  const float largest = key_value(key);
  const bool infinite = largest == __builtin_inff();
  const double most = infinite ? 0.0 : degrees(r, largest), base = floor(most), frac = most - base;

  const auto bucket_of = [&](float x) { return x == largest ? 0 : 1 + (int)fmin(base - floor(degrees(r, x)), (double)kBuckets); };

  for (int c = tid; c < parts; c += kPickThreads) {
    const PartHead h = heads[t * parts + c];
    const float its = key_value((uint32_t)(h.top >> 32));
    const bool none = its == -__builtin_inff() || (infinite && its != largest);
    const int b = none ? kBuckets : min(bucket_of(its), kBuckets);
    const double d = degrees(r, its);
    s.part_top[c] = b, s.part_equal[c] = (uint32_t)h.equal;
    s.part_extra[c] = b == 0 || none ? 0 : (uint32_t)h.equal * (unsigned long long)(sixteenth(d - floor(d)) * (double)(1ull << kFracBits) + 0.5);
  }
  __syncthreads();

  // a thread's bucket, of all parts (a part's begin with that of its largest, of the row's with bucket 1)
  uint32_t count = 0;
  unsigned long long extra = 0;
  if (tid < kBuckets) {
    constexpr int U = 8;
    const unsigned long long* row = hists + t * parts * kBuckets;
    for (int c0 = 0; c0 < parts; c0 += U) {
      unsigned long long h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u, shift = c < parts && !infinite ? max(s.part_top[c], 1) : kBuckets;
        h[u] = tid >= shift ? row[(int64_t)c * kBuckets + tid - shift] : 0;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u;
        count += (uint32_t)(h[u] >> kCountBit);
        extra += h[u] & ((1ull << kCountBit) - 1);
        if (c < parts && tid == s.part_top[c]) count += s.part_equal[c], extra += s.part_extra[c];
      }
    }
  }
  const double mass = tid == 0 ? (double)count
                               : ((double)count + (double)extra * (1.0 / (double)(1ull << kFracBits))) * exp2(-(tid - 1 + frac) / kPerOctave);
  uint32_t count_to = count;
  double upto = mass;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t uc = __shfl_up(count_to, o);
    const double um = __shfl_up(upto, o);
    if (lane >= o) count_to += uc, upto += um;
  }
  if (lane == 63) s.sums[wave] = upto, s.counts[wave] = count_to;
  __syncthreads();
  double wave_before = 0, total = 0;
  uint32_t waves_count = 0;
  for (int w = 0; w < kBuckets / 64; ++w) {
    if (w == wave) wave_before = total;
    if (w < wave) waves_count += s.counts[w];
    total += s.sums[w];
  }
  // (the sum in front of a bucket is that up to the one before it, bit for bit)
  const double inside = __shfl_up(upto, 1);
  const double before = lane ? wave_before + inside : wave_before;
  upto += wave_before, count_to += waves_count;
  if (tid < kBuckets) s.before[tid] = before, s.count_before[tid] = count_to - count;
  if (tid == 0) s.total = total, s.p1 = r.top_p < 1.0 ? kBuckets - 1 : -1, s.plo = r.top_p < 1.0 ? 0.0 : INFINITY;
  __syncthreads();
  choose_buckets(r, s, before, upto, count_to - count, count_to, frac);

  // parts that have tokens of those buckets
  for (int c = wave; c < parts; c += kPickThreads / 64) {
    const int top_bucket = s.part_top[c], shift = max(top_bucket, 1);
    if (top_bucket >= kBuckets) continue;
    bool some = flagged(s, top_bucket);
#pragma unroll
    for (int o = lane; o < kBuckets; o += 64)
      if (flagged(s, o) && o >= shift && !infinite && hists[(t * parts + c) * kBuckets + o - shift]) some = true;
    if (__any(some) && lane == 0) s.part_list[atomicAdd(&s.parts, 1u)] = c;
  }
  __syncthreads();
  // Runs of such buckets as bounds of the logits, with room for rounding: tokens are taken by these, and those that are of other
  // buckets after all left out afterwards.
  if (tid < kBuckets && flagged(s, tid)) {
    const bool from = tid == 0 || !flagged(s, tid - 1), to = tid == kBuckets - 1 || !flagged(s, tid + 1);
    uint32_t run = 0;
    for (int b = 0; b < kBuckets / 64; ++b) {            // runs that begin in front of this one, or with it
      const unsigned long long f = s.flags[b], starts = f & ~(f << 1 | (b ? s.flags[b - 1] >> 63 : 0));
      if (b * 64 <= tid) run += __popcll(tid - b * 64 >= 63 ? starts : starts & ((2ull << (tid - b * 64)) - 1));
    }
    const bool bounded = r.grid > 0 && !infinite;
    if (run <= kRuns) {
      if (from) {
        const double x = (base - tid + 2) / r.grid;
        s.upper[run - 1] = bounded && tid ? (float)(x + fabs(x) * 1e-6 + 1e-37) : INFINITY;
      }
      if (to) {
        const double x = (base - max(tid, 1) + 1) / r.grid;
        s.lower[run - 1] = bounded ? (float)(x - fabs(x) * 1e-6 - 1e-37) : -3.4028234e38f;
      }
    }
    if (to) atomicMax(&s.runs, run);
  }
  __syncthreads();
  const int runs = (int)s.runs;                  // (never more than kRuns: those of top_k, top_p, min_p and the draw)
  const float lo0 = s.lower[0], hi0 = s.upper[0], lo1 = runs > 1 ? s.lower[1] : INFINITY, hi1 = runs > 1 ? s.upper[1] : -INFINITY;
  const int per_part = part_size / 512, pieces = (int)s.parts * per_part;
  constexpr int U = DT == MDBF_F32 ? 2 : 4;
  for (int p0 = wave; p0 < pieces; p0 += U * (kPickThreads / 64)) {
    Raw8<DT> raw[U];
    int at[U], there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u * (kPickThreads / 64);
      at[u] = there[u] = 0;
      if (p < pieces) {
        at[u] = (int)s.part_list[p / per_part] * part_size + (p % per_part) * 512 + lane * 8;
        there[u] = a.vocab - at[u];
        if (there[u] > 0) load_raw8<DT>(a.logits, t * a.ld + at[u], there[u], raw[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      to_float8<DT>(raw[u], x);
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) mask |= (uint32_t)((x[e] >= lo0 && x[e] <= hi0) || (x[e] >= lo1 && x[e] <= hi1)) << e;
      for (int q = 2; q < runs; ++q) {
        const float lo = s.lower[q], hi = s.upper[q];
#pragma unroll
        for (int e = 0; e < 8; ++e) mask |= (uint32_t)(x[e] >= lo && x[e] <= hi) << e;
      }
      mask &= there[u] >= 8 ? 255u : there[u] > 0 ? (1u << there[u]) - 1 : 0u;
      if (!mask) continue;
      uint32_t n = atomicAdd(&s.n, (uint32_t)__popc(mask));
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (mask >> e & 1) {
          if (n < kList) s.list[n] = (unsigned long long)~order_key(x[e]) << 32 | (uint32_t)(at[u] + e);
          ++n;
        }
    }
  }
  __syncthreads();
  const int taken = (int)s.n;
  for (int x = tid; x < min(taken, kList); x += kPickThreads) {
    const float v = key_value(~(uint32_t)(s.list[x] >> 32));
    const int b = infinite && v != largest ? kBuckets : bucket_of(v);
    if (b >= kBuckets || !flagged(s, b)) s.list[x] = ~0ull, atomicAdd(&s.dropped, 1u);   // (goes to the end)
  }
  __syncthreads();
  const int n = taken - (int)s.dropped;
  if (taken > kList || n == 0) {
    __syncthreads();
    sample_digits<DT>(a, t, r, *(PickShared*)shared);
    return;
  }
  if (taken <= 64) {
    if (wave == 0) pick<64, 1>(a, t, r, s, taken, n, bucket_of);
  } else if (taken <= kPickThreads) {
    pick<kPickThreads, 1>(a, t, r, s, taken, n, bucket_of);
  } else {
    pick<kPickThreads, kList / kPickThreads>(a, t, r, s, taken, n, bucket_of);
  }
}

constexpr int kPartLeast = kPartThreads * 8, kPartMost = kPartThreads * 16;
static size_t sample_ws_bytes(int T, int vocab) {
  const size_t parts = ((size_t)vocab + kPartLeast - 1) / kPartLeast;
  return (size_t)T * parts * (sizeof(PartHead) + kBuckets * 8);
}

template <int DT>
static int launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  // parts of 8192 tokens where that leaves compute units idle, else of 16384
  const int part = (int64_t)a.T * ((a.vocab + kPartMost - 1) / kPartMost) < 512 ? kPartLeast : kPartMost;
  const int parts = (a.vocab + part - 1) / part;
  PartHead* heads = (PartHead*)ws;
  unsigned long long* hists = (unsigned long long*)(heads + (size_t)a.T * parts);
  static KernelSetup setup;
  const int e = kernel_setup(setup, [] {
    return hipFuncSetAttribute((const void*)sample_rows_kernel<DT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowShared));
  });
  if (e) return e;
  // (the grid's second dimension ends at 65535 rows)
  for (int t0 = 0; t0 < a.T; t0 += 65535) {
    SampleArgs b = a;
    b.T = a.T - t0 < 65535 ? a.T - t0 : 65535;
    b.logits = (const char*)a.logits + (size_t)t0 * a.ld * dtype_size(DT);
    const auto from = [&](auto* p) { return p ? p + t0 : p; };
    b.temperature = from(a.temperature), b.top_p = from(a.top_p), b.min_p = from(a.min_p), b.u = from(a.u), b.top_k = from(a.top_k);
    b.tokens = from(a.tokens), b.probs = from(a.probs);
    if (part == kPartLeast) sample_parts_kernel<DT, 8><<<dim3(parts, b.T), kPartThreads, 0, s>>>(b, heads, hists);
    else sample_parts_kernel<DT, 16><<<dim3(parts, b.T), kPartThreads, 0, s>>>(b, heads, hists);
    sample_rows_kernel<DT><<<b.T, kPickThreads, sizeof(RowShared), s>>>(b, heads, hists, parts, part);
  }
  return (int)hipGetLastError();
}



}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_sample_workspace_bytes(int T, int vocab, size_t* bytes_out) {
  if (T < 1 || vocab < 1 || !bytes_out) return MDBF_EINVAL;
  if (vocab > kSampleMaxVocab) return MDBF_EUNSUPPORTED;
  *bytes_out = sample_ws_bytes(T, vocab);
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
  const hipStream_t q = (hipStream_t)stream;
  return hip_fail(dtype == MDBF_F16 ? launch_sample<MDBF_F16>(a, workspace_dev, q)
                  : dtype == MDBF_BF16 ? launch_sample<MDBF_BF16>(a, workspace_dev, q) : launch_sample<MDBF_F32>(a, workspace_dev, q));
}

}  // extern "C"
