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
__device__ __forceinline__ RowSetting row_setting(const SampleArgs& a, int64_t t) {
  RowSetting r;
  const float temperature = a.temperature ? a.temperature[t] : 1.0f;
  r.greedy = !(temperature > 0.0f);
  r.per_degree = 1.0 / (double)temperature;
  r.grid = 16 * 1.44269504088896340736 / (double)temperature;   // sixteenths of a factor of two per unit of the logits
  r.top = 0, r.largest = 0;                     // (the row's largest, when it is known)
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

// Masses as whole numbers, whose sums do not go by the order of the additions: units of 2^-43, and what is left of a weight in units of 2^-65.
// (2^20 weights of 1 are 2^63 of the ones, their rests at most 2^42 of the others: there a count fits above them.)  A weight is off by 2^-66, so many
// equal ones, whose errors are the same and add up, by 2^-46 together; one word of 2^-43 alone would be off by 6e-8.
constexpr int kRestBits = 22, kTallyBit = 43;
struct Mass {
  unsigned long long units, rests;
  __device__ __forceinline__ Mass() : units(0), rests(0) {}
  __device__ __forceinline__ Mass(unsigned long long u, unsigned long long r) : units(u + (r >> kRestBits)), rests(r & ((1ull << kRestBits) - 1)) {}
  __device__ __forceinline__ explicit Mass(double w) {
    const double x = w * 0x1p43;
    units = (unsigned long long)x;
    rests = (unsigned long long)((x - (double)units) * (double)(1 << kRestBits) + 0.5);
  }
  __device__ __forceinline__ Mass operator+(const Mass& m) const { return Mass(units + m.units, rests + m.rests); }
  __device__ __forceinline__ double value() const { return ((double)units + (double)rests * (1.0 / (1 << kRestBits))) * 0x1p-43; }
};

struct PickShared {
  unsigned long long units[256], rests[256];     // (the rests' words: how many tokens, above kTallyBit)
  unsigned long long sum[2][kPickThreads / 64];
  uint32_t found[kPickThreads / 64];
  uint32_t digit, count_before;
  Mass before;
};
__device__ __forceinline__ uint32_t tokens_of(unsigned long long word) { return (uint32_t)(word >> kTallyBit); }
__device__ __forceinline__ Mass mass_of(unsigned long long units, unsigned long long word) { return Mass(units, word & ((1ull << kTallyBit) - 1)); }

// The place in the order of keys at which the number of tokens reaches `count`, or else their mass reaches `mass` (or goes beyond it).  Four
// digits of eight bits, the largest first.  `each` calls what it is given with a thread's keys.
struct Place {
  uint32_t key, ties, before;                   // of equal keys there are `ties`; tokens and mass in front of them
  Mass mass_before;
};
template <class Each, class Weight>
__device__ Place descend(const Each& each, const Weight& weight_of, PickShared& s, uint32_t count, double mass, bool beyond) {
  const int tid = threadIdx.x, lane = tid & 63;
  Place at = {0, 0, 0, {}};
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) s.units[tid] = 0, s.rests[tid] = 0;
    __syncthreads();
    each([&](uint32_t k) {
      if (shift < 24 && ((k ^ at.key) >> (shift + 8))) return;
      const Mass m(weight_of(k));
      atomicAdd(&s.rests[(k >> shift) & 255], 1ull << kTallyBit | m.rests);
      if (m.units) atomicAdd(&s.units[(k >> shift) & 255], m.units);
    });
    __syncthreads();
    if (tid < 64) {
      unsigned long long units = 0, word = 0;
      for (int q = 0; q < 4; ++q) units += s.units[255 - lane * 4 - q], word += s.rests[255 - lane * 4 - q];
      const uint32_t c = tokens_of(word);
      unsigned long long units_to = units, word_to = word;
      for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long uu = __shfl_up(units_to, o), uw = __shfl_up(word_to, o);
        if (lane >= o) units_to += uu, word_to += uw;
      }
      const auto reached = [&](uint32_t c, const Mass& m) { return count ? c >= count : beyond ? m.value() > mass : m.value() >= mass; };
      const unsigned long long hit = __ballot(c && reached(at.before + tokens_of(word_to), at.mass_before + mass_of(units_to, word_to))), any = __ballot(c != 0);
      const int who = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(any);
      if (lane == who) {
        uint32_t cb = at.before + tokens_of(word_to) - c;
        Mass mb = at.mass_before + mass_of(units_to - units, word_to - word);
        for (int q = 0; q < 4; ++q) {
          const uint32_t b = 255 - lane * 4 - q, cc = tokens_of(s.rests[b]);
          if (!cc) continue;
          s.digit = b, s.count_before = cb, s.before = mb;
          cb += cc, mb = mb + mass_of(s.units[b], s.rests[b]);
          if (reached(cb, mb)) break;
        }
      }
    }
    __syncthreads();
    at.key |= s.digit << shift;
    at.before = s.count_before, at.mass_before = s.before;
    at.ties = tokens_of(s.rests[s.digit]);
  }
  return at;
}

// A row that nothing else serves: read again for every digit.  `weighs`: whether a logit lies in the buckets, as below: the same tokens weigh nothing on both ways.  128256
// logits, us: 450 flat ones, 1050 with top_k and top_p too, 1030 equal ones (whose LDS additions all meet).
template <int DT, class Weighs>
__device__ void sample_digits(const SampleArgs& a, int64_t t, const RowSetting& r, PickShared& s, const Weighs& weighs) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto weight_of = [&](uint32_t key) { return weighs(key_value(key)) ? weight(r, key) : 0.0; };
  const auto each = [&](const auto& take) {
    for (int i = tid; i < a.vocab; i += kPickThreads) take(key_at<DT>(a, t, i));
  };
  // what is kept is a first part of the order, and so is what each bound leaves: the least of their masses
  Mass total, likely;
  each([&](uint32_t k) {
    const double x = weight_of(k);
    const Mass w(x);
    total = total + w;
    if (x >= r.min_p) likely = likely + w;
  });
  for (int q = 0; q < 2; ++q) {
    Mass v = q ? likely : total;
    for (int o = 1; o < 64; o <<= 1) v = v + Mass(__shfl_xor(v.units, o), __shfl_xor(v.rests, o));
    __syncthreads();
    if (lane == 0) s.sum[0][wave] = v.units, s.sum[1][wave] = v.rests;
    __syncthreads();
    v = Mass();
    for (int w = 0; w < kPickThreads / 64; ++w) v = v + Mass(s.sum[0][w], s.sum[1][w]);
    (q ? likely : total) = v;
  }
  double kept = total.value();
  if (r.top_k) {
    const Place p = descend(each, weight_of, s, r.top_k, 0.0, false);
    kept = p.mass_before.value() + (double)(r.top_k - p.before) * weight_of(p.key);
  }
  double least = kept;
  if (r.top_p < 1.0) {
    const double mass = r.top_p * kept;
    const Place p = descend(each, weight_of, s, 0, mass, false);
    const double w = weight_of(p.key), b = p.mass_before.value();
    double j = w > 0 ? ceil((mass - b) / w) : 1.0;
    j = fmin(fmax(j, 1.0), (double)p.ties);
    least = fmin(least, b + j * w);
  }
  if (r.min_p > 0.0) least = fmin(least, fmax(likely.value(), 1.0));
  kept = least;
  const double mass = r.u * kept;
  const Place p = descend(each, weight_of, s, 0, mass, true);
  const double w = weight_of(p.key), b = p.mass_before.value();
  const uint32_t key = p.key;
  const double j = w > 0 ? floor((mass - b) / w) : 0.0;
  const uint32_t tie = (uint32_t)fmin(fmax(j, 0.0), (double)(p.ties - 1));
  const double prob = w / kept;
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
// at by themselves, and the bounds applied exactly; the first launch leaves the tokens in the order of their buckets, so that these are a few runs of each
// part's.  Tokens that equal the part's largest are counted apart, so that those that equal the row's largest, of weight 1, make up a bucket of an exact mass:
// where many are alike, bounds fall on borders between them.
// The first launch's vector work (some 40 instructions a token, 20 of them fp64) and its LDS additions take longer than the logits: 200 rows of 128256 bf16
// (51 MB, 10 us at the rate of a read) 37.9 us, of which writing buckets and order is as much traffic again.  The second one is a chain of some thirty
// meetings and dependent loads: 11 us for one row of 128256 whose list is short, 21 for 64 rows of 32000 whose longest list is 740, 29 for 200 rows of
// 128256 with lists of up to 4000.  Before: one workgroup a row that reads it for every digit of every bound, 430, 200 and 680 us.
constexpr int kBuckets = 768;                    // of a row: the largest, then 767 sixteenths, down to 2^-47 of it; less weighs nothing
constexpr int kPerOctave = 16;
constexpr int kFracBits = 39;                    // of 2^(frac / 16) - 1 + kBias < 0.0443: a part's stay below 2^49, where the count begins
constexpr int kCountBit = 49;
constexpr int kList = 8192;                      // tokens of a row that the second launch looks at; rows that have more go by digits
constexpr int kPartThreads = 512, kPart = 8192, kEach = kPart / kPartThreads;   // tokens of a part, of a thread
constexpr double kSlack = 1e-7;                  // far more than sums of buckets and of tokens differ by

struct PartHead {
  unsigned long long top;                        // key of the part's largest, and, where that one is asked for, ~its index: of equal keys the lowest is largest
  unsigned long long equal;                      // tokens that equal it
};
// What the first launch leaves, part by part.
struct Parts {
  PartHead* heads;
  unsigned long long* hists;                     // kBuckets each
  uint16_t* starts;                              // kBuckets: where each bucket's tokens begin in what is left, or its end
  uint16_t* left;                                // kPart: tokens in the order of their buckets, their places in the part
};

// t, rounded: its floor, the bucket, goes with the order of the logits, in every part alike.
__device__ __forceinline__ double degrees(const RowSetting& r, float x) { return (double)x * r.grid; }
// t - floor without t's rounding, which at ten million temperatures from zero would be 1e-9 of a weight: a little below 0 or above 1 where t was rounded over
// a whole number.  (Distinct logits of 24 bits share buckets up to t = 2^34, so by at most 2^-20 of t.)
__device__ __forceinline__ double fraction(const RowSetting& r, float x, double floor) { return fma((double)x, r.grid, -floor); }
constexpr double kBias = 0x1p-16;                // a token adds this more, so that its whole number is none below 0

// What a token adds to its bucket: 1 in the count, and 2^(x / 16) - 1 + kBias in units of 2^-39 for x in [0, 1], the fraction of its t.  The polynomial
// of degree four whose largest error is least, 2.9e-12, of those that are 0 at 0 (found by linear programming): where all tokens weigh the same, an infinite
// temperature, their masses are exact.  The sum with 2^52 and the count's bit has the whole number in its last bits.
struct BucketWord {
  double c0, c1, c2, c3, c4;
  __device__ __forceinline__ BucketWord() {
    constexpr double unit = (double)(1ull << kFracBits);
    c4 = 1.4989737097980216e-07 * unit, c3 = 1.3548161761869753e-05 * unit, c2 = 9.383856709375404e-04 * unit, c1 = 0.043321698694471764 * unit;
    c0 = kBias * unit + 0x1p52 + (double)(1ull << kCountBit);
    // (as values that the compiler does not know they stay in scalar registers; it would copy constants into a sum's register every time)
    asm("" : "+s"(c0), "+s"(c1), "+s"(c2), "+s"(c3), "+s"(c4));
  }
  __device__ __forceinline__ unsigned long long operator()(double x) const {
    const double g = fma(x, fma(x, fma(x, fma(x, c4, c3), c2), c1), c0);
    return __builtin_bit_cast(unsigned long long, g) & 0xfffffffffffffull;
  }
};

// sums of the threads in front of this one, and of all, over a workgroup of 1024
__device__ __forceinline__ uint32_t scan_counts(uint32_t v, uint32_t& total, uint32_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t to = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(to, o);
    if (lane >= o) to += u;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = to;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w == wave) before = total;
    total += waves[w];
  }
  return before + to - v;
}

template <int DT>
__global__ __launch_bounds__(kPartThreads, 6) void sample_parts_kernel(SampleArgs a, Parts parts) {
  __shared__ __align__(16) uint16_t order[kPart];
  __shared__ unsigned long long hist[kBuckets];
  __shared__ uint32_t slot[kBuckets + 2];        // the next place in the order of those that equal the largest, then of each bucket's
  __shared__ float tops[kPartThreads / 64];
  __shared__ uint32_t waves[kPartThreads / 64], equal, left, first;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.y, part = t * gridDim.x + blockIdx.x;
  const int i0 = blockIdx.x * kPart;

  Raw8<DT> raw[kEach / 8];
#pragma unroll
  for (int p = 0; p < kEach / 8; ++p) {
    const int i = i0 + (p * kPartThreads + tid) * 8;
    if (i < a.vocab) load_raw8<DT>(a.logits, t * a.ld + i, a.vocab - i, raw[p]);
  }
  const RowSetting r = row_setting(a, t);
  for (int o = tid; o < kBuckets; o += kPartThreads) hist[o] = 0;
  if (tid == 0) equal = left = slot[0] = 0, first = 0xffffffffu;
  float v[kEach], best = -__builtin_inff();
#pragma unroll
  for (int p = 0; p < kEach / 8; ++p) {
    const int there = a.vocab - (i0 + (p * kPartThreads + tid) * 8);
    float x[8];
    to_float8<DT>(raw[p], x);
    if (there < 8) {                             // (NaN, which nothing below counts)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= there) x[e] = __builtin_nanf("");
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[p * 8 + e] = x[e], best = fmaxf(best, x[e]);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) best = fmaxf(best, __shfl_xor(best, o));
  if (lane == 0) tops[wave] = best;
  __syncthreads();
  float largest = tops[0];
#pragma unroll
  for (int w = 1; w < kPartThreads / 64; ++w) largest = fmaxf(largest, tops[w]);
  const auto place_of = [&](int e) { return (uint32_t)(((e / 8) * kPartThreads + tid) * 8 + e % 8); };
  const uint32_t key = order_key(largest);
  if (key <= kKeyNone || r.greedy) {             // then the first that equals it is all that is asked for
    uint32_t at = 0xffffffffu;
#pragma unroll
    for (int e = kEach - 1; e >= 0; --e)
      if (v[e] == largest) at = i0 + place_of(e);
    atomicMin(&first, at);
    __syncthreads();
    if (tid == 0) parts.heads[part].top = (unsigned long long)key << 32 | ~first;
    return;
  }
  const bool infinite = largest == __builtin_inff();    // then nothing else weighs
  const double base = floor(degrees(r, largest));
  const BucketWord bucket_word;
  uint32_t alike = 0;
  int down[kEach];                               // a token's slot: 0 of the largest, 1 + its bucket; beyond the last: none
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const bool same = v[e] == largest;
    alike += (uint32_t)__popcll(__ballot(same));
    down[e] = same ? 0 : kBuckets + 1;
    const double d = degrees(r, v[e]), f = floor(d), b = base - f;
    if (b < kBuckets && !same && !infinite) {           // (not of -inf, whose b is inf, and not of NaN)
      const int o = (int)b;
      down[e] = o + 1;
      atomicAdd(&hist[o], bucket_word(fraction(r, v[e], f)));
    }
  }
  if (lane == 0 && alike) atomicAdd(&equal, alike);
  __syncthreads();
  // Where each bucket's tokens begin, two buckets a thread, and how far they are left in order: no further than the row's own bounds can reach.
  const uint32_t n_equal = equal;
  const bool has = tid < kBuckets / 2;
  const unsigned long long h0 = has ? hist[2 * tid] : 0, h1 = has ? hist[2 * tid + 1] : 0;
  const uint32_t c0 = (uint32_t)(h0 >> kCountBit), c1 = (uint32_t)(h1 >> kCountBit);
  uint32_t start = c0 + c1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(start, o);
    if (lane >= o) start += u;
  }
  if (lane == 63) waves[wave] = start;
  __syncthreads();
  start += n_equal - (c0 + c1);
#pragma unroll
  for (int w = 0; w < kPartThreads / 64; ++w)
    if (w < wave) start += waves[w];
  // (top_p of what top_k leaves goes by the mass of tokens below min_p too)
  const double deepest = r.min_p == 0.0 || (r.top_k && r.top_p < 1.0) ? kBuckets : 4.0 - kPerOctave * log2(r.min_p);
  const bool reach0 = has && 2 * tid < deepest && (!r.top_k || start < r.top_k), reach1 = reach0 && 2 * tid + 1 < deepest && (!r.top_k || start + c0 < r.top_k);
  const unsigned long long reached = __ballot(reach0);          // (holds for the first buckets alone)
  if (reached && lane == 63 - __builtin_clzll(reached)) atomicMax(&left, start + c0 + (reach1 ? c1 : 0));
  if (has) {
    slot[2 * tid + 1] = reach0 ? start : kPart, slot[2 * tid + 2] = reach1 ? start + c0 : kPart;
    typedef unsigned long long Pair __attribute__((ext_vector_type(2)));
    *((MDBF_GLOBAL Pair*)(parts.hists + part * kBuckets) + tid) = Pair{h0, h1};
  }
  __syncthreads();
  const uint32_t n_left = max(left, n_equal);
  if (has) ((MDBF_GLOBAL uint32_t*)(parts.starts + part * kBuckets))[tid] = min(start, n_left) | min(start + c0, n_left) << 16;
  if (tid == 0) parts.heads[part] = {(unsigned long long)key << 32, n_equal};
  uint32_t place[kEach];                         // (asked for together, so that their trips overlap: one after another 39 us instead of 37.5)
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    place[e] = kPart;
    if (down[e] <= kBuckets) place[e] = atomicAdd(&slot[down[e]], 1u);
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    if (place[e] < kPart) order[place[e]] = (uint16_t)place_of(e);    // (slots that none reaches begin at kPart)
  __syncthreads();
  MDBF_GLOBAL U32x4* out = (MDBF_GLOBAL U32x4*)(parts.left + part * kPart);
  for (uint32_t x = tid; x * 8 < n_left; x += kPartThreads) out[x] = ((const U32x4*)order)[x];
}

// What the second launch has in LDS.
constexpr int kMaxParts = kSampleMaxVocab / kPart;
constexpr int kBins = kPickThreads;
constexpr int kRuns = 4;                         // runs of neighbouring buckets that are looked at
struct RowShared {
  unsigned long long list[kList];                // ~key, index: the order of the tokens
  unsigned long long few[64];
  double before[kBuckets];                       // mass and tokens in front of a bucket
  uint32_t count_before[kBuckets];
  uint16_t bin[kList];
  unsigned long long bin_mass[kBins];
  double bin_from[kBins];
  uint32_t bin_count[kBins], bin_first[kBins];
  double sums[kPickThreads / 64];
  uint32_t counts[kPickThreads / 64];
  unsigned long long tops[kPickThreads / 64];
  unsigned long long part_extra[kMaxParts];      // of a part: its largest's bucket in the row (kBuckets: nothing there weighs), how many equal it, and
  int32_t part_top[kMaxParts];                   // their fractions
  uint32_t part_equal[kMaxParts];
  double klo, khi, plo, phi, mlo, mhi, total;
  unsigned long long likely;
  double value;
  int k, p0, p1, m0, m1, u0, u1;
  int chosen[3];
  uint32_t n, n_few, key, ties;
  PickShared digits;
};

struct Runs {
  int from[kRuns], to[kRuns];                    // disjoint, rising; empty ones at the end have from > to
  int buckets;
};
// The union of up to four ranges.
__device__ __forceinline__ Runs runs_of(const int (&lo)[kRuns], const int (&hi)[kRuns]) {
  Runs r;
#pragma unroll
  for (int q = 0; q < kRuns; ++q) r.from[q] = hi[q] < lo[q] ? 1 << 20 : lo[q], r.to[q] = hi[q];
  const auto order = [&](int x, int y) {
    if (r.from[y] < r.from[x]) {
      const int f = r.from[x], t = r.to[x];
      r.from[x] = r.from[y], r.to[x] = r.to[y], r.from[y] = f, r.to[y] = t;
    }
  };
  order(0, 1), order(2, 3), order(0, 2), order(1, 3), order(1, 2);
  r.buckets = 0;
#pragma unroll
  for (int q = 0; q < kRuns; ++q) {
#pragma unroll
    for (int e = q + 1; e < kRuns; ++e)           // what touches it belongs to it
      if (r.from[e] <= r.to[q] + 1 && r.from[q] < 1 << 20) r.to[q] = max(r.to[q], r.to[e]), r.from[e] = 1 << 20, r.to[e] = -1;
    if (r.from[q] < 1 << 20) r.buckets += r.to[q] - r.from[q] + 1;
  }
  return r;
}

// Which buckets have to be looked at: those of the bounds and of the drawn number, the latter ones' ends by the least and the most that the bounds
// may leave.  k, p0 .., m0 .., u0 .. are set to no bound before.  `least`, `other`: min_p, resp. the other bounds, are sure to be undercut and
// need none of their tokens.
struct Choice {
  bool least, other;
  Runs runs;
};
__device__ __forceinline__ Choice choose_buckets(const RowSetting& r, RowShared& s, double before, double upto, uint32_t count_before, uint32_t count_to,
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
  const double plo = s.plo, phi = s.phi, mlo = s.mlo, mhi = s.mhi;
  const double ulo = r.u * fmin(klo, fmin(plo, mlo)) * (1 - kSlack), uhi = r.u * fmin(khi, fmin(phi, mhi)) * (1 + kSlack);
  if (in && before <= ulo && upto > ulo) s.u0 = o;
  if (in && before <= uhi && upto > uhi) s.u1 = o;
  __syncthreads();
  Choice c;
  c.least = mlo >= fmin(khi, phi), c.other = mhi <= fmin(klo, plo);
  const int lo[kRuns] = {s.k, s.p0, s.m0, s.u0}, hi[kRuns] = {c.other || s.k < 0 ? -2 : s.k, c.other ? -2 : s.p1, c.least ? -2 : s.m1, s.u1};
  c.runs = runs_of(lo, hi);
  return c;
}

enum Bound { kByCount, kByMass, kByDraw };
// Where in a bin of the list a bound lies: with kByCount and kByMass the mass of what it leaves, with kByDraw the token, which the
// threads that find it write.  `target`: so many tokens, so much mass.  In bins of up to 64 tokens a wave puts them in order; in others, where most
// often many are alike, the first four values are tried one after the other, and what comes behind goes by digits: 8000 different logits in one bin
// (an infinite temperature) take 200 us a row, from one value to the next they took 91 ms.
template <int DT>
__device__ double resolve(const SampleArgs& a, int64_t t, const RowSetting& r, RowShared& s, int n, int bin, double target, int what, double kept) {
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t here = s.bin_count[bin];
  double before = s.bin_from[bin];
  uint32_t first = s.bin_first[bin];
  __syncthreads();                               // (the last use of what follows is over)
  if (tid == 0) s.n_few = 0, s.key = 0, s.ties = 0;
  __syncthreads();
  if (here <= 64) {
    for (int x = tid; x < n; x += kPickThreads)
      if (s.bin[x] == bin) s.few[atomicAdd(&s.n_few, 1u)] = s.list[x];
    __syncthreads();
    if (tid < 64) {
      const int m = (int)here;
      unsigned long long v = tid < m ? s.few[tid] : ~0ull;
      int place = 0;
      for (int j = 0; j < m; ++j) place += __shfl(v, j) < v;
      if (tid < m) s.few[place] = v;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
      __builtin_amdgcn_wave_barrier();
      v = tid < m ? s.few[tid] : ~0ull;
      const double w = tid < m ? weight(r, ~(uint32_t)(v >> 32)) : 0.0;
      double to = w;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(to, o);
        if (lane >= o) to += u;
      }
      const double at = before + (to - w);
      to += before;
      const bool in = tid < m;
      if (what == kByDraw) {
        const unsigned long long b = __ballot(in && to > target);
        const int x = b ? __builtin_ctzll(b) : m - 1;    // (none goes beyond it only by rounding)
        if (tid == x) {
          a.tokens[t] = (int)(uint32_t)v;
          if (a.probs) a.probs[t] = (float)(w / kept);
        }
      } else {
        const bool holds = what == kByCount ? (double)(first + lane) < target : at < target || first + lane == 0;
        const unsigned long long b = __ballot(in && holds);
        const double m1 = b ? __shfl(to, 63 - __builtin_clzll(b)) : before;
        if (tid == 0) s.value = m1;
      }
    }
    __syncthreads();
    return s.value;
  }
  uint32_t last = 0xffffffffu, key = 0, ties = 0, seen = 0;
  double w = 0;
  for (int values = 0;; ++values) {
    if (values == 4) {
      const auto each = [&](const auto& take) {
        for (int x = tid; x < n; x += kPickThreads) {
          const uint32_t k = ~(uint32_t)(s.list[x] >> 32);
          if (s.bin[x] == bin && k < last) take(k);
        }
      };
      const uint32_t count = what == kByCount ? (uint32_t)target - first : 0;
      const Place p = descend(each, [&](uint32_t k) { return weight(r, k); }, s.digits, count, target - before, what == kByDraw);
      key = p.key, ties = p.ties, w = weight(r, key);
      before += p.mass_before.value(), first += p.before;
      break;
    }
    for (int x = tid; x < n; x += kPickThreads) {
      const uint32_t k = ~(uint32_t)(s.list[x] >> 32);
      if (s.bin[x] == bin && k < last) atomicMax(&s.key, k);
    }
    __syncthreads();
    key = s.key;
    for (int x = tid; x < n; x += kPickThreads)
      if (s.bin[x] == bin && ~(uint32_t)(s.list[x] >> 32) == key) atomicAdd(&s.ties, 1u);
    __syncthreads();
    ties = s.ties;
    w = weight(r, key);
    seen += ties;
    const double to = before + (double)ties * w;
    if (seen >= here || (what == kByCount ? (double)(first + ties) >= target : what == kByMass ? to >= target : to > target)) break;
    before = to, first += ties, last = key;
    __syncthreads();
    if (tid == 0) s.key = 0, s.ties = 0;
    __syncthreads();
  }
  if (what == kByCount) return before + fmin(target - (double)first, (double)ties) * w;
  if (what == kByMass) {
    const double j = w > 0 ? ceil((target - before) / w) : 0.0;
    return before + fmin(fmax(j, first == 0 ? 1.0 : 0.0), (double)ties) * w;
  }
  // the one with the right number among equal ones, by index: its thousand first, then itself
  uint32_t tie = (uint32_t)fmin(fmax(w > 0 ? floor((target - before) / w) : 0.0, 0.0), (double)(ties - 1)), group = 0, total;
  for (int level = 0; level < 2; ++level) {
    __syncthreads();
    s.bin_count[tid] = 0;
    __syncthreads();
    for (int x = tid; x < n; x += kPickThreads) {
      const unsigned long long v = s.list[x];
      const uint32_t i = (uint32_t)v;
      if (~(uint32_t)(v >> 32) == key && s.bin[x] == bin && (level == 0 || i >> 10 == group)) atomicAdd(&s.bin_count[level ? i & 1023 : i >> 10], 1u);
    }
    __syncthreads();
    const uint32_t c = s.bin_count[tid], from = scan_counts(c, total, s.counts);
    if (c && from <= tie && tie < from + c) s.chosen[0] = tid, s.n_few = from;
    __syncthreads();
    if (level == 0) group = (uint32_t)s.chosen[0], tie -= s.n_few;
  }
  if (tid == 0) {
    a.tokens[t] = (int)(group << 10 | (uint32_t)s.chosen[0]);
    if (a.probs) a.probs[t] = (float)(w / kept);
  }
  return 0.0;
}

// The bounds and the draw on the list.  Its tokens are sorted into bins, as many to each of the buckets as there are threads for, whose prefix
// sums tell the one in which a bound lies.
template <int DT, class Bucket>
__device__ __forceinline__ void pick(const SampleArgs& a, int64_t t, const RowSetting& r, RowShared& s, int n, const Choice& c, const Bucket& bucket_of) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int room = c.runs.buckets > 1 ? 32 - __builtin_clz(c.runs.buckets - 1) : 0, sub_bits = 10 - room;
  if (tid < 3) s.chosen[tid] = -1;
  if (tid == 0) s.likely = 0;
  s.bin_count[tid] = 0, s.bin_mass[tid] = 0;
  __syncthreads();
  unsigned long long likely = 0;
  for (int x = tid; x < n; x += kPickThreads) {
    const uint32_t k = ~(uint32_t)(s.list[x] >> 32);
    const float v = key_value(k);
    const int b = bucket_of(v);
    int at = b;
#pragma unroll
    for (int q = kRuns - 1; q > 0; --q)          // buckets between the runs have no bins
      if (b >= c.runs.from[q]) {
        at = b - c.runs.from[q];
#pragma unroll
        for (int e = 0; e < q; ++e)
          if (c.runs.from[e] <= c.runs.to[e]) at += c.runs.to[e] - c.runs.from[e] + 1;
        break;
      } else if (q == 1) {
        at = b - c.runs.from[0];
      }
    const double d = degrees(r, v);
    const int sub = b == 0 ? 0 : min((int)((1.0 - (d - floor(d))) * (1 << sub_bits)), (1 << sub_bits) - 1), bin = at << sub_bits | sub;
    s.bin[x] = (uint16_t)bin;
    const double w = weight(r, k);
    const unsigned long long m = (unsigned long long)(w * 0x1p50 + 0.5);
    atomicAdd(&s.bin_count[bin], 1u);
    atomicAdd(&s.bin_mass[bin], m);
    if (b >= s.m0 && b <= s.m1 && w >= r.min_p) likely += m;
  }
  if (s.m1 >= 0 && !c.least) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) likely += __shfl_xor(likely, o);
    if (lane == 0 && likely) atomicAdd(&s.likely, likely);
  }
  __syncthreads();
  const uint32_t count = s.bin_count[tid];
  const double mass = (double)s.bin_mass[tid] * 0x1p-50;
  uint32_t first = count;
  double to = mass;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t uc = __shfl_up(first, o);
    const double um = __shfl_up(to, o);
    if (lane >= o) first += uc, to += um;
  }
  if (lane == 63) s.sums[wave] = to, s.counts[wave] = first;
  __syncthreads();
  double from = to - mass;
  first -= count;
#pragma unroll
  for (int w = 0; w < kPickThreads / 64; ++w)
    if (w < wave) from += s.sums[w], first += s.counts[w];
  s.bin_from[tid] = from, s.bin_first[tid] = first;
  __syncthreads();
  // the bin's bucket, and what is in front of the bin: of the bucket in the row, and of the bin in the bucket
  int at = tid >> sub_bits, bucket = -1;
#pragma unroll
  for (int q = 0; q < kRuns; ++q) {
    const int len = c.runs.to[q] - c.runs.from[q] + 1;
    if (c.runs.from[q] > c.runs.to[q] || bucket >= 0) continue;
    if (at < len) bucket = c.runs.from[q] + at;
    at -= len;
  }
  const int head = tid >> sub_bits << sub_bits;
  const double in_bucket = from - s.bin_from[head];
  const uint32_t first_in = first - s.bin_first[head];
  __syncthreads();
  const double before = bucket < 0 ? 0.0 : s.before[bucket] + fmax(in_bucket, 0.0);
  const uint32_t count_before = bucket < 0 ? 0 : s.count_before[bucket] + first_in;
  s.bin_from[tid] = before, s.bin_first[tid] = count_before;

  // what is kept is a first part of the order, and so is what each bound leaves: the least of their masses
  const auto choose = [&](int which, bool holds) {
    const unsigned long long b = __ballot(count && holds);
    if (b && lane == 63 - __builtin_clzll(b)) atomicMax(&s.chosen[which], tid);
    __syncthreads();
    return s.chosen[which];
  };
  double kept = s.total;
  if (s.k >= 0 && !c.other) {
    const int bin = choose(0, bucket == s.k && count_before < r.top_k);
    kept = bin < 0 ? s.klo : resolve<DT>(a, t, r, s, n, bin, (double)r.top_k, kByCount, 1.0);
  }
  if (r.top_p < 1.0 && !c.other) {
    const double target = r.top_p * kept;
    const int bin = choose(1, bucket >= s.p0 && bucket <= s.p1 && (before < target || count_before == 0));
    kept = bin < 0 ? s.plo : resolve<DT>(a, t, r, s, n, bin, target, kByMass, 1.0);
  }
  if (s.m1 >= 0 && !c.least) kept = fmin(kept, r.min_p > 1.0 ? 1.0 : s.mlo + (double)s.likely * 0x1p-50);
  const double drawn = r.u * kept;
  const int bin = choose(2, bucket >= s.u0 && bucket <= s.u1 && (before <= drawn || count_before == s.count_before[s.u0]));
  if (bin >= 0) resolve<DT>(a, t, r, s, n, bin, drawn, kByDraw, kept);
}

// The same on a list of up to 64 tokens, by one wave, which puts all of them in order.
template <class Bucket>
__device__ __forceinline__ void pick_few(const SampleArgs& a, int64_t t, const RowSetting& r, RowShared& s, int n, const Choice& c, const Bucket& bucket_of) {
  const int lane = threadIdx.x;
  const auto meet = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
  };
  unsigned long long v = lane < n ? s.list[lane] : ~0ull;
  int place = 0;
  for (int j = 0; j < n; ++j) place += __shfl(v, j) < v;
  if (lane < n) s.few[place] = v;
  meet();
  v = lane < n ? s.few[lane] : ~0ull;
  const uint32_t key = ~(uint32_t)(v >> 32);
  const bool in = lane < n;
  const double w = in ? weight(r, key) : 0.0;
  const int bucket = in ? bucket_of(key_value(key)) : kBuckets;
  double to = w;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = __shfl_up(to, o);
    if (lane >= o) to += u;
  }
  // from a bucket's first token on, behind what is in front of the bucket in the row
  const int neighbour = __shfl_up(bucket, 1);
  const unsigned long long heads = __ballot(lane == 0 || bucket != neighbour);
  const int head = 63 - __builtin_clzll(heads & (~0ull >> (63 - lane)));
  const double at = in ? s.before[bucket] + (to - w - __shfl(to - w, head)) : 0.0;
  const uint32_t rank = in ? s.count_before[bucket] + (uint32_t)(lane - head) : 0;
  to = at + w;
  const auto bound = [&](bool holds, double none) {
    const unsigned long long b = __ballot(in && holds);
    return b ? __shfl(to, 63 - __builtin_clzll(b)) : none;
  };
  double kept = s.total;
  if (s.k >= 0 && !c.other) kept = bound(bucket == s.k && rank < r.top_k, s.klo);
  if (r.top_p < 1.0 && !c.other) {
    const double target = r.top_p * kept;
    kept = bound(bucket >= s.p0 && bucket <= s.p1 && (at < target || rank == 0), s.plo);
  }
  if (s.m1 >= 0 && !c.least) kept = fmin(kept, bound(bucket >= s.m0 && bucket <= s.m1 && (w >= r.min_p || rank == 0), s.mlo));
  const double drawn = r.u * kept;
  const bool mine = in && bucket >= s.u0 && bucket <= s.u1;
  const unsigned long long beyond = __ballot(mine && to > drawn), any = __ballot(mine);
  // (none goes beyond it only by the sums' rounding: the last one then)
  const int x = beyond ? __builtin_ctzll(beyond) : 63 - __builtin_clzll(any);
  if (lane == x) {
    a.tokens[t] = (int)(uint32_t)v;
    if (a.probs) a.probs[t] = (float)(w / kept);
  }
}

template <int DT>
__global__ __launch_bounds__(kPickThreads) void sample_rows_kernel(SampleArgs a, Parts left, int parts) {
  extern __shared__ char shared[];
  RowShared& s = *(RowShared*)shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x, row = t * parts;
  PartHead head = {};
  if (tid < parts) head = left.heads[row + tid];
  RowSetting r = row_setting(a, t);
  unsigned long long top = head.top;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long u = __shfl_xor(top, o);
    if (u > top) top = u;
  }
  if (lane == 0) s.tops[wave] = top;
  if (tid == 0) {
    s.n = 0;
    s.k = -1, s.p0 = s.m0 = s.u0 = 0, s.m1 = -1, s.u1 = kBuckets - 1;
    s.klo = s.khi = s.phi = s.mlo = s.mhi = INFINITY;
    s.p1 = r.top_p < 1.0 ? kBuckets - 1 : -1, s.plo = r.top_p < 1.0 ? 0.0 : INFINITY;
  }
  __syncthreads();
  top = s.tops[0];
  if (parts > 64 && s.tops[1] > top) top = s.tops[1];
  const uint32_t key = (uint32_t)(top >> 32);
  if (key <= kKeyNone || r.greedy) {
    if (tid == 0) {
      a.tokens[t] = key <= kKeyNone ? -1 : (int)~(uint32_t)top;
      if (a.probs) a.probs[t] = key <= kKeyNone ? 0.0f : 1.0f;
    }
    return;
  }
  const float largest = key_value(key);
  r.top = key, r.largest = (double)largest;
  const bool infinite = largest == __builtin_inff();
  const double base = infinite ? 0.0 : floor(degrees(r, largest));
  // (beyond 2^53 it is no fraction, and nothing but the largest weighs)
  const double frac = infinite ? 0.0 : fmin(fmax(fraction(r, largest, base), -kBias), 1 + kBias);
  const auto bucket_of = [&](float x) { return x == largest ? 0 : 1 + (int)fmin(base - floor(degrees(r, x)), (double)kBuckets); };

  if (tid < parts) {
    const float its = key_value((uint32_t)(head.top >> 32));
    const bool none = its == -__builtin_inff() || (infinite && its != largest);
    const int b = none ? kBuckets : min(bucket_of(its), kBuckets);
    s.part_top[tid] = b, s.part_equal[tid] = none ? 0 : (uint32_t)head.equal;
    s.part_extra[tid] = b == 0 || b >= kBuckets ? 0 : head.equal * (BucketWord()(fraction(r, its, floor(degrees(r, its)))) & ((1ull << kCountBit) - 1));
  }
  __syncthreads();

  // a thread's bucket, of all parts (a part's begin with that of its largest, of the row's with bucket 1)
  uint32_t count = 0;
  unsigned long long extra = 0;
  if (tid < kBuckets) {
    constexpr int U = 16;
    const unsigned long long* hists = left.hists + row * kBuckets;
    for (int c0 = 0; c0 < parts; c0 += U) {
      unsigned long long h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u, shift = c < parts && !infinite ? max(s.part_top[c], 1) : kBuckets;
        h[u] = tid >= shift ? hists[(int64_t)c * kBuckets + tid - shift] : 0;
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
                               : ((double)count * (1 - kBias) + (double)extra * (1.0 / (double)(1ull << kFracBits))) * exp2(-(tid - 1 + frac) / kPerOctave);
  uint32_t count_to = count;
  double upto = mass;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t uc = __shfl_up(count_to, o);
    const double um = __shfl_up(upto, o);
    if (lane >= o) count_to += uc, upto += um;
  }
  if (lane == 63) s.sums[wave] = upto, s.counts[wave] = count_to;
  __syncthreads();
  double wave_before = 0, total = 0;
  uint32_t waves_count = 0;
#pragma unroll
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
  if (tid == 0) s.total = total;
  const Choice c = choose_buckets(r, s, before, upto, count_to - count, count_to, frac);

  // Tokens of those buckets: of each part runs of what the first launch has left in order.
  for (int p = wave; p < parts; p += kPickThreads / 64) {
    const int top_bucket = s.part_top[p], shift = max(top_bucket, 1);
    if (top_bucket >= kBuckets) continue;
    const uint16_t* starts = left.starts + (row + p) * kBuckets;
    const uint16_t* tokens = left.left + (row + p) * kPart;
    int begin[kRuns], end[kRuns];
#pragma unroll
    for (int q = 0; q < kRuns; ++q) {
      const int from = c.runs.from[q], to = c.runs.to[q], o0 = max(from - shift, 0), o1 = infinite ? -1 : to - shift;
      const bool with_top = from <= top_bucket && top_bucket <= to;
      begin[q] = end[q] = 0;
      if (o0 <= o1 && from <= to) begin[q] = starts[o0], end[q] = starts[o1 + 1];     // (o1 is the last bucket but one at most)
      if (with_top) {
        begin[q] = 0;
        if (o0 > o1) end[q] = (int)s.part_equal[p];
      }
    }
#pragma unroll
    for (int q = 0; q < kRuns; ++q) {
      const int m = end[q] - begin[q];
      if (m <= 0) continue;
      uint32_t place = 0;
      if (lane == 0) place = atomicAdd(&s.n, (uint32_t)m);
      place = __builtin_amdgcn_readfirstlane(place);
      for (int x = lane; x < m && place + x < kList; x += 64) {
        const int i = p * kPart + tokens[begin[q] + x];
        s.list[place + x] = (unsigned long long)~order_key(load_as_float(a.logits, t * a.ld + i, DT)) << 32 | (uint32_t)i;
      }
    }
  }
  __syncthreads();
  const int n = (int)s.n;
  if (n > kList || n == 0) {
    __syncthreads();
    sample_digits<DT>(a, t, r, *(PickShared*)shared, [&](float x) { return bucket_of(x) < kBuckets; });
    return;
  }
  if (n <= 64) {
    if (wave == 0) pick_few(a, t, r, s, n, c, bucket_of);
  } else {
    pick<DT>(a, t, r, s, n, c, bucket_of);
  }
}

static size_t sample_parts(int vocab) { return ((size_t)vocab + kPart - 1) / kPart; }
static size_t sample_ws_bytes(int T, int vocab) {
  return (size_t)T * sample_parts(vocab) * (sizeof(PartHead) + kBuckets * (8 + 2) + kPart * 2);
}

template <int DT>
static int launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  const int parts = (int)sample_parts(a.vocab);
  const size_t all = (size_t)a.T * parts;
  Parts left;
  left.hists = (unsigned long long*)ws;
  left.heads = (PartHead*)(left.hists + all * kBuckets);
  left.left = (uint16_t*)(left.heads + all);
  left.starts = left.left + all * kPart;
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
    sample_parts_kernel<DT><<<dim3(parts, b.T), kPartThreads, 0, s>>>(b, left);
    sample_rows_kernel<DT><<<b.T, kPickThreads, sizeof(RowShared), s>>>(b, left, parts);
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
