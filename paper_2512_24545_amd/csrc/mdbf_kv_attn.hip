// Attention over the 4-bit cache in pages (format and layout: include/mdbf.h).
//
// For a query row (a new token's head) and the tokens j that it sees:  z_j = scale q . k_j,  out = sum_j e^(z_j - m) v_j /
// sum_j e^(z_j - m), in one pass over the cache with a running maximum m and sum.  The query heads that share a kv head
// are rows of one product, so a page is read once for all of them.
//
// On the matrix cores the scores are K Q^T (tokens x rows) and the results V^T P^T (channels x rows): a lane holds one
// query row throughout, the scores' registers are the second product's operand as they lie, and maxima and sums need two
// exchanges between lanes.  Values become fp16 or bf16 numbers, exactly, with their block's scale by the conversion
// instruction on their way into LDS, where transposing reads take them.  So do keys for few query rows, in the registers that
// feed the product; for prompts their codes are an operand as they are (below).  Scores, maxima, sums and results are fp32; the
// numerators e^(z_j - m) are rounded to the values' type and the sum is of what was not rounded.  The rounding errs by half a unit
// of a numerator's last place; in fp16 also by 2^-32 of the reference's numerator at most, where the type's exponents end: numerators carry a
// factor of 2^7 there (kLift), so that 200000 tokens at that end are 5e-5 of the sum (without it: 0.6 %, and a third of the result
// where the token at the reference has small values).
#include <math.h>

#include <algorithm>
#include <utility>

#include "mdbf_fp6.h"
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
  float* part;
  int32_t table_width, requests, T, pages, kv_heads, group, head_dim, page_shift, causal, window, row_tiles, shares, join_rows;
  uint32_t group_mul, group_shift;      // i / group = i * group_mul >> group_shift for i < 2^31
  float scale;                 // of the scores, times log2(e); its sign is the queries' (flip: 0x80008000)
  uint32_t flip;
  uint8_t wide_q, wide_o, nth;
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
// a scale byte as loaded: beyond the type's largest it stands for NaN (as it is, its block's numbers could be infinite, and a weight of
// zero would carry them to rows that do not see the token)
template <int DT>
__device__ __forceinline__ uint32_t known_scale(uint32_t scale_byte) { return scale_byte > kKvScaleMax[DT] ? kKvNanScale : scale_byte; }
__device__ __forceinline__ float unit_of(uint32_t scale_byte) { return __builtin_bit_cast(float, scale_byte << 23); }

// a wave's LDS operations execute in order: this keeps the compiler from moving them across
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// the new token that query row R of a request and kv head belongs to
__device__ __forceinline__ int token_of(const AttnArgs& a, int R) { return (int)((uint64_t)(uint32_t)R * a.group_mul >> a.group_shift); }

// A request's part of the step: its first row, its new tokens and its length, cut to what the buffers hold.
struct Request {
  int start, fresh, len;
};
__device__ __forceinline__ Request request_of(const AttnArgs& a, int b) {
  Request r;
  r.start = min(max(a.cu[b], 0), a.T);
  r.fresh = (int)min(max((int64_t)a.cu[b + 1] - r.start, (int64_t)0), (int64_t)(a.T - r.start));
  r.len = (int)min((int64_t)max(a.lengths[b], 0), min((int64_t)a.table_width << a.page_shift, (int64_t)0x7ffffc00));
  return r;
}
// the tokens lo <= j < hi that new token i sees
struct Sees {
  int lo, hi;
};
__device__ __forceinline__ Sees sees(const AttnArgs& a, const Request& r, int i) {
  if (!a.causal) return {0, r.len};
  const int end = max(r.len - r.fresh + i + 1, 0);
  return {a.window ? max(end - a.window, 0) : 0, end};
}

// channels c0 .. c0 + N - 1 of a finished row: its sums over the sum of its numerators; zeros if it sees nothing
template <int DT, int N>
__device__ __forceinline__ void store_row(const AttnArgs& a, const Request& rq, int head, int R, int c0, const float (&o)[N], float sum) {
  const int i = token_of(a, R), g = R - i * a.group;
  const Sees s = sees(a, rq, i);
  const float inv = 1.0f / sum;
  uint32_t w[N / 2];
#pragma unroll
  for (int c = 0; c < N / 2; ++c) w[c] = s.hi > s.lo ? round2<DT>(o[2 * c] * inv, o[2 * c + 1] * inv) : 0u;
  MDBF_GLOBAL uint16_t* to = (MDBF_GLOBAL uint16_t*)a.out + (int64_t)(rq.start + i) * a.ldo + (int64_t)(head * a.group + g) * a.head_dim + c0;
  if (a.wide_o) {
#pragma unroll
    for (int c = 0; c < N / 4; ++c) ((MDBF_GLOBAL U32x2*)to)[c] = U32x2{w[2 * c], w[2 * c + 1]};
  } else {
#pragma unroll
    for (int c = 0; c < N / 2; ++c) {
      to[2 * c] = (uint16_t)w[c];
      to[2 * c + 1] = (uint16_t)(w[c] >> 16);
    }
  }
}

constexpr int kTile = 64;        // tokens per step of a wave
constexpr int kWaves = 4;
constexpr int kRows = 16;        // query rows of a workgroup
constexpr float kSlack = 8;      // powers of two by which a score may exceed the running reference
// powers of two by which numerators are larger than e^(z - m), a factor that the division takes out again: with kSlack they stay
// below 2^15 in fp16; bf16 has fp32's exponents
template <int DT>
constexpr float kLift = DT == MDBF_F16 ? 7 : 0;

// The tokens that a tile of ROWS query rows sees.
struct Span {
  int lo, hi;              // what any row sees
  int all_lo, all_hi;      // what all rows see
  int from, units;         // the tiles of tokens from the first one's on; one where nothing is seen: the rows are written
};
template <int ROWS>
__device__ __forceinline__ Span span_of(const AttnArgs& a, const Request& rq, int tile, int rows) {
  const Sees s0 = sees(a, rq, token_of(a, tile * ROWS)), s1 = sees(a, rq, token_of(a, min(tile * ROWS + ROWS - 1, rows - 1)));
  Span s = {s0.lo, s1.hi, s1.lo, s0.hi, s0.lo & ~(kTile - 1), 1};
  if (s.hi > s.lo) s.units = (s.hi - s.from + kTile - 1) / kTile;
  return s;
}

__device__ __forceinline__ int64_t uniform(int64_t x) {
  return ((int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// sum over a wave up to and with this lane's x
__device__ __forceinline__ int64_t scan_64(int64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(x, o);
    if (lane >= o) x += u;
  }
  return x;
}
// sum over a workgroup of four waves up to and with this thread's x; `total` of all
__device__ __forceinline__ int64_t scan_256(int64_t x, int64_t& total, int64_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = scan_64(x);
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) x += waves[w];
    total += waves[w];
  }
  return x;
}

// What a workgroup does: tiles of ROWS query rows of a request and kv head, one after the other, and of their tokens the units
// (tiles of 64) u0 .. u1 - 1.
//
// Either each takes row tiles with all of their tokens.  Or the units of all requests, row tiles and kv heads, one after the
// other and COST more in front of them for each row tile (what beginning and ending one takes), are cut into equal shares, a
// workgroup's each, so that requests of any lengths keep the device evenly busy.  A workgroup finishes the row tiles that lie
// whole in its share; of the first and the last one it may have a part only, whose sums it leaves in the workspace (two places
// each), and where a row tile begins in a share and ends in a later one a note for the join: request, row tile, kv head, and
// the number of workgroups whose shares it lies in, this one the first; 0 if none begins here.
typedef int32_t Note __attribute__((ext_vector_type(4)));
constexpr int kLeastShare = 4;      // units
template <int ROWS, int COST>
struct Work {
  int b, rt, head, u0 = 0, u1 = 0;
  int64_t left = 0, share = 0;
  Request rq;
  Span sp;

  // of a request's row tiles from, from + step, ..., in all kv heads
  __device__ static __forceinline__ int64_t units_of(const AttnArgs& a, int b, int from, int step) {
    const Request r = request_of(a, b);
    const int rows = r.fresh * a.group;
    int64_t n = 0;
    for (int t = from; t * ROWS < rows; t += step) n += span_of<ROWS>(a, r, t, rows).units + COST;
    return n * a.kv_heads;
  }
  // the units of the row tile that lie in the share, which goes on with this place among COST + units
  __device__ __forceinline__ void cut(int place) {
    const int most = (int)min((int64_t)(sp.units + COST - place), left);
    u0 = max(place - COST, 0), u1 = place + most - COST;
    left -= most;
  }
  // all tokens of a row tile, if the request has it
  __device__ __forceinline__ void whole(const AttnArgs& a, int b_, int rt_, int head_) {
    b = b_, rt = rt_, head = head_;
    rq = request_of(a, b);
    const int rows = rq.fresh * a.group;
    if (rt * ROWS >= rows) return;
    sp = span_of<ROWS>(a, rq, rt, rows);
    u1 = sp.units;
  }
  // All tokens of a row tile, the idx-th of those that 64 requests or less have in a kv head: last ones first (which see most), of
  // all requests.  A lane counts a request's, then, for a place in the requests, the row tiles at later ones.
  __device__ __forceinline__ void whole_nth(const AttnArgs& a, int idx, int head_) {
    const int lane = threadIdx.x & 63;
    const int mine = lane < a.requests ? (request_of(a, lane).fresh * a.group + ROWS - 1) / ROWS : 0;
    int all = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) all += __shfl_xor(all, o);
    if (idx >= __builtin_amdgcn_readfirstlane(all)) return;
#pragma unroll 1
    for (int t = 0;; t += 64) {        // (later than a request's last are none: some place has idx or less)
      int later = 0;
#pragma unroll 1
      for (int r = 0; r < a.requests; ++r) later += max(__builtin_amdgcn_readlane(mine, r) - (t + lane + 1), 0);
      const uint64_t here = __ballot(later <= idx);
      if (!here) continue;
      const int l = __builtin_ctzll(here), nth = idx - __builtin_amdgcn_readlane(later, l);
      const bool has = mine > t + l;
      const uint64_t have = __ballot(has);
      whole(a, __builtin_ctzll(__ballot(has && __popcll(have & ((1ull << lane) - 1)) == nth)), t + l, head_);
      return;
    }
  }
  // This workgroup's share: prefix sums over the requests, of up to 64 by every wave for itself, which deals its lanes out to
  // them, else by the workgroup, 256 at a time, first of all and then again up to the one where the share begins; and in that
  // one over its row tiles, 64 at a time.  1500 rows of 8 heads and 1 kv head of 128 against 9500 tokens, 94 row tiles: 74 us, 93
  // where a lane went over them one by one.  `find`: six words of LDS that nothing else uses.
  __device__ __forceinline__ void first(const AttnArgs& a, int64_t* find) {
    const int tid = threadIdx.x, lane = tid & 63;
    const bool few = a.requests <= 64;
    int64_t total = 0, sum, mine = 0, end = 0;
    if (few) {
      int bits = 6;                    // one lane each, or where there are row tiles to go over 64 >> bits, of 2^bits requests or less
      if (a.row_tiles > 1) bits = 32 - __builtin_clz(a.requests) - !(a.requests & (a.requests - 1));
      const int of = lane & ((1 << bits) - 1);
      if (of < a.requests) mine = units_of(a, of, lane >> bits, 64 >> bits);
      for (int o = 1 << bits; o < 64; o <<= 1) mine += __shfl_xor(mine, o);
      if (lane >> bits) mine = 0;
      end = scan_64(mine);
      total = __shfl(end, 63);
    } else {
      for (int r0 = 0; r0 < a.requests; r0 += 256) {
        scan_256(r0 + tid < a.requests ? units_of(a, r0 + tid, 0, 1) : 0, sum, find);
        total += sum;
      }
    }
    total = uniform(total);      // (what the loops below go by must be known to be the same in all lanes)
    share = max((total + a.shares - 1) / a.shares, (int64_t)kLeastShare);
    const int64_t start = blockIdx.x * share;
    if (tid == 0) ((MDBF_GLOBAL Note*)a.part)[blockIdx.x] = Note{0, 0, 0, 0};
    if (start >= total) return;
    left = min(share, total - start);
    int64_t rest;
    if (few) {
      b = __builtin_ctzll(__ballot(start >= end - mine && start < end));
      rest = start - __shfl(end - mine, b);
    } else {
      int64_t before = 0;
      for (int r0 = 0; r0 < a.requests; r0 += 256) {
        mine = r0 + tid < a.requests ? units_of(a, r0 + tid, 0, 1) : 0;
        end = before + scan_256(mine, sum, find);
        if (start >= end - mine && start < end) find[4] = r0 + tid, find[5] = end - mine;
        before += sum;
        if (start < before) break;
      }
      __syncthreads();
      b = (int)find[4];
      rest = start - find[5];
    }
    b = __builtin_amdgcn_readfirstlane(b);
    rest = uniform(rest);
    rq = request_of(a, b);
    const int rows = rq.fresh * a.group;
    rt = 0;
    for (int t0 = 0; rows > ROWS; t0 += 64) {      // (rest is less than the request's units: one of its row tiles has it)
      mine = 0;
      if ((t0 + lane) * ROWS < rows) mine = (int64_t)(span_of<ROWS>(a, rq, t0 + lane, rows).units + COST) * a.kv_heads;
      end = scan_64(mine);
      const uint64_t past = __ballot(rest < end);
      if (past) {
        rt = t0 + __builtin_ctzll(past);
        rest = uniform(rest - __shfl(end - mine, rt - t0));
        break;
      }
      rest = uniform(rest - __shfl(end, 63));
    }
    sp = span_of<ROWS>(a, rq, rt, rows);
    head = (int)(rest / (sp.units + COST));
    cut((int)(rest % (sp.units + COST)));
  }
  __device__ __forceinline__ bool any() const { return u1 > 0; }      // (a share may end before a row tile's first unit)
  __device__ __forceinline__ bool part() const { return u1 - u0 < sp.units; }
  __device__ __forceinline__ void note(const AttnArgs& a) const {
    if (u0 == 0 && u1 < sp.units && threadIdx.x == 0)
      ((MDBF_GLOBAL Note*)a.part)[blockIdx.x] = Note{b, rt, head, 1 + (int)((sp.units - u1 + share - 1) / share)};
  }
  // on to what is next
  __device__ __forceinline__ void next(const AttnArgs& a) {
    int rows = rq.fresh * a.group;
    u1 = 0;
    if (!a.shares) {
      rt += a.row_tiles;
      if ((int64_t)rt * ROWS >= rows) return;
      sp = span_of<ROWS>(a, rq, rt, rows);
      u1 = sp.units;
      return;
    }
    if (left <= 0) return;
    if (++head == a.kv_heads) {
      head = 0;
      ++rt;
      while (rt * ROWS >= rows) {        // (units are left: there is a request with rows)
        rq = request_of(a, ++b);
        rows = rq.fresh * a.group;
        rt = 0;
      }
      sp = span_of<ROWS>(a, rq, rt, rows);
    }
    cut(0);
  }
};
// sums of a part of a row tile: ROWS x D of them, then ROWS maxima and ROWS sums of numerators; where this workgroup's go, and those
// of the p-th workgroup of a note at wg (the first part lies in the second place)
template <int D, int ROWS>
constexpr int part_floats = ROWS * (D + 2);
template <int D, int ROWS>
__device__ __forceinline__ MDBF_GLOBAL float* part_at(const AttnArgs& a, int wg, bool second) {
  return (MDBF_GLOBAL float*)((MDBF_GLOBAL Note*)a.part + a.shares) + (int64_t)(2 * wg + second) * part_floats<D, ROWS>;
}

// Few rows: what beginning and ending a row tile costs.  64 requests of up to 8192 tokens, 8 kv heads of 128: 79 us with 0, 62.4
// with 3, 59.2 with 6, 58.6 with 10, 60.5 with 16.
constexpr int kRowsCost = 8;
// the workgroups that the device holds at once
template <int D>
constexpr int kFewShares = 256 * (D == 64 ? 4 : D == 128 ? 3 : 2);

constexpr int kNonTemporal = 2;  // of the buffer loads: the cache is read once

// Where a wave's tile of 64 tokens lies: NP pages' parts for the head (as buffers: a lane's place in the tile is the offset), and
// whether those are pages of the pool.
template <int NP>
struct Place {
  const uint8_t* base[NP];
  __amdgpu_buffer_rsrc_t buf[NP];
  int off[NP];               // of the first token in its page
  bool there[NP];
  __device__ __forceinline__ void set(const AttnArgs& a, int head, int head_bytes, int tok, const int (&page)[NP]) {
#pragma unroll
    for (int f = 0; f < NP; ++f) {
      there[f] = (uint32_t)page[f] < (uint32_t)a.pages;
      base[f] = a.cache + ((int64_t)(there[f] ? page[f] : 0) * a.kv_heads + head) * head_bytes;
      buf[f] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base[f]), 0, head_bytes, 0x00027000);
      off[f] = (tok + kTile / NP * f) & ((1 << a.page_shift) - 1);
    }
  }
};

// Codes and scales of the tile's keys and values as loaded.  Nothing in the loads looks at what they bring: they are in flight
// while the tile before is worked on.
template <int D, int NP>
struct Codes {
  static constexpr int KW = D / 32;                  // dwords of codes per lane and 16 keys = matrix steps over the channels
  static constexpr int KS = D <= 128 ? 1 : D / 128;  // scales among them
  static constexpr int VU = D / 64;                  // 16-byte units of values per lane and 32 tokens
  uint32_t kc[4][KW], ks[4][KS];
  U32x4 vc[2][VU];
  uint32_t vs[2][VU];

  __device__ __forceinline__ void load_keys(const Place<NP>& at, int page_shift, int lane) {
    const int P = 1 << page_shift, r = lane & 15, h = lane >> 4;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int pg = f * NP / 4, off = at.off[pg] + 16 * (f - pg * (4 / NP));
      if (KW == 2) {
        const U32x2 v = __builtin_amdgcn_raw_buffer_load_b64(at.buf[pg], r * (D / 2) + h * (D / 8), off * (D / 2), kNonTemporal);
        kc[f][0] = v[0], kc[f][1] = v[1];
      } else {
#pragma unroll
        for (int s = 0; s < KW; s += 4) {
          const U32x4 v = __builtin_amdgcn_raw_buffer_load_b128(at.buf[pg], r * (D / 2) + h * (D / 8) + 4 * s, off * (D / 2), kNonTemporal);
#pragma unroll
          for (int w = 0; w < 4; ++w) kc[f][(s + w) % KW] = v[w];
        }
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
        ks[f][s] = __builtin_amdgcn_raw_buffer_load_b8(at.buf[pg], r * (D / 32) + (D == 64 ? h >> 1 : h * KS + s), P * D + off * (D / 32), 0);
    }
  }
  // a lane's units: 32 tokens x D / 32 blocks, one after the other
  __device__ __forceinline__ void load_values(const Place<NP>& at, int page_shift, int lane) {
    const int P = 1 << page_shift;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int n = 0; n < VU; ++n) {
        if (NP == 4 && D == 64) {      // a load's halves lie in different pages
          const MDBF_GLOBAL uint8_t* from = (const MDBF_GLOBAL uint8_t*)(lane < 32 ? at.base[2 * g % NP] : at.base[(2 * g + 1) % NP]);
          const uint32_t o = lane < 32 ? at.off[2 * g % NP] : at.off[(2 * g + 1) % NP], u = lane & 31;
          vc[g][n] = __builtin_nontemporal_load((const MDBF_GLOBAL U32x4*)(from + (P + o) * (D / 2) + u * 16));
          vs[g][n] = from[P * (D + D / 32) + o * (D / 32) + u];
        } else {
          const int f = NP == 4 ? 2 * g + n / (VU / 2 ? VU / 2 : 1) : 2 * g;      // 16 tokens that the unit's page begins with
          const int pg = f * NP / 4, first = at.off[pg] + 16 * (f - pg * (4 / NP));
          const int u = (NP == 4 ? n % (VU / 2 ? VU / 2 : 1) : n) * 64 + lane;
          vc[g][n] = __builtin_amdgcn_raw_buffer_load_b128(at.buf[pg], u * 16, (P + first) * (D / 2), kNonTemporal);
          vs[g][n] = __builtin_amdgcn_raw_buffer_load_b8(at.buf[pg], u, P * (D + D / 32) + first * (D / 32), 0);
        }
      }
  }
};

// max over the four lanes that hold a query row, and their sum
__device__ __forceinline__ float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  x = fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
  const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t b0 = b[0], b1 = b[1];
  return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// 16 query rows of one kv head at a time, the tiles of their tokens dealt out to the four waves, which meet at the end.  The
// registers that a tile's keys were in take the next tile's as soon as the scores are there, those of its values once they
// are in LDS; page numbers are looked up a tile earlier still.  NP: pages per tile of 64 tokens (1, 2 or 4).
//
// Bound by the cache's bytes where that is long: 64 requests of up to 8192 tokens, 32 heads on 8 of 128 (295 MB), 55 us and 5 for
// the join, 5.2 TB/s of the 6.0 that a plain read reaches; one of 200000 tokens (218 MB) 41 and 6 us.  Matrix cores are busy for an
// eighth of that.  Short caches are a launch's latency and each wave's chain of page number, codes, scores, values and the meeting of the
// waves: 4 requests of up to 701 tokens, 32 heads of 128 (8 MB), 10.6 us.
template <int D, int DT, int NP>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 4 : D == 128 ? 3 : 2) void attn_few_kernel(AttnArgs a) {
  using Tile = Codes<D, NP>;
  constexpr int KW = Tile::KW, KS = Tile::KS, VU = Tile::VU;
  constexpr int kGroup = 32;                  // tokens whose values are in LDS at a time
  // A token's values in LDS: 64 bytes per block, 16 more after each (D = 64) or every second one, rows an odd multiple of 32
  // bytes apart: neither the writes nor the transposing reads meet on a bank.
  constexpr int VROW = D == 64 ? 160 : D == 128 ? 288 : 608;
  auto block_at = [](int g) { return g * 64 + (D == 64 ? g : g >> 1) * 16; };
  constexpr int CT = D / 16;                  // channel tiles
  constexpr int OROW = D + 4;                 // floats of a row of results in LDS
  static_assert(kGroup * VROW >= kRows * OROW * 4, "the results fit the values' place");
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves][kGroup * VROW];
  __shared__ float stat[kWaves][2][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
  const int head_bytes = (int)kv_head_bytes(1 << a.page_shift, D);
  unsigned char* vals = lds[wave];

  Work<kRows, kRowsCost> work;
  if (a.shares) {
    __shared__ int64_t find[6];
    work.first(a, find);
  } else {      // a workgroup per row tile that the launch was sized for
    const uint32_t idx = blockIdx.x / a.row_tiles;
    work.whole(a, idx / a.kv_heads, blockIdx.x % a.row_tiles, idx % a.kv_heads);
  }

  for (; work.any(); work.next(a)) {
    const Request rq = work.rq;
    const Span sp = work.sp;
    const int b = work.b, rt = work.rt, head = work.head, u0 = work.u0, u1 = work.u1, rows = rq.fresh * a.group;
    const MDBF_CONST int32_t* table = (const MDBF_CONST int32_t*)a.table + b * a.table_ld;
    const int R = rt * kRows + r;
    const bool valid = R < rows;
    const int i = valid ? token_of(a, R) : 0, g = valid ? R - i * a.group : 0;
    Sees me = sees(a, rq, i);
    if (!valid) me.hi = me.lo = 0;
    const int tmin = u0 ? sp.from + u0 * kTile : sp.lo, tmax = u1 < sp.units ? sp.from + u1 * kTile : sp.hi;

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
        qf[s] ^= a.flip;
      }
    }

    float m = -INFINITY, l = 0;
    uint32_t nan_blocks = 0;       // blocks of channels in which the row sees a NaN
    F32x4 acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = F32x4{0, 0, 0, 0};

    // page numbers of a tile; behind the last token's none is looked up
    auto pages_of = [&](int t, int (&page)[NP]) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < NP; ++f) page[f] = table[min(t + kTile / NP * f, rq.len - 1) >> a.page_shift];
    };

    constexpr int kStep = kWaves * kTile;
    int t0 = (tmin & ~(kTile - 1)) + wave * kTile;
    if (t0 < tmax) {
      Tile x;
      Place<NP> at, next;
      int page[NP];
      pages_of(t0, page);
      at.set(a, head, head_bytes, t0, page);
      x.load_keys(at, a.page_shift, lane);
      x.load_values(at, a.page_shift, lane);
      pages_of(t0 + kStep, page);
      for (;;) {
        const bool more = t0 + kStep < tmax;
        next.set(a, head, head_bytes, t0 + kStep, page);
        pages_of(t0 + 2 * kStep, page);

        // scores (without their factor): a lane holds those of its row with tokens 4 h + 0 .. 3 of each 16
        F32x4 z[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          if (!at.there[f * NP / 4]) {      // a page that is none reads as NaN
#pragma unroll
            for (int s = 0; s < KS; ++s) x.ks[f][s] = kKvNanScale;
          }
          z[f] = F32x4{0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < KW; ++s) z[f] = mma16<DT>(numbers<DT>(x.kc[f][s], unit_of(known_scale<DT>(x.ks[f][KS == 1 ? 0 : s / 4]))), qf[s], z[f]);
        }
        if (more) x.load_keys(next, a.page_shift, lane);
        const bool inside = t0 >= sp.all_lo && t0 + kTile <= sp.all_hi;     // every row sees every token
        if (!inside) {
#pragma unroll
          for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int tok = t0 + 16 * f + 4 * h + j;
              if (tok < me.lo || tok >= me.hi) z[f][j] = -INFINITY;
            }
        }
        // A row's reference m follows its maximum only where that has grown by more than kSlack (numerators stay below
        // 2^(kSlack + kLift), in reach of fp16): most tiles exchange nothing between lanes and rescale nothing.  Rows that others bring here keep theirs
        // (a factor of 1): a row's bits depend on its own scores alone.
        float top = z[0][0];
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
          for (int j = 0; j < 4; ++j) top = fmaxf(top, z[f][j]);
        top *= a.scale;
        if (__any(top > m + kSlack)) {
          const float high = row_max(top), mn = high > m + kSlack ? high : m;
          const float alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
          m = mn;
          l *= alpha;
#pragma unroll
          for (int c = 0; c < CT; ++c) acc[c] *= alpha;
        }
        const float use = m == -INFINITY ? 0.0f : m - kLift<DT>;
        U32x4 pf[2];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) z[f][j] = __builtin_amdgcn_exp2f(z[f][j] * a.scale - use);
          l += (z[f][0] + z[f][1]) + (z[f][2] + z[f][3]);
          pf[f / 2][f % 2 * 2] = round2<DT>(z[f][0], z[f][1]);
          pf[f / 2][f % 2 * 2 + 1] = round2<DT>(z[f][2], z[f][3]);
        }

#pragma unroll
        for (int g = 0; g < 2; ++g) {
          // values that no row sees are zeros; NaN among the others goes to the rows that see it, not through the product, where
          // a zero weight would bring it to all rows
#pragma unroll
          for (int n = 0; n < VU; ++n) {
            const int unit = n * 64 + lane, row = unit / (D / 32), tok = t0 + kGroup * g + row;
            if (NP > 1 || !at.there[0]) {
              const int f = 2 * g + row / 16;
              bool there = at.there[0];
#pragma unroll
              for (int k = 1; k < NP; ++k)
                if (f * NP / 4 == k) there = at.there[k];
              if (!there) x.vs[g][n] = kKvNanScale;
            }
            if (!inside && (tok < sp.lo || tok >= sp.hi)) {
              x.vc[g][n] = U32x4{0, 0, 0, 0};
              x.vs[g][n] = 127;
            }
            uint64_t bad = __ballot(x.vs[g][n] > kKvScaleMax[DT]);
            if (bad) {
              if (x.vs[g][n] > kKvScaleMax[DT]) {
                x.vc[g][n] = U32x4{0, 0, 0, 0};
                x.vs[g][n] = 127;
              }
              for (; bad; bad &= bad - 1) {
                const int bu = n * 64 + __builtin_ctzll(bad), bt = t0 + kGroup * g + bu / (D / 32);
                if (bt >= me.lo && bt < me.hi) nan_blocks |= 1u << bu % (D / 32);
              }
            }
            const float unit_f = unit_of(x.vs[g][n]);
            unsigned char* to = vals + row * VROW + block_at(unit % (D / 32));
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<U32x4*>(to + w * 16) = numbers<DT>(x.vc[g][n][w], unit_f);
          }
          if (g == 1 && more) x.load_values(next, a.page_shift, lane);
          wave_lds_order();
          // a lane's channel of tokens 4 h + 0 .. 3 of each 16: the order of the scores' registers
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            const unsigned char* from = vals + (4 * h + (r >> 2)) * VROW + block_at(c / 2) + (c & 1) * 32 + (r & 3) * 8;
            const U32x2 v0 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)from));
            const U32x2 v1 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)(from + 16 * VROW)));
            acc[c] = mma16<DT>(U32x4{v0[0], v0[1], v1[0], v1[1]}, pf[g], acc[c]);
          }
          wave_lds_order();
        }
        if (!more) break;
        at = next;
        t0 += kStep;
      }
    }

#pragma unroll
    for (int c = 0; c < CT; ++c)
      if (nan_blocks >> (c / 2) & 1) acc[c] = F32x4{NAN, NAN, NAN, NAN};

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
      const int row = threadIdx.x >> 4, piece = threadIdx.x & 15;
      const int Ro = rt * kRows + row;
      if (Ro < rows) {
        float top = stat[0][0][row];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, stat[w][0][row]);
        const float use = top == -INFINITY ? 0.0f : top;
        float sum = 0, o[N];
#pragma unroll
        for (int c = 0; c < N; ++c) o[c] = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(stat[w][0][row] - use);
          sum += f * stat[w][1][row];
          const float* from = reinterpret_cast<const float*>(lds[w]) + row * OROW + piece * N;
#pragma unroll
          for (int c = 0; c < N; ++c) o[c] += f * from[c];
        }
        if (work.part()) {
          MDBF_GLOBAL float* to = part_at<D, kRows>(a, blockIdx.x, u0 == 0);
          if (piece == 0) {
            to[kRows * D + row] = top;
            to[kRows * (D + 1) + row] = sum;
          }
#pragma unroll
          for (int c = 0; c < N / 4; ++c)
            ((MDBF_GLOBAL F32x4*)(to + row * D + piece * N))[c] = F32x4{o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]};
        } else {
          store_row<DT, N>(a, rq, head, Ro, piece * N, o, sum);
        }
      }
    }
    work.note(a);
    __syncthreads();
  }
}

// Joins the parts of the row tiles that several shares have: W waves per row and share where one begins.  D / 4 lanes side by
// side on the channels take a part at a time, other lanes and waves the next ones; the order is fixed.
template <int D, int DT, int ROWS, int W>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int L = D / 4, GROUPS = 64 / L, AHEAD = 8;
  __shared__ F32x4 sums[W][L];
  const int lane = threadIdx.x & 63, l = lane % L, grp = lane / L, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = W == 1 ? 0 : wave;
  const uint32_t idx = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  const int row0 = idx % a.join_rows, wg = idx / a.join_rows;
  if (wg >= a.shares) return;
  const Note note = ((const MDBF_GLOBAL Note*)a.part)[wg];
  const int rt = note[1], head = note[2], count = note[3];
  if (count < 2) return;
  const Request rq = request_of(a, note[0]);
  const int rows = rq.fresh * a.group;
  auto part = [&](int p) { return (const MDBF_GLOBAL float*)part_at<D, ROWS>(a, wg + p, p == 0); };
  for (int row = row0; row < ROWS && rt * ROWS + row < rows; row += a.join_rows) {
    float top = -INFINITY;
    for (int p = lane; p < count; p += 64) top = fmaxf(top, part(p)[ROWS * D + row]);
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
    const float use = top == -INFINITY ? 0.0f : top;
    F32x4 o = {0, 0, 0, 0};
    float sum = 0;
    for (int p0 = 0; p0 < count; p0 += 64) {
      const int some = min(64, count - p0);
      float f = 0;
      if (lane < some) {
        const MDBF_GLOBAL float* q = part(p0 + lane);
        f = __builtin_amdgcn_exp2f(q[ROWS * D + row] - use);
        sum += f * q[ROWS * (D + 1) + row];
      }
      for (int p = mine * GROUPS; p < some; p += GROUPS * W * AHEAD) {
        F32x4 v[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int at = p + k * GROUPS * W + grp;
          if (at < some) v[k] = *(const MDBF_GLOBAL F32x4*)(part(p0 + at) + row * D + l * 4);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int at = p + k * GROUPS * W + grp;
          const float w = __shfl(f, at & 63);
          if (at < some) o += w * v[k];
        }
      }
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
#pragma unroll
    for (int w = L; w < 64; w <<= 1)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += __shfl_xor(o[c], w);
    if (W > 1) {
      if (grp == 0) sums[mine][l] = o;
      __syncthreads();
      if (mine == 0)
#pragma unroll
        for (int w = 1; w < W; ++w) o += sums[w][l];
    }
    const float v[4] = {o[0], o[1], o[2], o[3]};
    if (grp == 0 && mine == 0) store_row<DT, 4>(a, rq, head, rt * ROWS + row, l * 4, v, sum);
    if (W > 1) __syncthreads();
  }
}

// ---- prompts ---------------------------------------------------------------------------------------------
// 128 query rows of one kv head per workgroup, 32 per wave, which all read the tile of 64 tokens that the workgroup has in
// LDS: key codes as they are, values as numbers.  Two buffers:
// while one is worked on, the next tile's codes, which came in while the one before was, are written into the other.
//
// K Q^T are block-scaled products of fp4 and fp6, at four times the 16-bit rate, so that three or four of them, one for each limb
// of the queries, are no dearer than one of 16 bits and its conversions of the keys.  Long prompts are bound by instruction
// issue: two waves a SIMD, for whose softmax and values the vector unit is busy 57 % of the cycles and the matrix core 49 %, seldom
// both.  2048 tokens behind 14336, 32 heads on 8 of 128 (515 Gflop): 425 to 444 us, 1.16 to 1.21 Pflop/s of the 1.26 that a large
// 16-bit product reaches; in fp16, a limb more, 485 to 500.
// Short ones are latency: 1.0 us (D = 64) or 1.25 (128) per tile of tokens with one workgroup on a compute unit, 1.1 or 1.85 for two.
// Tried: eight waves in two halves that take turns at the tiles and add up at the end, half as many workgroups: 512 tokens of 32
// heads 17.0 -> 16.3 us, calls in shares as before, prompts of 300 tokens of 4 requests 42 -> 48: not kept.
constexpr int kManyWaves = 4, kManyRows = 32 * kManyWaves;
constexpr int kManyCost = 4;      // units that beginning and ending a row tile costs
template <int D>
constexpr int kManyShares = 256 * (D <= 128 ? 2 : 1);
typedef float F32x16 __attribute__((ext_vector_type(16)));

template <int DT>
__device__ __forceinline__ F32x16 mma32(U32x4 a, U32x4 b, F32x16 c) {
  if (DT == MDBF_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b), c, 0, 0, 0);
}
// Key codes (fp4, 32 per lane, with their block's scale byte at SA of `scales`) times limb L of the queries, summed into c.
typedef int V8i __attribute__((ext_vector_type(8)));
template <int SA, int L>
__device__ __forceinline__ F32x16 mx32(U32x4 codes, uint32_t scales, v6u limb, uint32_t limb_scales, F32x16 c) {
  const V8i x = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
  const V8i y = {(int)limb[0], (int)limb[1], (int)limb[2], (int)limb[3], (int)limb[4], (int)limb[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 2, SA, (int)scales, L, (int)limb_scales);
}
// f(0), f(1), ... with indices that are constants
template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// 32 channels of a query as a sum of NL fp6 numbers, each limb's scale 2^-4 of the one before: an absolute error of 1.07 * 2^-(4 NL + 2)
// of the largest of the 32 at most.  Three limbs for bf16 and four for fp16: in a score of ten that is no more than the rounding of its
// numerator, 2^-9 and 2^-12, and for a channel down to a 32nd (bf16) or 64th (fp16) of the largest no more than half a spacing of the
// type.  Where one channel is far beyond the others it is much of what those are (a thousand times: 2.4 % of the result in bf16 if
// the keys are as far the other way, 0.17 in fp16; 32 times: 0.1 and 0.007): MDBF_ATTN_EXACT_QUERIES.
template <int NL>
struct Limbs {
  v6u limb[NL];
  uint32_t scales = 0;      // a byte each
  // whether all values are finite; where not, the limbs mean nothing
  __device__ __forceinline__ bool set(float (&q)[32]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) top = max(top, __builtin_bit_cast(uint32_t, q[j]) & 0x7fffffffu);
    const int e = min(max((int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x700000u), 16), 254);      // at most 7.5 units
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      const float unit = __builtin_bit_cast(float, (uint32_t)(e - 4 * k) << 23);
      scales |= (uint32_t)(e - 4 * k) << (8 * k);
      limb[k] = fp6_encode32(q, unit);
      if (k + 1 < NL) {
        const v32f back = fp6_decode32(limb[k], unit);
#pragma unroll
        for (int j = 0; j < 32; ++j) q[j] -= back[j];
      }
    }
    return (top >> 23) != 255;
  }
};

// max over the two lanes that hold a query row
__device__ __forceinline__ float pair_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  return fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
}

// CROWD: waves that feed products go first (see kCrowds).  EXACT: queries as they are, in 16-bit products for which every wave makes
// numbers of the key codes: 2048 tokens behind 14336, 32 heads on 8 of 128, 427 -> 479 us (fp16 476 -> 500), 1000 behind 5000, 32 of
// 64, 84 -> 97; 300 behind 2000 of 2 requests, 16 on 4 of 256 in fp16, 50 -> 47.
template <int D, int DT, bool CROWD, bool EXACT>
__global__ __launch_bounds__(64 * kManyWaves, D <= 128 ? 2 : 1) void attn_many_kernel(AttnArgs a) {
  constexpr int BL = D / 32;                       // blocks of a token
  constexpr int UNITS = kTile * BL;                // 16-byte units of a tile's keys, and of its values
  constexpr int U = UNITS < 256 ? 1 : UNITS / 256; // of each per thread; with D = 64 half of the threads take keys, half values
  constexpr int KROW = D / 2 + 16;                 // bytes of a token's key codes in LDS: reads of 16 bytes a lane meet on no bank
  // of its values: blocks 80 bytes apart and rows 64 more than a multiple of 256, so that the writes and the transposing reads
  // (which take two times 16 channels of four rows at once) do not meet on a bank where a row has four blocks.  With D = 64, two
  // blocks a row, writes of rows four apart do: 22 % of the LDS' cycles in prompts of odd lengths (D = 128: 6 %).
  constexpr int VROW = D == 256 ? 832 : 320;
  auto block_at = [](int g) { return g * 80; };
  constexpr int ST = D / 64;                       // pairs of blocks
  constexpr int NL = DT == MDBF_F16 ? 4 : 3;       // limbs of the queries
  constexpr int CT = D / 32;                       // channel tiles
  struct Buffer {
    unsigned char keys[kTile * KROW];
    unsigned char values[kTile * VROW];
    unsigned char key_scales[kTile * BL], value_scales[kTile * BL];
  };
  __shared__ __attribute__((aligned(16))) Buffer lds[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, hh = lane >> 5;
  const int P = 1 << a.page_shift, head_bytes = (int)kv_head_bytes(P, D);

  Work<kManyRows, kManyCost> work;
  if (a.shares) {
    __shared__ int64_t find[6];
    work.first(a, find);
  } else {      // kv heads next to each other (their row tiles then share an XCD's cache), the row tiles that see most first
    const uint32_t idx = blockIdx.x / a.kv_heads;
    if (a.nth) work.whole_nth(a, idx, blockIdx.x % a.kv_heads);
    else work.whole(a, idx % a.requests, a.row_tiles - 1 - idx / a.requests, blockIdx.x % a.kv_heads);
  }

  for (; work.any(); work.next(a)) {
    const Request rq = work.rq;
    const Span sp = work.sp;
    const int rt = work.rt, head = work.head, rows = rq.fresh * a.group;
    const MDBF_GLOBAL int32_t* table = (const MDBF_GLOBAL int32_t*)a.table + work.b * a.table_ld;
    const MDBF_GLOBAL uint8_t* cache = (const MDBF_GLOBAL uint8_t*)a.cache + (int64_t)head * head_bytes;
    const int R = rt * kManyRows + wave * 32 + r;
    const bool valid = R < rows;
    const int i = valid ? token_of(a, R) : 0, g = valid ? R - i * a.group : 0;
    Sees me = sees(a, rq, i);
    if (!valid) me.hi = me.lo = 0;

    // a thread's units of a tile: its page is looked up a tile before its codes are requested
    U32x4 kc[U], vc[U];
    uint32_t ks[U], vs[U];
    int page[U];
    bool there[U];
    auto unit_of_thread = [&](int n) { return D == 64 ? tid & 127 : n * 256 + tid; };
    auto look_up = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < U; ++n) page[n] = table[max(min(t + unit_of_thread(n) / BL, rq.len - 1), 0) >> a.page_shift];
    };
    auto request = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < U; ++n) {
        const int u = unit_of_thread(n), off = (t + u / BL) & (P - 1), bl = u % BL;
        there[n] = (uint32_t)page[n] < (uint32_t)a.pages;
        const MDBF_GLOBAL uint8_t* from = cache + (int64_t)(there[n] ? page[n] : 0) * a.kv_heads * head_bytes;
        if (D != 64 || tid < 128) {
          kc[n] = *(const MDBF_GLOBAL U32x4*)(from + off * (D / 2) + bl * 16);
          ks[n] = from[P * D + off * BL + bl];
        }
        if (D != 64 || tid >= 128) {
          vc[n] = *(const MDBF_GLOBAL U32x4*)(from + (P + off) * (D / 2) + bl * 16);
          vs[n] = from[P * (D + BL) + off * BL + bl];
        }
      }
    };
    // tokens that no row sees: their values are zeros; NaN among the others stays in value_scales
    auto put = [&](Buffer& to, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < U; ++n) {
        const int u = unit_of_thread(n), row = u / BL, bl = u % BL, tok = t + row;
        if (D != 64 || tid < 128) {
          *reinterpret_cast<U32x4*>(to.keys + row * KROW + bl * 16) = kc[n];
          to.key_scales[u] = there[n] ? known_scale<DT>(ks[n]) : kKvNanScale;
        }
        if (D != 64 || tid >= 128) {
          uint32_t sc = there[n] ? vs[n] : kKvNanScale;
          if (tok < sp.lo || tok >= sp.hi) sc = 0;
          to.value_scales[u] = sc;
          if (sc - 1 >= kKvScaleMax[DT]) vc[n] = U32x4{0, 0, 0, 0}, sc = 127;      // 0, or read as NaN
#pragma unroll
          for (int w = 0; w < 4; ++w) *reinterpret_cast<U32x4*>(to.values + row * VROW + block_at(bl) + w * 16) = numbers<DT>(vc[n][w], unit_of(sc));
        }
      }
    };

    // the first tile is on its way while the queries are prepared
    const int tiles = sp.hi > sp.lo ? work.u1 - work.u0 : 0, begin = sp.from + work.u0 * kTile;
    look_up(begin);
    // queries: channels 64 s + 32 hh + 0 .. 31 of the lane's row for step s
    U32x4 raw[ST][4] = {};
    if (valid) {
      const MDBF_GLOBAL uint16_t* p = (const MDBF_GLOBAL uint16_t*)a.q + (int64_t)(rq.start + i) * a.ldq + (int64_t)(head * a.group + g) * D + 32 * hh;
#pragma unroll
      for (int s = 0; s < ST; ++s) {
        if (a.wide_q) {
#pragma unroll
          for (int w = 0; w < 4; ++w) raw[s][w] = ((const MDBF_GLOBAL U32x4*)(p + 64 * s))[w];
        } else {
#pragma unroll
          for (int w = 0; w < 16; ++w) raw[s][w / 4][w % 4] = (uint32_t)p[64 * s + 2 * w] | ((uint32_t)p[64 * s + 2 * w + 1] << 16);
        }
      }
    }
    request(begin);
    look_up(begin + kTile);
    Limbs<NL> ql[ST];
    bool finite = true;
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      if constexpr (EXACT) {
#pragma unroll
        for (int w = 0; w < 4; ++w) raw[s][w] ^= a.flip;
        continue;
      }
      float q[32];
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const uint32_t x = raw[s][w / 4][w % 4] ^ a.flip;
        if (DT == MDBF_F16) {
          const F16x2 v = __builtin_bit_cast(F16x2, x);
          q[2 * w] = (float)v[0] * a.scale, q[2 * w + 1] = (float)v[1] * a.scale;
        } else {
          q[2 * w] = __builtin_bit_cast(float, x << 16) * a.scale, q[2 * w + 1] = __builtin_bit_cast(float, x & 0xffff0000u) * a.scale;
        }
      }
      finite &= ql[s].set(q);
    }

    // The products' sums begin at -m, so that they end as the exponentials' arguments; with D = 256 no registers are left for
    // that, and 16-bit queries do not carry the scale.
    constexpr bool FROM_M = D <= 128 && !EXACT;
    F32x16 from_m;
#pragma unroll
    for (int j = 0; j < 16; ++j) from_m[j] = 0;
    float m = -INFINITY, use = 0, l = finite ? 0.0f : NAN;      // (a query that is not finite has no finite result)
    uint32_t nan_blocks = 0;
    F32x16 acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[c][j] = 0;

    if (tiles) {
      put(lds[0], begin);
      if (tiles > 1) {
        request(begin + kTile);
        look_up(begin + 2 * kTile);
      }
      __syncthreads();
    }
    for (int n = 0; n < tiles; ++n) {
      const int t0 = begin + n * kTile;
      if (n + 1 < tiles) put(lds[(n + 1) & 1], t0 + kTile);
      if (n + 2 < tiles) {
        request(t0 + 2 * kTile);
        look_up(t0 + 3 * kTile);
      }
      const Buffer& in = lds[n & 1];

      // scores: a lane holds those of its row with tokens 32 f + 8 (j / 4) + 4 hh + j % 4; two chains of products side by side
      F32x16 z[2];
      uint32_t sc[2][(BL + 3) / 4];      // the blocks' scale bytes, this half's at the even places
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const unsigned char* from = in.key_scales + (32 * f + r) * BL;
#pragma unroll
        for (int w = 0; w < (BL + 3) / 4; ++w)
          sc[f][w] = (BL == 2 ? *reinterpret_cast<const uint16_t*>(from) : reinterpret_cast<const uint32_t*>(from)[w]) >> (8 * hh);
        z[f] = from_m;
      }
      if (CROWD) __builtin_amdgcn_s_setprio(1);
      each_of([&](auto st) __attribute__((always_inline)) {
        constexpr int s = decltype(st)::value;
        U32x4 codes[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) codes[f] = *reinterpret_cast<const U32x4*>(in.keys + (32 * f + r) * KROW + (2 * s + hh) * 16);
        if constexpr (EXACT) {
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int f = 0; f < 2; ++f)
              z[f] = mma32<DT>(numbers<DT>(codes[f][w], unit_of(sc[f][s / 2] >> (16 * (s & 1)) & 255u)), raw[s][w], z[f]);
        } else each_of([&](auto k) __attribute__((always_inline)) {
          constexpr int L = NL - 1 - decltype(k)::value;      // the smallest first
#pragma unroll
          for (int f = 0; f < 2; ++f) z[f] = mx32<2 * (s & 1), L>(codes[f], sc[f][s / 2], ql[s].limb[L], ql[s].scales, z[f]);
        }, std::make_integer_sequence<int, NL>{});
      }, std::make_integer_sequence<int, ST>{});
      U32x2 v[2][CT][2];
      auto read = [&](int k) __attribute__((always_inline)) {
        const unsigned char* from = in.values + (16 * k + 4 * hh + ((lane & 15) >> 2)) * VROW + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          v[k & 1][c][0] = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)(from + block_at(c))));
          v[k & 1][c][1] = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)(from + block_at(c) + 8 * VROW)));
        }
      };
      read(0);
      if (CROWD) __builtin_amdgcn_s_setprio(0);
      if (t0 < sp.all_lo || t0 + kTile > sp.all_hi) {      // not every row sees every token
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int tok = t0 + 32 * f + 8 * (j / 4) + 4 * hh + j % 4;
            if (tok < me.lo || tok >= me.hi) z[f][j] = -INFINITY;
          }
      }
      float top = z[0][0];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, z[f][j]);
      if (EXACT) top *= a.scale;
      if (FROM_M) top += use;
      if (__any(top > m + kSlack)) {      // as in attn_few_kernel
        const float high = pair_max(top), mn = high > m + kSlack ? high : m;
        const float alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
        const float before = use;
        m = mn;
        use = m == -INFINITY ? 0.0f : m - kLift<DT>;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c] *= alpha;
        if (FROM_M) {
#pragma unroll
          for (int j = 0; j < 16; ++j) from_m[j] = -use, z[0][j] -= use - before, z[1][j] -= use - before;
        }
      }
      U32x4 pf[4];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          float p[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) p[k] = __builtin_amdgcn_exp2f(FROM_M ? z[f][j + k] : EXACT ? z[f][j + k] * a.scale - use : z[f][j + k] - use);
          l += (p[0] + p[1]) + (p[2] + p[3]);
          pf[2 * f + j / 8][j / 4 % 2 * 2] = round2<DT>(p[0], p[1]);
          pf[2 * f + j / 8][j / 4 % 2 * 2 + 1] = round2<DT>(p[2], p[3]);
        }

      // NaN among the values: to the rows that see it
      {
        // bytes beyond the type's largest, four at a time: the high bit, and a carry from the other seven into it
        constexpr uint32_t kRest = 0x7f7f7f7fu, kTo = (0xffu - kKvScaleMax[DT]) * 0x01010101u;
        uint32_t bad = 0;
#pragma unroll
        for (int w = 0; w < UNITS / 256; ++w) {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(in.value_scales + w * 256 + lane * 4);
          bad |= ((x & kRest) + kTo) & x;
        }
        if (UNITS < 256) {
          const uint32_t x = reinterpret_cast<const uint16_t*>(in.value_scales)[lane];
          bad |= ((x & kRest) + kTo) & x;
        }
        bad &= 0x80808080u;
        if (__any(bad)) {
          for (int u = 0; u < UNITS; ++u)
            if (in.value_scales[u] > kKvScaleMax[DT]) {
              const int tok = t0 + u / BL;
              if (tok >= me.lo && tok < me.hi) nan_blocks |= 1u << u % BL;
            }
        }
      }

      if (CROWD) __builtin_amdgcn_s_setprio(1);
      // results: 16 tokens at a time, in the order of the scores' registers; the values of the next 16 are read before the products
      // of these
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k < 3) read(k + 1);
#pragma unroll
        for (int c = 0; c < CT; ++c)
          acc[c] = mma32<DT>(U32x4{v[k & 1][c][0][0], v[k & 1][c][0][1], v[k & 1][c][1][0], v[k & 1][c][1][1]}, pf[k], acc[c]);
      }
      if (CROWD) __builtin_amdgcn_s_setprio(0);
      __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (valid && work.part()) {
      MDBF_GLOBAL float* to = part_at<D, kManyRows>(a, blockIdx.x, work.u0 == 0);
      const int row = wave * 32 + r;
      if (hh == 0) to[kManyRows * D + row] = m, to[kManyRows * (D + 1) + row] = l;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const bool nan = nan_blocks >> c & 1;
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          F32x4 v = {acc[c][j], acc[c][j + 1], acc[c][j + 2], acc[c][j + 3]};
          if (nan) v = F32x4{NAN, NAN, NAN, NAN};
          *(MDBF_GLOBAL F32x4*)(to + row * D + 32 * c + 2 * j + 4 * hh) = v;
        }
      }
    } else if (valid) {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const bool nan = nan_blocks >> c & 1;
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const float v[4] = {acc[c][j], acc[c][j + 1], acc[c][j + 2], acc[c][j + 3]};
          store_row<DT, 4>(a, rq, head, R, 32 * c + 2 * j + 4 * hh, v, nan ? NAN : l);
        }
      }
    }
    work.note(a);
  }
}

static int check_attn(const mdbf_kv_t* kv, const mdbf_attn_t* at, int requests, int T) {
  int st = check_kv(kv);
  if (st) return st;
  if (!at || requests < 1 || T < 1) return MDBF_EINVAL;
  if (at->q_heads <= 0 || at->q_heads % kv->kv_heads || at->window < 0 || at->max_fresh < 1 || at->max_length < 1 || !isfinite(at->scale) || at->scale == 0.0f)
    return MDBF_EINVAL;
  if (at->window && !(at->flags & MDBF_ATTN_CAUSAL)) return MDBF_EINVAL;
  if ((at->flags & ~(MDBF_ATTN_CAUSAL | MDBF_ATTN_EXACT_QUERIES)) || at->q_heads > (1 << 16)) return MDBF_EUNSUPPORTED;
  return MDBF_OK;
}

// Which kernel a call takes, and whether its work is cut into shares: by estimates of the time, in us, from the sizes that the
// caller bounds the call by.  Fitted to calls of 1 to 8192 new tokens behind 0 to 30000; what they get wrong costs up to a fifth
// where requests are of unequal lengths.  128 new tokens behind 30000, 32 heads on 8 of 128: few rows 161 us, prompts 515 whole and
// 78 cut; 40 behind 3000 of 8 requests: 32, 60 and 34; 1000 behind 4000: 188, 93 and 99.
constexpr int kWhole = 1024;      // tokens up to which nothing is cut: the join, a launch, would cost more
struct AttnCosts {
  double few;              // a unit of the few-row kernel where it fills the device
  double one, full;        // one of the prompts' kernel, with one workgroup on a compute unit, and with all that fit
  double parts;            // the parts that all workgroups of the prompts' kernel leave and the join takes
  int few_shares, many_shares;
};
static AttnCosts attn_costs(int d) {
  if (d == 64) return {1.5, 1.0, 1.1, 12, kFewShares<64>, kManyShares<64>};
  if (d == 128) return {1.0, 1.25, 1.85, 24, kFewShares<128>, kManyShares<128>};
  return {1.7, 2.45, 2.6, 24, kFewShares<256>, kManyShares<256>};
}
struct AttnGeom {
  int row_tiles;           // of a request and kv head; nth: of all requests and a kv head
  bool shares, many, nth, exact;
  bool distant;            // a row tile of the prompts' kernel sees 4096 tokens or more on average
};
static bool attn_cuts(const mdbf_attn_t& at) { return (at.window ? std::min(at.max_length, at.window) : at.max_length) > kWhole; }
static AttnGeom attn_geom(const mdbf_kv_t& kv, const mdbf_attn_t& at, int all, int T) {
  const AttnCosts k = attn_costs(kv.head_dim);
  const int fresh = std::min(at.max_fresh, T), requests = (int)(((int64_t)T + fresh - 1) / fresh);      // requests with as many new tokens as any
  const double rows = (double)fresh * (at.q_heads / kv.kv_heads);
  auto tiles_of = [&](int per) { return ceil(rows / per); };
  // units of a row tile: of the one that sees most, and on average
  auto units_of = [&](int per, bool most) {
    double span = at.max_length;
    if ((at.flags & MDBF_ATTN_CAUSAL) && !most) span -= std::min<double>(fresh, span) / 2;
    if (at.window) span = std::min<double>(span, at.window + (double)per * fresh / rows);
    return span / kTile + 1;
  };
  const bool cuts = attn_cuts(at);
  const double few_tiles = requests * (double)kv.kv_heads * tiles_of(kRows), many_tiles = requests * (double)kv.kv_heads * tiles_of(kManyRows);
  double few = k.few * few_tiles * (units_of(kRows, false) + kRowsCost) / k.few_shares + 8;
  if (!cuts) few = std::max(few, k.few * units_of(kRows, true));
  const double even = many_tiles * (units_of(kManyRows, false) + kManyCost) / k.many_shares, crowd = std::min(1.0, std::max(0.0, many_tiles / 256 - 1));
  const double whole = std::max((k.one + crowd * (k.full - k.one)) * (units_of(kManyRows, true) + kManyCost), k.full * even);
  const double cut = k.full * even + 12 + k.parts * std::min(1.0, even / kLeastShare);
  AttnGeom g = {};
  g.many = rows > kRows && std::min(whole, cuts ? cut : whole) < few;
  g.shares = cuts && (!g.many || cut < whole);
  g.exact = at.flags & MDBF_ATTN_EXACT_QUERIES;
  g.row_tiles = (int)std::min(tiles_of(g.many ? kManyRows : kRows), 65536.0);
  // Row tiles without shares: each workgroup takes one that its request may have, or the n-th of those that there are, for which
  // it looks through the requests.  That takes 0.5 to 2 us but spreads them evenly where most requests are much shorter than the
  // bound: else a compute unit gets two and three while others, whose workgroups had none, are idle.  Five requests of 1 to 500 new
  // tokens behind 1501 (14 heads on 2 of 64, 1111 visible): 30.7 -> 24.7 us, of 1 to 997: 31.9 -> 32.1.
  const int64_t there = (int64_t)T * (at.q_heads / kv.kv_heads) / kManyRows + all;
  g.distant = units_of(kManyRows, false) >= 64;
  g.nth = g.many && !g.shares && all <= 64 && there * kv.kv_heads <= 512 && there < 0.75 * all * g.row_tiles;
  if (g.nth) g.row_tiles = (int)there;
  return g;
}
static unsigned attn_grid(const AttnGeom& g, int shares, int requests, int kv_heads) {
  return g.shares ? (unsigned)shares : (unsigned)((int64_t)(g.nth ? 1 : requests) * kv_heads * g.row_tiles);
}
// Where two workgroups share a compute unit, a wave of each a SIMD, the one that feeds products goes before the one that is at its
// softmax, if row tiles see much: 32 heads on 8 of 128, 2048 tokens behind 14336 455 -> 435 us (fp16 511 -> 486), 7000 248 -> 239,
// 4000 163 -> 158, 2000 107 -> 106, none 49 -> 52: the instructions' order that it keeps costs something too.  With one
// workgroup on a compute unit it only costs (512 tokens 16.4 -> 17.1; D = 256, 2000 behind 8000, 655 -> 691); with D = 64 nothing
// is gained (32 on 32, 1000 behind 5000, 84.5 -> 84.7).
template <int D>
constexpr bool kCrowds = D == 128;
static bool attn_crowds(const AttnGeom& g, unsigned grid) { return g.many && g.distant && grid >= 512; }
// One size for all calls with these heads and bounds or smaller ones; nothing where no cache is long enough to be cut.
template <int D>
static size_t workspace_of(bool few) {
  const size_t bytes_few = kFewShares<D> * (sizeof(Note) + sizeof(float) * 2 * part_floats<D, kRows>);
  return few ? bytes_few : std::max(bytes_few, kManyShares<D> * (sizeof(Note) + sizeof(float) * 2 * part_floats<D, kManyRows>));
}
static size_t attn_workspace(const mdbf_kv_t& kv, const mdbf_attn_t& at) {
  if (!attn_cuts(at)) return 0;
  const bool few = (int64_t)at.max_fresh * (at.q_heads / kv.kv_heads) <= kRows;
  return kv.head_dim == 64 ? workspace_of<64>(few) : kv.head_dim == 128 ? workspace_of<128>(few) : workspace_of<256>(few);
}

template <int D, int DT, bool EXACT>
static void launch_many(unsigned grid, const AttnArgs& a, const AttnGeom& g, hipStream_t s) {
  if (kCrowds<D> && attn_crowds(g, grid)) attn_many_kernel<D, DT, kCrowds<D>, EXACT><<<grid, 64 * kManyWaves, 0, s>>>(a);
  else attn_many_kernel<D, DT, false, EXACT><<<grid, 64 * kManyWaves, 0, s>>>(a);
}
template <int D, int DT>
static int launch_kernels(AttnArgs& a, const AttnGeom& g, hipStream_t s) {
  a.shares = !g.shares ? 0 : g.many ? kManyShares<D> : kFewShares<D>;
  const unsigned grid = attn_grid(g, a.shares, a.requests, a.kv_heads);
  if (g.many && g.exact) launch_many<D, DT, true>(grid, a, g, s);
  else if (g.many) launch_many<D, DT, false>(grid, a, g, s);
  else if (a.page_shift == 4) attn_few_kernel<D, DT, 4><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (a.page_shift == 5) attn_few_kernel<D, DT, 2><<<grid, 64 * kWaves, 0, s>>>(a);
  else attn_few_kernel<D, DT, 1><<<grid, 64 * kWaves, 0, s>>>(a);
  int e = (int)hipGetLastError();
  if (e == 0 && g.shares) {
    const unsigned rows = (unsigned)(a.shares * a.join_rows);
    if (g.many) attn_join_kernel<D, DT, kManyRows, 1><<<(rows + 3) / 4, 256, 0, s>>>(a);
    else if (a.shares / ((int64_t)a.requests * a.kv_heads * g.row_tiles) >= 16) attn_join_kernel<D, DT, kRows, 4><<<rows, 256, 0, s>>>(a);      // few row tiles, each in many shares
    else attn_join_kernel<D, DT, kRows, 1><<<(rows + 3) / 4, 256, 0, s>>>(a);
    e = (int)hipGetLastError();
  }
  return e;
}
template <int DT>
static int launch_attn(int d, AttnArgs& a, const AttnGeom& g, hipStream_t s) {
  return d == 64 ? launch_kernels<64, DT>(a, g, s) : d == 128 ? launch_kernels<128, DT>(a, g, s) : launch_kernels<256, DT>(a, g, s);
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_kv_attention_workspace_bytes(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T, size_t* bytes_out) {
  if (!bytes_out) return MDBF_EINVAL;
  int st = check_attn(kv, attn, requests, T);
  if (st) return st;
  *bytes_out = attn_workspace(*kv, *attn);
  return MDBF_OK;
}

const char* mdbf_kv_attention_kernel(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T) {
  if (check_attn(kv, attn, requests, T)) return "";
  const AttnGeom g = attn_geom(*kv, *attn, requests, T);
  if (!g.many) return g.shares ? "few rows, shares" : "few rows";
  const AttnCosts k = attn_costs(kv->head_dim);
  const bool crowd = (kv->head_dim == 64 ? kCrowds<64> : kv->head_dim == 128 ? kCrowds<128> : kCrowds<256>) &&
                     attn_crowds(g, attn_grid(g, k.many_shares, requests, kv->kv_heads));
  if (g.shares) return crowd ? "prompts, shares, products first" : "prompts, shares";
  if (g.nth) return crowd ? "prompts, n-th row tiles, products first" : "prompts, n-th row tiles";
  return crowd ? "prompts, products first" : "prompts";
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
  const AttnGeom geom = attn_geom(*kv, *attn, requests, T);
  const size_t need = attn_workspace(*kv, *attn);
  if (need && !workspace_dev) return MDBF_EINVAL;
  if (workspace_bytes < need) return MDBF_EWORKSPACE;
  const int group = attn->q_heads / kv->kv_heads;
  // (rows and requests are counted in steps of up to 8192, by 32 bits)
  if ((int64_t)requests * kv->kv_heads * geom.row_tiles > 0x7fffffff || (int64_t)T * group > 0x70000000 || requests > 0x70000000) return MDBF_EUNSUPPORTED;
  AttnArgs a = {};
  a.cache = (const uint8_t*)cache_dev, a.table = table_dev, a.cu = cu_dev, a.lengths = lengths_dev, a.q = q_dev, a.out = out_dev;
  a.table_ld = table_ld, a.ldq = ldq, a.ldo = ldo, a.table_width = table_width, a.requests = requests, a.T = T, a.pages = kv->pages;
  a.kv_heads = kv->kv_heads, a.group = group, a.head_dim = kv->head_dim;
  a.page_shift = kv_page_shift(kv->page_size), a.causal = attn->flags & MDBF_ATTN_CAUSAL, a.window = attn->window;
  a.row_tiles = geom.row_tiles, a.nth = geom.nth, a.part = (float*)workspace_dev;
  a.join_rows = (int)std::min<int64_t>((int64_t)std::min(attn->max_fresh, T) * a.group, geom.many ? kManyRows : kRows);
  a.scale = (float)(fabs((double)attn->scale) * 1.4426950408889634), a.flip = attn->scale < 0 ? 0x80008000u : 0u;
  int bits = 0;
  while ((1 << bits) < group) ++bits;
  a.group_shift = 31 + bits, a.group_mul = (uint32_t)(((1ull << a.group_shift) + group - 1) / group);
  a.wide_q = ldq % 8 == 0, a.wide_o = ldo % 4 == 0;
  return hip_fail(kv->dtype == MDBF_F16 ? launch_attn<MDBF_F16>(kv->head_dim, a, geom, (hipStream_t)stream)
                                        : launch_attn<MDBF_BF16>(kv->head_dim, a, geom, (hipStream_t)stream));
}

}  // extern "C"
