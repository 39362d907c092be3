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
  float* part;
  int32_t table_width, T, pages, kv_heads, group, head_dim, page_shift, causal, window, row_tiles, splits, chunk, join_rows;
  float scale;                 // of the scores, times log2(e); its sign is the queries' (flip: 0x80008000)
  uint32_t flip;
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
  r.len = (int)min((int64_t)max(a.lengths[b], 0), min((int64_t)a.table_width << a.page_shift, (int64_t)0x7ffffe00));
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

// channels c0 .. c0 + N - 1 of a finished row: its sums over the sum of its numerators; zeros if it sees nothing
template <int DT, int N>
__device__ __forceinline__ void store_row(const AttnArgs& a, const Request& rq, int head, int64_t R, int c0, const float (&o)[N], float sum) {
  const int i = (int)(R / a.group), g = (int)(R % a.group);
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

constexpr int kTile = 32;        // tokens per step of a wave
constexpr int kWaves = 4;
constexpr int kRows = 16;        // query rows of a workgroup
constexpr float kSlack = 8;      // powers of two by which a score may exceed the running reference

// The tokens that the rows of a tile of query rows see, and their part of each workgroup: `chunk` tokens from the first one's
// tile on, the rest of them for the last workgroup.
struct Span {
  int lo, hi;              // what any row sees
  int all_lo, all_hi;      // what all rows see
  int from;                // where the first part begins
  int parts;
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, const Request& rq, int64_t tile, int64_t rows, int splits) {
  const Sees s0 = sees(a, rq, (int)(tile * kRows / a.group)), s1 = sees(a, rq, (int)(min(tile * kRows + kRows - 1, rows - 1) / a.group));
  Span s = {s0.lo, s1.hi, s1.lo, s0.hi, s0.lo & ~(kTile - 1), 1};
  if (splits > 1 && s.hi > s.from) s.parts = (int)min((int64_t)splits, ((int64_t)s.hi - s.from + a.chunk - 1) / a.chunk);
  return s;
}

// where the results of one part of a tile of rows go: kRows x D sums, then kRows maxima and kRows sums of numerators
template <int D>
__device__ __forceinline__ int64_t part_floats() { return kRows * (D + 2); }

constexpr int kNonTemporal = 2;  // of the buffer loads: the cache is read once

// One wave's tile of tokens: codes and scales of its keys and values as loaded.  It lies in one page (ONE), or its halves of 16
// tokens lie in one each (pages of 16 tokens).
template <int D, bool ONE>
struct Codes {
  static constexpr int KW = D / 32;                  // dwords of codes per lane and 16 keys = matrix steps over the channels
  static constexpr int KS = D <= 128 ? 1 : D / 128;  // scales among them
  static constexpr int VU = D / 64;                  // 16-byte units of values per lane
  static constexpr int VH = D == 64 ? 1 : VU / 2;    // of them in each half
  uint32_t kc[2][KW], ks[2][KS];
  U32x4 vc[VU];
  uint32_t vs[VU];
  // the half of a unit, and its place there: 16 tokens x D / 32 blocks
  __device__ static __forceinline__ int half(int n, int lane) { return D == 64 ? lane >> 5 : n / VH; }
  __device__ static __forceinline__ int unit(int n, int lane) { return D == 64 ? lane & 31 : (n % VH) * 64 + lane; }

  bool there[2];             // whether the halves' pages are pages of the pool

  // `page`: of the two halves' tokens, which begin at tok.  Nothing here looks at what the loads bring: they are in flight while
  // the tile before is worked on.  (Buffer loads: a page's part for the head is the buffer, a lane's place in a tile the offset.)
  __device__ __forceinline__ void load(const AttnArgs& a, int head, int64_t head_bytes, int tok, const int (&page)[2], int lane) {
    const int P = 1 << a.page_shift, r = lane & 15, h = lane >> 4;
    const uint8_t* base[2];
    __amdgpu_buffer_rsrc_t buf[2];
    int off[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      if (ONE && f) {
        there[1] = there[0], buf[1] = buf[0], off[1] = off[0] + 16;
        continue;
      }
      there[f] = (uint32_t)page[f] < (uint32_t)a.pages;
      base[f] = a.cache + ((int64_t)(there[f] ? page[f] : 0) * a.kv_heads + head) * head_bytes;
      buf[f] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base[f]), 0, (int)head_bytes, 0x00027000);
      off[f] = (tok + 16 * f) & (P - 1);
    }
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int at = r * (D / 2) + h * (D / 8);
      if (KW == 2) {
        const U32x2 v = __builtin_amdgcn_raw_buffer_load_b64(buf[f], at, off[f] * (D / 2), kNonTemporal);
        kc[f][0] = v[0], kc[f][1] = v[1];
      } else {
#pragma unroll
        for (int s = 0; s < KW; s += 4) {
          const U32x4 v = __builtin_amdgcn_raw_buffer_load_b128(buf[f], at + 4 * s, off[f] * (D / 2), kNonTemporal);
#pragma unroll
          for (int w = 0; w < 4; ++w) kc[f][(s + w) % KW] = v[w];
        }
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
        ks[f][s] = __builtin_amdgcn_raw_buffer_load_b8(buf[f], r * (D / 32) + (D == 64 ? h >> 1 : h * KS + s), P * D + off[f] * (D / 32), 0);
    }
#pragma unroll
    for (int n = 0; n < VU; ++n) {
      if (!ONE && D == 64) {      // the halves of one load in different pages
        const MDBF_GLOBAL uint8_t* at = (const MDBF_GLOBAL uint8_t*)(lane < 32 ? base[0] : base[1]);
        const uint32_t o = lane < 32 ? off[0] : off[1], u = lane & 31;
        vc[n] = __builtin_nontemporal_load((const MDBF_GLOBAL U32x4*)(at + (P + o) * (D / 2) + u * 16));
        vs[n] = at[P * (D + D / 32) + o * (D / 32) + u];
      } else {
        const int f = ONE ? 0 : n / VH, u = (ONE ? n : n % VH) * 64 + lane;
        vc[n] = __builtin_amdgcn_raw_buffer_load_b128(buf[f], u * 16, (P + off[f]) * (D / 2), kNonTemporal);
        vs[n] = __builtin_amdgcn_raw_buffer_load_b8(buf[f], u, P * (D + D / 32) + off[f] * (D / 32), 0);
      }
    }
  }
  // a page that is none reads as NaN
  __device__ __forceinline__ void check(int lane) {
    if (there[0] && there[1]) return;
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int s = 0; s < KS; ++s)
        if (!there[f]) ks[f][s] = kKvNanScale;
#pragma unroll
    for (int n = 0; n < VU; ++n)
      if (!(half(n, lane) ? there[1] : there[0])) vs[n] = kKvNanScale;
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

// One kv head, 16 query rows, one part of their tokens; the part's tiles are dealt out to the four waves, which meet at
// the end.  A tile's loads are issued before the products of the one before it, and its page numbers a tile earlier still.
template <int D, int DT, bool ONE>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 4 : D == 128 ? 3 : 2) void attn_few_kernel(AttnArgs a) {
  using Tile = Codes<D, ONE>;
  constexpr int KW = Tile::KW, KS = Tile::KS, VU = Tile::VU;
  // A token's values in LDS: 64 bytes per block, 16 more after each (D = 64) or every second one, rows an odd multiple of 32
  // bytes apart: neither the writes nor the transposing reads meet on a bank.
  constexpr int VROW = D == 64 ? 160 : D == 128 ? 288 : 608;
  auto block_at = [](int g) { return g * 64 + (D == 64 ? g : g >> 1) * 16; };
  constexpr int CT = D / 16;                  // channel tiles
  constexpr int OROW = D + 4;                 // floats of a row of results in LDS
  static_assert(kTile * VROW >= kRows * OROW * 4, "the results fit the values' place");
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves][kTile * VROW];
  __shared__ float stat[kWaves][2][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
  uint32_t idx = blockIdx.x;
  const int part = idx % a.splits;
  idx /= a.splits;
  const int rt0 = idx % a.row_tiles;
  idx /= a.row_tiles;
  const int head = idx % a.kv_heads, b = idx / a.kv_heads;
  const Request rq = request_of(a, b);
  const int64_t rows = (int64_t)rq.fresh * a.group;
  const int64_t head_bytes = kv_head_bytes(1 << a.page_shift, D);
  const MDBF_CONST int32_t* table = (const MDBF_CONST int32_t*)a.table + b * a.table_ld;
  unsigned char* vals = lds[wave];

  // (tiles of rows beyond those that the launch was sized for are not split)
  for (int64_t rt = rt0; rt * kRows < rows; rt += a.row_tiles) {
    const Span sp = span_of(a, rq, rt, rows, rt == rt0 ? a.splits : 1);
    if (part >= sp.parts) continue;
    const int64_t R = rt * kRows + r;
    const bool valid = R < rows;
    const int i = valid ? (int)(R / a.group) : 0, g = valid ? (int)(R % a.group) : 0;
    Sees me = sees(a, rq, i);
    if (!valid) me.hi = me.lo = 0;
    const int64_t first = sp.from + (int64_t)part * a.chunk;
    const int tmin = max(sp.lo, (int)first), tmax = part == sp.parts - 1 ? sp.hi : (int)(first + a.chunk);

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

    // page numbers of a tile's halves; behind the last token's none is looked up
    auto pages_of = [&](int t, int (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < (ONE ? 1 : 2); ++f) page[f] = table[min(t + 16 * f, rq.len - 1) >> a.page_shift];
    };
    auto work = [&](Tile& x, int t0) __attribute__((always_inline)) {
      x.check(lane);
      // scores (without their factor): a lane holds those of its row with tokens 4 h + 0 .. 3 of each half
      F32x4 z[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        z[f] = F32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KW; ++s) z[f] = mma16<DT>(numbers<DT>(x.kc[f][s], unit_of(x.ks[f][KS == 1 ? 0 : s / 4])), qf[s], z[f]);
      }
      const bool inside = t0 >= sp.all_lo && t0 + kTile <= sp.all_hi;     // every row sees every token
      if (!inside) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int tok = t0 + 16 * f + 4 * h + j;
            if (tok < me.lo || tok >= me.hi) z[f][j] = -INFINITY;
          }
      }
      // The reference m follows the maximum only where that has grown by more than kSlack (numerators stay below 2^kSlack, in
      // reach of fp16): most tiles exchange nothing between lanes and rescale nothing.
      const float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3]))) * a.scale;
      if (__any(top > m + kSlack)) {
        const float mn = fmaxf(m, row_max(top)), alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
        m = mn;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c] *= alpha;
      }
      const float use = m == -INFINITY ? 0.0f : m;
      F32x4 p[2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) p[f][j] = __builtin_amdgcn_exp2f(z[f][j] * a.scale - use);
      l += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
      const U32x4 pf = {round2<DT>(p[0][0], p[0][1]), round2<DT>(p[0][2], p[0][3]), round2<DT>(p[1][0], p[1][1]), round2<DT>(p[1][2], p[1][3])};

      // values that no row sees are zeros; NaN among the others goes to the rows that see it, not through the product, where a
      // zero weight would bring it to all rows
#pragma unroll
      for (int n = 0; n < VU; ++n) {
        const int unit = Tile::unit(n, lane), row = 16 * Tile::half(n, lane) + unit / (D / 32), tok = t0 + row;
        if (!inside && (tok < sp.lo || tok >= sp.hi)) {
          x.vc[n] = U32x4{0, 0, 0, 0};
          x.vs[n] = 127;
        }
        uint64_t bad = __ballot(x.vs[n] == kKvNanScale);
        if (bad) {
          if (x.vs[n] == kKvNanScale) {
            x.vc[n] = U32x4{0, 0, 0, 0};
            x.vs[n] = 127;
          }
          for (; bad; bad &= bad - 1) {
            const int from = __builtin_ctzll(bad), bu = Tile::unit(n, from);
            const int bt = t0 + 16 * Tile::half(n, from) + bu / (D / 32), bg = bu % (D / 32);
            if (bt >= me.lo && bt < me.hi) nan_blocks |= 1u << bg;
          }
        }
        const float unit_f = unit_of(x.vs[n]);
        unsigned char* to = vals + row * VROW + block_at(unit % (D / 32));
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<U32x4*>(to + w * 16) = numbers<DT>(x.vc[n][w], unit_f);
      }
      wave_lds_order();
      // a lane's channel of tokens 4 h + 0 .. 3 of each half: the order of the scores' registers
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const unsigned char* from = vals + (4 * h + (r >> 2)) * VROW + block_at(c / 2) + (c & 1) * 32 + (r & 3) * 8;
        const U32x2 v0 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)from));
        const U32x2 v1 = __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MDBF_LDS S16x4*)(from + 16 * VROW)));
        acc[c] = mma16<DT>(U32x4{v0[0], v0[1], v1[0], v1[1]}, pf, acc[c]);
      }
      wave_lds_order();
    };

    constexpr int kStep = kWaves * kTile;
    int t0 = (tmin & ~(kTile - 1)) + wave * kTile;
    if (t0 < tmax) {
      Tile x, y;
      int page[2];
      pages_of(t0, page);
      x.load(a, head, head_bytes, t0, page, lane);
      pages_of(t0 + kStep, page);
      for (;;) {
        if (t0 + kStep < tmax) y.load(a, head, head_bytes, t0 + kStep, page, lane);
        pages_of(t0 + 2 * kStep, page);
        work(x, t0);
        t0 += kStep;
        if (t0 >= tmax) break;
        if (t0 + kStep < tmax) x.load(a, head, head_bytes, t0 + kStep, page, lane);
        pages_of(t0 + 2 * kStep, page);
        work(y, t0);
        t0 += kStep;
        if (t0 >= tmax) break;
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
      const int64_t Ro = rt * kRows + row;
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
        if (sp.parts > 1) {
          MDBF_GLOBAL float* to = (MDBF_GLOBAL float*)a.part + (int64_t)blockIdx.x * part_floats<D>();
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
    __syncthreads();
  }
}

// Joins the parts of a query row: a workgroup per row that the launch was sized for and CH of its channels, CH / 4 lanes side by
// side on them; the groups of lanes take the parts in turn and meet in LDS, in one order.  A chain of two trips to memory at
// most: the first parts' sums are requested before the weights are known.
constexpr int kMostSplits = 1024;
template <int D, int DT, int CH>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int L = CH / 4, GROUPS = 256 / L, AHEAD = 8;
  uint32_t idx = blockIdx.x;
  const int c0 = idx % (D / CH) * CH;
  idx /= D / CH;
  const int row0 = idx % a.join_rows;
  idx /= a.join_rows;
  const uint32_t tile = idx;               // of the launch before
  const int rt = idx % a.row_tiles;
  idx /= a.row_tiles;
  const int head = idx % a.kv_heads, b = idx / a.kv_heads;
  const Request rq = request_of(a, b);
  const int64_t rows = (int64_t)rq.fresh * a.group;
  if ((int64_t)rt * kRows + row0 >= rows) return;
  const Span sp = span_of(a, rq, rt, rows, a.splits);
  if (sp.parts <= 1) return;
  const MDBF_GLOBAL float* from = (const MDBF_GLOBAL float*)a.part + (int64_t)tile * a.splits * part_floats<D>();
  __shared__ float weight[kMostSplits], stat[4], total[4];
  __shared__ F32x4 sums[GROUPS][L];
  const int tid = threadIdx.x, l = tid % L, grp = tid / L;

  for (int row = row0; row < kRows && (int64_t)rt * kRows + row < rows; row += a.join_rows) {
    const MDBF_GLOBAL float* mine = from + row * D + c0 + l * 4;
    F32x4 ahead[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (grp + k * GROUPS < sp.parts) ahead[k] = *(const MDBF_GLOBAL F32x4*)(mine + (grp + k * GROUPS) * part_floats<D>());
    float top = -INFINITY, tops[kMostSplits / 256], parts_sum[kMostSplits / 256];
#pragma unroll
    for (int k = 0; k < kMostSplits / 256; ++k) {
      const int p = tid + k * 256;
      tops[k] = -INFINITY, parts_sum[k] = 0;
      if (p < sp.parts) {
        tops[k] = from[p * part_floats<D>() + kRows * D + row];
        parts_sum[k] = from[p * part_floats<D>() + kRows * (D + 1) + row];
        top = fmaxf(top, tops[k]);
      }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if ((tid & 63) == 0) stat[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(stat[0], stat[1]), fmaxf(stat[2], stat[3]));
    const float use = top == -INFINITY ? 0.0f : top;
    float sum = 0;
#pragma unroll
    for (int k = 0; k < kMostSplits / 256; ++k)
      if (tid + k * 256 < sp.parts) {
        const float f = __builtin_amdgcn_exp2f(tops[k] - use);
        weight[tid + k * 256] = f;
        sum += f * parts_sum[k];
      }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63) == 0) total[tid >> 6] = sum;
    __syncthreads();
    sum = (total[0] + total[1]) + (total[2] + total[3]);
    F32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (grp + k * GROUPS < sp.parts) o += weight[grp + k * GROUPS] * ahead[k];
    for (int p = grp + AHEAD * GROUPS; p < sp.parts; p += GROUPS) o += weight[p] * *(const MDBF_GLOBAL F32x4*)(mine + p * part_floats<D>());
    sums[grp][l] = o;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int w = 1; w < GROUPS; ++w) o += sums[w][l];
      const float v[4] = {o[0], o[1], o[2], o[3]};
      store_row<DT, 4>(a, rq, head, (int64_t)rt * kRows + row, c0 + l * 4, v, sum);
    }
    __syncthreads();
  }
}

static int check_attn(const mdbf_kv_t* kv, const mdbf_attn_t* at, int requests, int T) {
  int st = check_kv(kv);
  if (st) return st;
  if (!at || requests < 1 || T < 1) return MDBF_EINVAL;
  if (at->q_heads <= 0 || at->q_heads % kv->kv_heads || at->window < 0 || at->max_fresh < 1 || at->max_length < 1 || !isfinite(at->scale) || at->scale == 0.0f)
    return MDBF_EINVAL;
  if (at->window && !(at->flags & MDBF_ATTN_CAUSAL)) return MDBF_EINVAL;
  if ((at->flags & ~MDBF_ATTN_CAUSAL) || at->q_heads > (1 << 16)) return MDBF_EUNSUPPORTED;
  return MDBF_OK;
}

// How a call is cut up: tiles of query rows per request and kv head, and parts of the tokens of each.
struct AttnGeom {
  int64_t tiles;           // over all requests and kv heads
  int row_tiles, splits, chunk;
  size_t part_bytes;
};
// A part is one workgroup's: enough of them to fill the device several times over, so that requests of unequal length even
// out, but none shorter than kLeastChunk tokens, two steps of its waves.
constexpr int kLeastChunk = 256, kPartsWanted = 2048;
static AttnGeom attn_geom(const mdbf_kv_t& kv, const mdbf_attn_t& at, int requests, int T) {
  AttnGeom g;
  const int64_t group = at.q_heads / kv.kv_heads, most = std::min(at.max_fresh, T);
  g.row_tiles = (int)std::min<int64_t>((most * group + kRows - 1) / kRows, 1 << 16);
  g.tiles = (int64_t)requests * kv.kv_heads * g.row_tiles;
  int64_t span = at.max_length;
  if (at.window) span = std::min<int64_t>(span, (int64_t)at.window + kRows + kTile);
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({kPartsWanted / g.tiles, span / kLeastChunk, kMostSplits}));
  const int64_t step = kWaves * kTile;
  g.chunk = (int)(((span + splits - 1) / splits + step - 1) / step * step);
  g.splits = (int)((span + g.chunk - 1) / g.chunk);
  g.part_bytes = g.splits > 1 ? (size_t)g.tiles * g.splits * kRows * (kv.head_dim + 2) * 4 : 0;
  return g;
}

template <int D, int DT>
static int launch_few(const AttnArgs& a, const AttnGeom& g, hipStream_t s) {
  if (a.page_shift == 4) attn_few_kernel<D, DT, false><<<(unsigned)(g.tiles * g.splits), 64 * kWaves, 0, s>>>(a);
  else attn_few_kernel<D, DT, true><<<(unsigned)(g.tiles * g.splits), 64 * kWaves, 0, s>>>(a);
  int e = (int)hipGetLastError();
  if (e == 0 && g.splits > 1) {
    // few parts: all channels in one workgroup
    if (g.splits > 16) attn_join_kernel<D, DT, 32><<<(unsigned)(g.tiles * a.join_rows * (D / 32)), 256, 0, s>>>(a);
    else attn_join_kernel<D, DT, D><<<(unsigned)(g.tiles * a.join_rows), 256, 0, s>>>(a);
    e = (int)hipGetLastError();
  }
  return e;
}
template <int DT>
static int launch_attn(int d, const AttnArgs& a, const AttnGeom& g, hipStream_t s) {
  return d == 64 ? launch_few<64, DT>(a, g, s) : d == 128 ? launch_few<128, DT>(a, g, s) : launch_few<256, DT>(a, g, s);
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int mdbf_kv_attention_workspace_bytes(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T, size_t* bytes_out) {
  if (!bytes_out) return MDBF_EINVAL;
  int st = check_attn(kv, attn, requests, T);
  if (st) return st;
  *bytes_out = attn_geom(*kv, *attn, requests, T).part_bytes;
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
  const AttnGeom geom = attn_geom(*kv, *attn, requests, T);
  if (geom.part_bytes && !workspace_dev) return MDBF_EINVAL;
  if (workspace_bytes < geom.part_bytes) return MDBF_EWORKSPACE;
  if (geom.tiles * std::max(geom.splits, kRows * 8) > 0x7fffffff) return MDBF_EUNSUPPORTED;
  AttnArgs a = {};
  a.cache = (const uint8_t*)cache_dev, a.table = table_dev, a.cu = cu_dev, a.lengths = lengths_dev, a.q = q_dev, a.out = out_dev;
  a.table_ld = table_ld, a.ldq = ldq, a.ldo = ldo, a.table_width = table_width, a.T = T, a.pages = kv->pages;
  a.kv_heads = kv->kv_heads, a.group = attn->q_heads / kv->kv_heads, a.head_dim = kv->head_dim;
  a.page_shift = kv_page_shift(kv->page_size), a.causal = attn->flags & MDBF_ATTN_CAUSAL, a.window = attn->window;
  a.row_tiles = geom.row_tiles, a.splits = geom.splits, a.chunk = geom.chunk, a.part = (float*)workspace_dev;
  a.join_rows = (int)std::min<int64_t>((int64_t)std::min(attn->max_fresh, T) * a.group, kRows);
  a.scale = (float)(fabs((double)attn->scale) * 1.4426950408889634), a.flip = attn->scale < 0 ? 0x80008000u : 0u;
  a.wide_q = ldq % 8 == 0, a.wide_o = ldo % 4 == 0;
  return hip_fail(kv->dtype == MDBF_F16 ? launch_attn<MDBF_F16>(kv->head_dim, a, geom, (hipStream_t)stream)
                                        : launch_attn<MDBF_BF16>(kv->head_dim, a, geom, (hipStream_t)stream));
}

}  // extern "C"
