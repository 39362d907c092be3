// Low-rank adapters of many requests beside a shared projection: the order of a step's rows, and Y += scale B (A X).
#include "mdbf_rows.h"

namespace mdbf {

// ---- rows by adapter ------------------------------------------------------------------------------------
// A counting sort by one workgroup: tokens of each adapter (integer sums in LDS), a scan over the adapters for their first places and
// tiles, then the requests in their order, 1024 at a time, each behind those of the same adapter in front of it: in its wave by a look at each
// of the 64, then wave after wave.  The key `adapters` stands for none and comes last.  All latency: 5.5 us for 64 requests with a row each
// (of which a launch is some 4); 500 prompts of 250740 rows take 8.1, most of it 4017 tiles, and 4.1 for the rows in a second launch.
constexpr int kRowThreads = 1024;
constexpr int kRowMaxAdapters = 8192;     // three words each in LDS
constexpr int kRowOneLaunch = 8192;       // rows, of up to kRowThreads requests, up to which the first launch writes them
constexpr int kRowChunk = 1024;           // rows per workgroup of the second launch

struct RowArgs {
  const int32_t *cu, *adapter;
  int32_t *rows, *tiles, *places;
  int64_t tile_room;
  int32_t T, requests, adapters, rows_here;
};

__device__ __forceinline__ int cut(int v, int most) { return min(max(v, 0), most); }

// The place of a row that is no request's (lo: the last request that begins at it or before, -1: none).  The requests' rows, from `first` to `end`, take the
// places from 0 on: rows in front of them come right behind those, and rows behind them keep theirs, so that each place has one row.
__device__ __forceinline__ uint32_t place_of_no_request(int t, int lo, int first, int end) { return lo < 0 ? (uint32_t)end - (uint32_t)first + (uint32_t)t : (uint32_t)t; }

// inclusive sums over the workgroup's threads
__device__ __forceinline__ void row_scan(uint32_t& a, uint32_t& b, uint32_t (*waves)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t ua = __shfl_up(a, o), ub = __shfl_up(b, o);
    if (lane >= o) a += ua, b += ub;
  }
  if (lane == 63) waves[wave][0] = a, waves[wave][1] = b;
  __syncthreads();
  for (int w = 0; w < wave; ++w) a += waves[w][0], b += waves[w][1];
}

__global__ __launch_bounds__(kRowThreads) void adapter_rows_kernel(RowArgs a) {
  extern __shared__ uint32_t words[];
  uint32_t *count = words, *place = count + a.adapters + 1, *tile = place + a.adapters + 1;
  __shared__ uint32_t waves[kRowThreads / 64][2];
  __shared__ int32_t keys[kRowThreads], fresh[kRowThreads], first_row[kRowThreads + 1], first_place[kRowThreads];
  const int tid = threadIdx.x, N = a.adapters;

  // a request's first row, rows and key
  const auto request = [&](int i, int& from, int& f, int& k) {
    const int asked = a.adapter[i];
    from = cut(a.cu[i], a.T);
    f = max(cut(a.cu[i + 1], a.T) - from, 0);
    k = asked >= 0 && asked < N ? asked : N;
  };
  int from = 0, f = 0, k = N;
  if (tid < a.requests) request(tid, from, f, k);
  for (int k = tid; k <= N; k += kRowThreads) count[k] = 0;
  __syncthreads();
  if (f > 0) atomicAdd(&count[k], (uint32_t)f);
  for (int i = tid + kRowThreads; i < a.requests; i += kRowThreads) {
    int from_i, f_i, k_i;
    request(i, from_i, f_i, k_i);
    if (f_i > 0) atomicAdd(&count[k_i], (uint32_t)f_i);
  }
  __syncthreads();

  // first places and tiles: each thread sums a run of adapters
  const int run = (N + 1 + kRowThreads - 1) / kRowThreads, k0 = min(tid * run, N + 1), k1 = min(k0 + run, N + 1);
  uint32_t rows = 0, tiles = 0;
  for (int k = k0; k < k1; ++k) {
    rows += count[k];
    if (k < N) tiles += (count[k] + MDBF_ADAPTER_TILE - 1) / MDBF_ADAPTER_TILE;
  }
  uint32_t rows_to = rows, tiles_to = tiles;
  row_scan(rows_to, tiles_to, waves);
  rows = rows_to - rows, tiles = tiles_to - tiles;
  for (int k = k0; k < k1; ++k) {
    place[k] = rows, tile[k] = tiles;
    rows += count[k];
    if (k < N) tiles += (count[k] + MDBF_ADAPTER_TILE - 1) / MDBF_ADAPTER_TILE;
  }
  __syncthreads();
  const uint32_t all_tiles = tile[N];
  for (int64_t t = tid; t < a.tile_room; t += kRowThreads) {
    int32_t out[4] = {-1, 0, 0, 0};
    if (t < all_tiles) {
      int lo = 0, hi = N;                  // the last adapter whose first tile is not behind t: the one that has it
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile[mid] <= (uint32_t)t) lo = mid;
        else hi = mid;
      }
      const uint32_t done = ((uint32_t)t - tile[lo]) * MDBF_ADAPTER_TILE;
      out[0] = lo, out[1] = (int)(place[lo] + done), out[2] = (int)min(count[lo] - done, (uint32_t)MDBF_ADAPTER_TILE);
    }
    *((MDBF_GLOBAL U32x4*)a.tiles + t) = U32x4{(uint32_t)out[0], (uint32_t)out[1], (uint32_t)out[2], 0u};
  }

  for (int i0 = 0; i0 < a.requests; i0 += kRowThreads) {
    const int i = i0 + tid, n = min(a.requests - i0, kRowThreads);
    if (i0) {                              // (the first ones' are in registers)
      from = f = 0, k = N;
      if (tid < n) request(i, from, f, k);
    }
    keys[tid] = k, fresh[tid] = f, first_row[tid] = from;
    uint32_t mine = 0;
    if ((tid & ~63) < n) {
#pragma unroll
      for (int j = 0; j < 63; ++j) {
        const int kj = __builtin_amdgcn_readlane(k, j), fj = __builtin_amdgcn_readlane(f, j);
        if (k == kj && (tid & 63) > j) mine += (uint32_t)fj;
      }
    }
    __syncthreads();                       // (the tiles are out of `place`)
    for (int w = 0; w * 64 < n; ++w) {
      if (tid >> 6 == w && tid < n) {
        mine += place[k];
        a.places[i] = (int)mine;
        first_place[tid] = (int)mine;
      }
      __syncthreads();
      if (tid >> 6 == w && tid < n && f) atomicAdd(&place[k], (uint32_t)f);
      __syncthreads();
    }
  }
  if (!a.rows_here) return;
  // (up to kRowThreads requests, all of them in LDS)
  __syncthreads();
  for (int t = tid; t < a.T; t += kRowThreads) {
    int lo = -1, hi = a.requests;          // the last request that begins at t or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first_row[mid] <= t) lo = mid;
      else hi = mid;
    }
    const bool in = lo >= 0 && t - first_row[lo] < fresh[lo];
    const uint32_t at = in ? (uint32_t)first_place[lo] + (uint32_t)(t - first_row[lo])
                           : place_of_no_request(t, lo, first_row[0], first_row[a.requests - 1] + fresh[a.requests - 1]);
    if (at < (uint32_t)a.T) a.rows[at] = in && keys[lo] < N ? t : -1;
  }
}

// The rows of long steps, by bisection of cu.
__global__ __launch_bounds__(kRowChunk) void adapter_places_kernel(RowArgs a) {
  const int t = blockIdx.x * kRowChunk + threadIdx.x;
  if (t >= a.T) return;
  int lo = -1, hi = a.requests;
  while (hi - lo > 1) {
    const int mid = (int)(((int64_t)lo + hi) >> 1);
    if (cut(a.cu[mid], a.T) <= t) lo = mid;
    else hi = mid;
  }
  const int from = lo < 0 ? 0 : cut(a.cu[lo], a.T);
  const bool in = lo >= 0 && t < cut(a.cu[lo + 1], a.T);
  const int k = in ? a.adapter[lo] : -1;
  const uint32_t at = in ? (uint32_t)a.places[lo] + (uint32_t)(t - from)
                         : place_of_no_request(t, lo, cut(a.cu[0], a.T), cut(a.cu[a.requests], a.T));
  if (at < (uint32_t)a.T) a.rows[at] = k >= 0 && k < a.adapters ? t : -1;
}

// ---- products -------------------------------------------------------------------------------------------
// Two launches: V = A X by tiles of rows, ranks and parts of the channels, then Y += scale B V by tiles of rows and columns of
// Y.  Both on 16x16x32 products.  What has to be moved is X, the adapters in use and Y, twice: a tile of rows shares its adapter, and what
// a projection shares with the next one, X, is read once for up to four tiles of ranks.  Measured, us of the two launches: q, k and v of 4096 for
// 64 requests on 28 adapters of rank 16 (24 MB) 6.6 + 9.1, latency; two projections of 11008 for 256 requests on 4 adapters of rank 64 (37 MB) 9.4 + 19,
// where the second launch adds up the first one's eight splits in every workgroup; q, k and v of 6458 rows of prompts (332 MB) 14.5 + 59, HBM.
constexpr int kInSlots = 4;                    // tiles of 16 ranks per workgroup of the first launch
constexpr int kMaxRank = 256;
constexpr int kMaxWidth = 1 << 23;             // channels and columns: the second launch's grid ends at 65535 times 256 columns
constexpr int64_t kMaxTiles = (1 << 24) - 1;    // a launch has less than 2^32 threads: beyond, their number wraps without an error
constexpr int kMaxGroups = MDBF_ADAPTER_MAX * kMaxRank / 16 / kInSlots;
constexpr int kOutBlock = 64;                  // columns of Y that a wave takes at a time

typedef float Acc4 __attribute__((ext_vector_type(4)));
typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 F16x8 __attribute__((ext_vector_type(8)));

template <int DT>
__device__ __forceinline__ Acc4 product(const U32x4& a, const U32x4& b, const Acc4& c) {
  if (DT == MDBF_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b), c, 0, 0, 0);
}

// workgroups of the first launch that share X: tiles of 16 ranks, of one projection or of several
struct InGroup {
  const void* X;
  int64_t ldx;
  int32_t n, slots;
  uint8_t proj[kInSlots], tile[kInSlots];
};
struct InArgs {
  InGroup g[kMaxGroups];
  const void* A[MDBF_ADAPTER_MAX];
  int32_t r[MDBF_ADAPTER_MAX], column[MDBF_ADAPTER_MAX];   // rank, and the projection's first column of V
  const int32_t *rows, *tiles;
  float* V;                                    // splits x T x width, by place
  int32_t adapters, T, width, splits;
};
struct OutProj {
  const void* B;
  void* Y;
  const float* scale;
  int64_t ldy;
  int32_t m, r, column, yd, chunk;             // chunk: columns of Y per workgroup
};
struct OutArgs {
  OutProj p[MDBF_ADAPTER_MAX];
  const int32_t *rows, *tiles;
  const float* V;
  int32_t adapters, T, width, splits;
};

// the tile's adapter, first place and rows; false for one that is none
__device__ __forceinline__ bool tile_of(const int32_t* tiles, int64_t t, int adapters, int T, int& adapter, int& first, int& count) {
  const U32x4 w = *((const MDBF_GLOBAL U32x4*)tiles + t);
  adapter = (int)w[0], first = (int)w[1], count = min((int)w[2], MDBF_ADAPTER_TILE);
  if (adapter < 0 || adapter >= adapters || first < 0 || first >= T || count <= 0) return false;
  count = min(count, T - first);
  return true;
}

// V[split][place][rank] = sum over the split's channels of A[rank][c] X[row][c], 128 channels at a time.  A product's operand has a row per lane, and
// sixteen rows are sixteen cache lines: so rows are loaded side by side, 256 bytes of each, and go through LDS (two buffers; the
// sixteen pieces of a row lie exclusive-or its number, so that neither writes nor reads of sixteen lanes meet on a bank).  A wave has 16 rows
// of X; where a tile has fewer than 64 the other waves take some of the four products along the channels, and their sums meet in
// LDS.  6458 rows of 4096 channels, three projections of rank 16 (55 MB): 13.8 us, 32 with operands loaded as the products want them.
constexpr int kInChannels = 128;
template <int DT, int NS>
__device__ __forceinline__ void in_tile(const InArgs& a, const InGroup& g, int adapter, int first, int count, int split, U32x4 (*lds)[(4 + kInSlots) * 256]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, kg = lane >> 4;
  const int subs = count <= 16 ? 1 : count <= 32 ? 2 : 4, sub = wave & (subs - 1), piece = wave / subs, pieces = 4 / subs;
  const int stages = (g.n + kInChannels - 1) / kInChannels;
  const int s0 = (int)((int64_t)stages * split / a.splits), s1 = (int)((int64_t)stages * (split + 1) / a.splits);

  // loading: a sixteenth of the threads per row, rows 16 apart
  const int lr = tid >> 4, lc = tid & 15, slot = lr * 16 + (lc ^ lr);
  int64_t x0[4], a0[NS];
  const void* A[NS];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q < subs ? cut(a.rows[first + min(q * 16 + lr, count - 1)], a.T - 1) : 0;    // (a row that is none is left out at the end)
    x0[q] = (int64_t)row * g.ldx + lc * 8;
  }
#pragma unroll
  for (int q = 0; q < NS; ++q) {
    const int p = g.proj[q], r = a.r[p];
    A[q] = a.A[p];
    a0[q] = ((int64_t)adapter * r + min(g.tile[q] * 16 + lr, r - 1)) * g.n + lc * 8;
  }
  Raw8<DT> rx[4], ra[NS];
  const auto load = [&](int s) {
    const int c = s * kInChannels, there = g.n - c - lc * 8;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < subs) load_raw8<DT>(g.X, x0[q] + c, there, rx[q]);
#pragma unroll
    for (int q = 0; q < NS; ++q) load_raw8<DT>(A[q], a0[q] + c, there, ra[q]);
  };
  const auto store = [&](int b) {
#pragma unroll
    for (int q = 0; q < NS; ++q) lds[b][q * 256 + slot] = ra[q].w[0];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < subs) lds[b][(NS + q) * 256 + slot] = rx[q].w[0];
  };
  Acc4 acc[NS] = {};
  const auto products = [&](int b, int u) {
    const int at = i * 16 + ((u * 4 + kg) ^ i);
    const U32x4 x = lds[b][(NS + sub) * 256 + at];
#pragma unroll
    for (int q = 0; q < NS; ++q) acc[q] = product<DT>(x, lds[b][q * 256 + at], acc[q]);
  };
  if (s0 < s1) load(s0), store(0);
  if (s0 + 1 < s1) load(s0 + 1);
  __syncthreads();
  for (int s = s0; s < s1; ++s) {
    const int b = (s - s0) & 1;
    if (subs == 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) products(b, u);
    } else if (subs == 2) {
      products(b, piece * 2);
      products(b, piece * 2 + 1);
    } else {
      products(b, piece);
    }
    if (s + 1 < s1) store(b ^ 1);
    if (s + 2 < s1) load(s + 2);
    __syncthreads();
  }
  if (pieces > 1) {
    Acc4* part = (Acc4*)lds;
    if (piece) {
#pragma unroll
      for (int q = 0; q < NS; ++q) part[((wave - subs) * NS + q) * 64 + lane] = acc[q];
    }
    __syncthreads();
    if (piece) return;
    for (int w = sub; w < 4 - subs; w += subs)
#pragma unroll
      for (int q = 0; q < NS; ++q) acc[q] += part[(w * NS + q) * 64 + lane];
  }
  // lane: rank i of the tile, rows 4 kg ..
#pragma unroll
  for (int q = 0; q < NS; ++q) {
    const int p = g.proj[q], rank = g.tile[q] * 16 + i;
    float* v = a.V + ((int64_t)split * a.T + first + sub * 16 + kg * 4) * a.width + a.column[p] + rank;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (sub * 16 + kg * 4 + e < count) v[(int64_t)e * a.width] = rank < a.r[p] ? acc[q][e] : 0.0f;
  }
}

template <int DT>
__global__ __launch_bounds__(256) void adapter_in_kernel(InArgs a) {
  __shared__ U32x4 lds[2][(4 + kInSlots) * 256];
  int adapter, first, count;
  if (!tile_of(a.tiles, blockIdx.x, a.adapters, a.T, adapter, first, count)) return;
  const InGroup& g = a.g[blockIdx.z];
  if (g.slots == 1) in_tile<DT, 1>(a, g, adapter, first, count, blockIdx.y, lds);
  else if (g.slots == 2) in_tile<DT, 2>(a, g, adapter, first, count, blockIdx.y, lds);
  else if (g.slots == 3) in_tile<DT, 3>(a, g, adapter, first, count, blockIdx.y, lds);
  else in_tile<DT, 4>(a, g, adapter, first, count, blockIdx.y, lds);
}

// V goes into the second product as numbers of 16 bits that add up to it: three of bf16, which have all of its bits, or two of fp16, off by 2^-23 of
// a value at most (what is left behind the first one's 11 bits are multiples of 2^-23 of up to 2^-11, and the second one's step is 2^-22 there).
template <int DT>
constexpr int kNumbers = DT == MDBF_BF16 ? 3 : 2;
// How they lie along the contraction: pieces of eight ranks, four to a product.  Up to two of them (rank 16) the numbers follow each other, the
// first one's pieces, the second one's, and so on over as many products as that takes; beyond, a product has four pieces of one number.  Either way one
// operand of B serves all numbers.  (q, k and v of 6458 rows of prompts, 58.9 us as with two numbers a value; 61.7 with an operand of B for the third ones.)
struct Pieces {
  int eights, b_steps, limbs;                  // operands of B, and products per operand
  bool packed;
};
template <int NL>
__host__ __device__ inline Pieces pieces_of(int r) {
  const int eights = (r + 7) / 8;
  if (eights <= 2) return {eights, 1, (eights * NL + 3) / 4, true};
  return {eights, (eights + 3) / 4, NL, false};
}

// Y[row][c] += scale sum over ranks of V[row][rank] B[c][rank].  fp16 has not fp32's exponents: there a row is brought to a largest of 2^14 to 2^15 first, so that the numbers of ranks far below the largest are there too, down to
// 2^-24 (2^-39 of the largest; with a largest of 1 they ended at 2^-24 of it).  The columns of the products' tiles are laid out so that a lane
// ends with 16 neighbouring columns of one row.  A wave takes 64 columns and all of the tile's rows, SUBS times 16, at a time; what it needs of B and Y for
// the first ones is on its way while V is made.
template <int DT, int YD, int SUBS>
__device__ __forceinline__ void out_tile(const OutArgs& a, const OutProj& p, int adapter, int first, int count, U32x4* limbs, const int32_t* rows,
                                         int32_t* exponents) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, kg = lane >> 4;
  constexpr int NL = kNumbers<DT>;
  const Pieces f = pieces_of<NL>(p.r);
  const int c_end = (int)min((int64_t)p.m, ((int64_t)blockIdx.y + 1) * p.chunk);

  const auto load_b = [&](int cb, int s, Raw8<DT>(&w)[4]) {
    const int piece = s * 4 + kg, j8 = (f.packed ? piece % f.eights : piece) * 8;
    const bool there = f.packed || piece < f.eights;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // product row i of tile j is the column cb + (i / 4) * 16 + j * 4 + i % 4
      const int c = min(cb + (i >> 2) * 16 + j * 4 + (i & 3), p.m - 1);
      w[j] = {};
      if (there) load_raw8<DT>(p.B, ((int64_t)adapter * p.m + c) * p.r + j8, p.r - j8, w[j]);
    }
  };
  const auto load_y = [&](int cb, Raw8<YD>(&y)[SUBS][2]) {
    const int c = cb + kg * 16;
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const int row = rows[sub * 16 + i];
      if (row >= 0 && c < p.m) {
        const int64_t at = (int64_t)row * p.ldy + c;
        load_raw8<YD>(p.Y, at, p.m - c, y[sub][0]);
        if (c + 8 < p.m) load_raw8<YD>(p.Y, at + 8, p.m - c - 8, y[sub][1]);
      }
    }
  };
  int cb = (int)blockIdx.y * p.chunk + wave * kOutBlock;
  Raw8<DT> w[4];
  Raw8<YD> y[SUBS][2];
  if (cb < c_end) load_b(cb, 0, w), load_y(cb, y);

  // pieces behind the last (here, while B and Y are on their way)
  const int steps = f.packed ? f.limbs : f.b_steps, numbers = f.packed ? 1 : NL;
  for (int t = tid; t < SUBS * 16; t += 256)
    for (int piece = f.packed ? f.eights * NL : f.eights; piece < steps * 4; ++piece)
      for (int l = 0; l < numbers; ++l)
        limbs[((t >> 4) * steps * numbers + (piece >> 2) * numbers + l) * 64 + (piece & 3) * 16 + (t & 15)] = U32x4{0, 0, 0, 0};

  // a row's pieces of eight ranks lie in a power of two of neighbouring lanes (V's columns behind a rank are zeros up to a multiple of 16)
  const int shift = f.eights > 1 ? 32 - __builtin_clz(f.eights - 1) : 0;
  for (int cell = tid; cell < SUBS << (4 + shift); cell += 256) {
    const int t = cell >> shift, j = cell & ((1 << shift) - 1);
    const bool in = t < count && j < f.eights;
    float v[8] = {};
    if (in) {
      const float* src = a.V + (int64_t)(first + t) * a.width + p.column + j * 8;
      const int64_t apart = (int64_t)a.T * a.width;
      constexpr int U = 4;
      for (int s0 = 0; s0 < a.splits; s0 += U) {
        F32x4 x[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (s0 + u < a.splits) {
            const MDBF_GLOBAL F32x4* q = (const MDBF_GLOBAL F32x4*)(src + (s0 + u) * apart);
            x[u][0] = q[0], x[u][1] = q[1];
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (s0 + u < a.splits) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[u][0][e], v[4 + e] += x[u][1][e];
          }
      }
    }
    if (DT == MDBF_F16) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {            // (an infinity, which an adapter may hold, is one at any power of two)
        const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
        m = max(m, b < 0x7f800000u ? b : 0u);
      }
      for (int o = 1; o < 1 << shift; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
      // the power of two that brings a row's largest finite value into [2^14, 2^15)
      const int b = (int)(m >> 23), e2 = b == 0 ? 0 : b - 127 - 14;
      if (j == 0) exponents[t] = e2;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_ldexpf(v[e], -e2);
    }
    if (j >= f.eights) continue;
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      U32x4 out;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t h = round2<DT>(v[2 * q], v[2 * q + 1]);
        out[q] = h;
        float lo, hi;
        if (DT == MDBF_F16) {
          const F16x2 z = __builtin_bit_cast(F16x2, h);
          lo = (float)z[0], hi = (float)z[1];
        } else {
          lo = __builtin_bit_cast(float, h << 16), hi = __builtin_bit_cast(float, h & 0xffff0000u);
        }
        // (what is not finite is carried by the first number alone)
        v[2 * q] = __builtin_isfinite(lo) ? v[2 * q] - lo : 0.0f;
        v[2 * q + 1] = __builtin_isfinite(hi) ? v[2 * q + 1] - hi : 0.0f;
      }
      const int piece = f.packed ? l * f.eights + j : j, step = f.packed ? piece >> 2 : (piece >> 2) * NL + l;
      limbs[((t >> 4) * f.b_steps * f.limbs + step) * 64 + (piece & 3) * 16 + (t & 15)] = out;
    }
  }
  __syncthreads();

  const float scale = p.scale ? p.scale[adapter] : 1.0f;
  while (cb < c_end) {
    const int c = cb + kg * 16;
    Acc4 acc[SUBS][4] = {};
    for (int s = 0; s < f.b_steps; ++s) {
      Raw8<DT> b[4];
      const bool more = s + 1 < f.b_steps;
      if (more) load_b(cb, s + 1, b);
#pragma unroll NL
      for (int l = 0; l < f.limbs; ++l)
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
          const U32x4 v = limbs[((sub * f.b_steps + s) * f.limbs + l) * 64 + lane];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[sub][j] = product<DT>(w[j].w[0], v, acc[sub][j]);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (more) w[j] = b[j];
    }
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const int t = sub * 16 + i, row = rows[t];
      if (row < 0) continue;
      const int e2 = DT == MDBF_F16 ? exponents[t] : 0;    // (into the sum, which stays far from fp32's ends; a scale may be near them)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (c + 8 * h >= p.m) break;
        float out[8];
        to_float8<YD>(y[sub][h], out);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float sum = acc[sub][2 * h + e / 4][e % 4];
          out[e] = fmaf(scale, DT == MDBF_F16 ? __builtin_ldexpf(sum, e2) : sum, out[e]);
        }
        store_float8<YD, false>(p.Y, (int64_t)row * p.ldy + c + 8 * h, p.m - c - 8 * h, out);
      }
    }
    cb += 4 * kOutBlock;
    if (cb < c_end) load_b(cb, 0, w), load_y(cb, y);
  }
}

template <int DT, int YD>
__global__ __launch_bounds__(256, YD == MDBF_F32 ? 2 : 3) void adapter_out_kernel(OutArgs a) {
  extern __shared__ U32x4 limbs[];             // [sub][operand of B][number][lane]
  __shared__ int32_t rows[MDBF_ADAPTER_TILE], exponents[MDBF_ADAPTER_TILE];
  const OutProj& p = a.p[blockIdx.z];
  int adapter, first, count;
  if (p.yd != YD || (int64_t)blockIdx.y * p.chunk >= p.m) return;
  if (!tile_of(a.tiles, blockIdx.x, a.adapters, a.T, adapter, first, count)) return;
  if (threadIdx.x < MDBF_ADAPTER_TILE) {
    const int row = (int)threadIdx.x < count ? a.rows[first + threadIdx.x] : -1;
    rows[threadIdx.x] = row < a.T ? row : -1;
  }
  __syncthreads();
  if (count <= 16) out_tile<DT, YD, 1>(a, p, adapter, first, count, limbs, rows, exponents);
  else if (count <= 32) out_tile<DT, YD, 2>(a, p, adapter, first, count, limbs, rows, exponents);
  else out_tile<DT, YD, 4>(a, p, adapter, first, count, limbs, rows, exponents);
}

// How a call is cut.
struct AdapterShape {
  int width, splits;
  size_t split_bytes;                          // V of one split
};
static AdapterShape adapter_shape(int count, const mdbf_adapter_t* list, int T, int64_t tile_room) {
  AdapterShape sh = {0, 1, 0};
  int64_t slots = 0;
  int n = 1;
  for (int i = 0; i < count; ++i) {
    sh.width += (list[i].r + 15) / 16 * 16;
    slots += (list[i].r + 15) / 16;
    n = list[i].n > n ? list[i].n : n;
  }
  // enough workgroups to fill the device twice, of 256 channels at least: the second launch reads every split's sums once per chunk of columns
  const int64_t groups = (slots + kInSlots - 1) / kInSlots;
  const int64_t want = 512 / (tile_room * groups);
  const int most = n / 256 < 16 ? n / 256 : 16;
  sh.splits = (int)(want < most ? want : most);
  // (and of the more rows a tile has, the more that is)
  const int64_t rows = T / tile_room > 1 ? T / tile_room : 1, few = 256 / rows > 4 ? 256 / rows : 4;
  if (sh.splits > few) sh.splits = (int)few;
  if (sh.splits < 1) sh.splits = 1;
  sh.split_bytes = (size_t)T * sh.width * 4;
  return sh;
}

static int check_adapters(int count, const mdbf_adapter_t* list, int dtype, int adapters, int T, int64_t tile_room) {
  if (!list || count < 1 || count > MDBF_ADAPTER_MAX || adapters < 1 || T < 1 || tile_room < 1) return MDBF_EINVAL;
  if (dtype != MDBF_F16 && dtype != MDBF_BF16) return MDBF_EDTYPE;
  for (int i = 0; i < count; ++i) {
    const mdbf_adapter_t& l = list[i];
    if (l.n < 1 || l.m < 1 || l.r < 1) return MDBF_EINVAL;
    if (!row_dtype(l.y_dtype)) return MDBF_EDTYPE;
    if (l.r > kMaxRank || l.n > kMaxWidth || l.m > kMaxWidth) return MDBF_EUNSUPPORTED;
  }
  return tile_room > kMaxTiles ? MDBF_EUNSUPPORTED : MDBF_OK;
}

template <int NL>
static size_t limb_bytes(int r) {
  const Pieces f = pieces_of<NL>(r);
  return (size_t)(MDBF_ADAPTER_TILE / 16) * f.b_steps * f.limbs * 1024;
}

template <int DT, int YD>
static int launch_out(const OutArgs& o, int count, int64_t tile_room, int chunks, int rank, hipStream_t s) {
  constexpr int NL = kNumbers<DT>;
  static KernelSetup setup;
  const int e = kernel_setup(setup, [] {
    return hipFuncSetAttribute((const void*)adapter_out_kernel<DT, YD>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)limb_bytes<NL>(kMaxRank));
  });
  if (e) return e;
  adapter_out_kernel<DT, YD><<<dim3((unsigned)tile_room, chunks, count), 256, limb_bytes<NL>(rank), s>>>(o);
  return (int)hipGetLastError();
}

template <int DT>
static int launch_adapters(int count, const mdbf_adapter_t* list, int adapters, int T, const int32_t* rows, const int32_t* tiles, int64_t tile_room,
                           float* V, size_t workspace_bytes, hipStream_t s) {
  AdapterShape sh = adapter_shape(count, list, T, tile_room);
  // (fewer rows may be cut into more splits than the workspace of a larger step has room for)
  if (workspace_bytes / sh.split_bytes < (size_t)sh.splits) sh.splits = (int)(workspace_bytes / sh.split_bytes);
  InArgs in = {};
  OutArgs out = {};
  in.rows = out.rows = rows, in.tiles = out.tiles = tiles, in.V = V, out.V = V;
  in.adapters = out.adapters = adapters, in.T = out.T = T, in.width = out.width = sh.width, in.splits = out.splits = sh.splits;
  int64_t wide = 0;                            // workgroups per tile that take 512 columns each
  for (int i = 0; i < count; ++i) wide += (list[i].m + 8 * kOutBlock - 1) / (8 * kOutBlock);
  int groups = 0, column = 0, yds = 0, ranks[3] = {}, chunks[3] = {};
  for (int i = 0; i < count; ++i) {
    const mdbf_adapter_t& l = list[i];
    in.A[i] = l.A_dev, in.r[i] = l.r, in.column[i] = column;
    for (int t = 0; t < (l.r + 15) / 16; ++t) {
      InGroup* g = groups ? &in.g[groups - 1] : nullptr;
      if (!g || g->slots == kInSlots || g->X != l.X_dev || g->ldx != l.ldx || g->n != l.n) {
        g = &in.g[groups++];
        g->X = l.X_dev, g->ldx = l.ldx, g->n = l.n;
      }
      g->proj[g->slots] = (uint8_t)i, g->tile[g->slots] = (uint8_t)t;
      ++g->slots;
    }
    const int chunk = 4 * kOutBlock * (tile_room * wide >= 512 ? 2 : 1);
    out.p[i] = {l.B_dev, l.Y_dev, l.scale_dev, l.ldy, l.m, l.r, column, l.y_dtype, chunk};
    column += (l.r + 15) / 16 * 16;
    yds |= 1 << l.y_dtype;
    const int c = (l.m + chunk - 1) / chunk;
    if (c > chunks[l.y_dtype]) chunks[l.y_dtype] = c;
    if (l.r > ranks[l.y_dtype]) ranks[l.y_dtype] = l.r;
  }
  adapter_in_kernel<DT><<<dim3((unsigned)tile_room, sh.splits, groups), 256, 0, s>>>(in);
  int e = (int)hipGetLastError();
  if (!e && (yds & 1 << MDBF_F16)) e = launch_out<DT, MDBF_F16>(out, count, tile_room, chunks[MDBF_F16], ranks[MDBF_F16], s);
  if (!e && (yds & 1 << MDBF_BF16)) e = launch_out<DT, MDBF_BF16>(out, count, tile_room, chunks[MDBF_BF16], ranks[MDBF_BF16], s);
  if (!e && (yds & 1 << MDBF_F32)) e = launch_out<DT, MDBF_F32>(out, count, tile_room, chunks[MDBF_F32], ranks[MDBF_F32], s);
  return e;
}

}  // namespace mdbf

using namespace mdbf;

extern "C" {

int64_t mdbf_adapter_tiles(int T, int requests, int adapters) {
  if (T < 1 || requests < 1 || adapters < 1) return MDBF_EINVAL;
  // an adapter's last tile may be short, and only one with rows has one
  const int used = requests < adapters ? requests : adapters;
  return (int64_t)T / MDBF_ADAPTER_TILE + (used < T ? used : T);
}

int mdbf_adapter_rows(int T, int requests, int adapters, const int32_t* cu_dev, const int32_t* adapter_dev, int32_t* rows_dev,
                      int32_t* tiles_dev, int64_t tile_room, int32_t* places_dev, void* stream) {
  if (T < 1 || requests < 1 || adapters < 1 || !cu_dev || !adapter_dev || !rows_dev || !tiles_dev || !places_dev) return MDBF_EINVAL;
  if (tile_room < mdbf_adapter_tiles(T, requests, adapters)) return MDBF_EINVAL;
  if (adapters > kRowMaxAdapters || requests > (1 << 30) || tile_room > (1ll << 30)) return MDBF_EUNSUPPORTED;
  const void* ptrs[] = {cu_dev, adapter_dev, rows_dev, places_dev};
  for (const void* p : ptrs)
    if (!ptr_aligned(p, 4)) return MDBF_EALIGN;
  if (!ptr_aligned(tiles_dev, 16)) return MDBF_EALIGN;
  const int here = T <= kRowOneLaunch && requests <= kRowThreads;
  const RowArgs a = {cu_dev, adapter_dev, rows_dev, tiles_dev, places_dev, tile_room, T, requests, adapters, here};
  const size_t lds = (size_t)(adapters + 1) * 12;
  static KernelSetup setup;
  int e = kernel_setup(setup, [] {
    return hipFuncSetAttribute((const void*)adapter_rows_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (kRowMaxAdapters + 1) * 12);
  });
  if (e) return hip_fail(e);
  adapter_rows_kernel<<<1, kRowThreads, lds, (hipStream_t)stream>>>(a);
  if (!here) adapter_places_kernel<<<(unsigned)(((int64_t)T + kRowChunk - 1) / kRowChunk), kRowChunk, 0, (hipStream_t)stream>>>(a);
  return hip_fail((int)hipGetLastError());
}

int mdbf_adapters_workspace_bytes(int count, const mdbf_adapter_t* list, int dtype, int adapters, int T, int64_t tile_room,
                                  size_t* bytes_out) {
  if (!bytes_out) return MDBF_EINVAL;
  const int st = check_adapters(count, list, dtype, adapters, T, tile_room);
  if (st) return st;
  const AdapterShape sh = adapter_shape(count, list, T, tile_room);
  *bytes_out = sh.splits * sh.split_bytes;
  return MDBF_OK;
}

int mdbf_adapters(int count, const mdbf_adapter_t* list, int dtype, int adapters, int T, const int32_t* rows_dev,
                  const int32_t* tiles_dev, int64_t tile_room, void* workspace_dev, size_t workspace_bytes, void* stream) {
  const int st = check_adapters(count, list, dtype, adapters, T, tile_room);
  if (st) return st;
  if (!rows_dev || !tiles_dev || !workspace_dev) return MDBF_EINVAL;
  if (!ptr_aligned(rows_dev, 4) || !ptr_aligned(tiles_dev, 16) || !ptr_aligned(workspace_dev, 16)) return MDBF_EALIGN;
  for (int i = 0; i < count; ++i) {
    const mdbf_adapter_t& l = list[i];
    if (!l.A_dev || !l.B_dev || !l.X_dev || !l.Y_dev || l.ldx < l.n || l.ldy < l.m) return MDBF_EINVAL;
    const void* ptrs[] = {l.A_dev, l.B_dev, l.X_dev, l.Y_dev};
    for (const void* p : ptrs)
      if (!ptr_aligned(p, 16)) return MDBF_EALIGN;
    if (!ptr_aligned(l.scale_dev, 4)) return MDBF_EALIGN;
    for (int j = 0; j < i; ++j)
      if (list[j].Y_dev == l.Y_dev) return MDBF_EINVAL;
  }
  if (workspace_bytes < adapter_shape(count, list, T, tile_room).split_bytes) return MDBF_EWORKSPACE;
  float* V = (float*)workspace_dev;
  return hip_fail(dtype == MDBF_F16
                      ? launch_adapters<MDBF_F16>(count, list, adapters, T, rows_dev, tiles_dev, tile_room, V, workspace_bytes, (hipStream_t)stream)
                      : launch_adapters<MDBF_BF16>(count, list, adapters, T, rows_dev, tiles_dev, tile_room, V, workspace_bytes, (hipStream_t)stream));
}

}  // extern "C"
