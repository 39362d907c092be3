// Low-rank adapters of many requests beside a shared projection: the order of a step's rows, and Y += scale B (A X).
#include "mdbf_rows.h"

namespace mdbf {

// ---- rows by adapter ------------------------------------------------------------------------------------
// A counting sort by one workgroup: tokens of each adapter (integer sums in LDS), a scan over the adapters for their first places and
// tiles, then the requests in their order, 1024 at a time, each behind those of the same adapter in front of it.  The key
// `adapters` stands for none and comes last.
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

  for (int k = tid; k <= N; k += kRowThreads) count[k] = 0;
  __syncthreads();
  for (int i = tid; i < a.requests; i += kRowThreads) {
    const int f = cut(a.cu[i + 1], a.T) - cut(a.cu[i], a.T), k = a.adapter[i];
    if (f > 0) atomicAdd(&count[k >= 0 && k < N ? k : N], (uint32_t)f);
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
    __syncthreads();                       // the places of the requests before are in `place`, its readers are done
    int from = 0, f = 0, k = N;
    if (tid < n) {
      from = cut(a.cu[i], a.T);
      f = max(cut(a.cu[i + 1], a.T) - from, 0);
      const int asked = a.adapter[i];
      if (asked >= 0 && asked < N) k = asked;
      keys[tid] = k, fresh[tid] = f, first_row[tid] = from;
    }
    __syncthreads();
    uint32_t mine = 0;
    if (tid < n) {
      mine = place[k];
      for (int j = 0; j < tid; ++j) mine += keys[j] == k ? (uint32_t)fresh[j] : 0u;
      a.places[i] = (int)mine;
      first_place[tid] = (int)mine;
    }
    __syncthreads();
    if (tid < n && f) atomicAdd(&place[k], (uint32_t)f);
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
    const uint32_t at = in ? (uint32_t)first_place[lo] + (uint32_t)(t - first_row[lo]) : (uint32_t)t;
    // (rows behind the last request keep their places: there the tables end)
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
  const uint32_t at = in ? (uint32_t)a.places[lo] + (uint32_t)(t - from) : (uint32_t)t;
  if (at < (uint32_t)a.T) a.rows[at] = k >= 0 && k < a.adapters ? t : -1;
}

// ---- products -------------------------------------------------------------------------------------------
struct AdapterProj {
  const void *A, *B, *X;
  void* Y;
  const float* scale;
  float* V;                      // workspace: T x r, by place
  int64_t ldx, ldy;
  int32_t n, m, r, yd;
};
struct AdapterArgs {
  AdapterProj p[MDBF_ADAPTER_MAX];
  const int32_t *rows, *tiles;
  int32_t adapters, T;
};

// the tile's adapter, first place and rows; false for one that is none
__device__ __forceinline__ bool tile_of(const AdapterArgs& a, int64_t t, int& adapter, int& first, int& count) {
  const U32x4 w = *((const MDBF_GLOBAL U32x4*)a.tiles + t);
  adapter = (int)w[0], first = (int)w[1], count = min((int)w[2], MDBF_ADAPTER_TILE);
  if (adapter < 0 || adapter >= a.adapters || first < 0 || first >= a.T || count <= 0) return false;
  count = min(count, a.T - first);
  return true;
}

// The simplest form: a wave per row and rank, then a thread per result.
template <int DT>
__global__ __launch_bounds__(256) void adapter_in_kernel(AdapterArgs a) {
  const AdapterProj& p = a.p[blockIdx.y];
  int adapter, first, count;
  if (!tile_of(a, blockIdx.x, adapter, first, count)) return;
  const int lane = threadIdx.x & 63;
  for (int i = threadIdx.x >> 6; i < count * p.r; i += 4) {
    const int row = a.rows[first + i / p.r], j = i % p.r;
    if (row < 0 || row >= a.T) continue;
    float sum = 0;
    for (int c = lane; c < p.n; c += 64)
      sum += load_as_float(p.X, row * p.ldx + c, DT) * load_as_float(p.A, ((int64_t)adapter * p.r + j) * p.n + c, DT);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) p.V[(int64_t)(first + i / p.r) * p.r + j] = sum;
  }
}

template <int DT>
__global__ __launch_bounds__(256) void adapter_out_kernel(AdapterArgs a) {
  const AdapterProj& p = a.p[blockIdx.y];
  int adapter, first, count;
  if (!tile_of(a, blockIdx.x, adapter, first, count)) return;
  const float scale = p.scale ? p.scale[adapter] : 1.0f;
  for (int i = 0; i < count; ++i) {
    const int row = a.rows[first + i];
    if (row < 0 || row >= a.T) continue;
    for (int c = threadIdx.x; c < p.m; c += 256) {
      float sum = 0;
      for (int j = 0; j < p.r; ++j)
        sum += p.V[(int64_t)(first + i) * p.r + j] * load_as_float(p.B, ((int64_t)adapter * p.m + c) * p.r + j, DT);
      store_from_float(p.Y, row * p.ldy + c, p.yd, load_as_float(p.Y, row * p.ldy + c, p.yd) + scale * sum);
    }
  }
}

static int check_adapters(int count, const mdbf_adapter_t* list, int dtype, int adapters, int T, int64_t tile_room) {
  if (!list || count < 1 || count > MDBF_ADAPTER_MAX || adapters < 1 || T < 1 || tile_room < 1) return MDBF_EINVAL;
  if (dtype != MDBF_F16 && dtype != MDBF_BF16) return MDBF_EDTYPE;
  for (int i = 0; i < count; ++i) {
    const mdbf_adapter_t& l = list[i];
    if (l.n < 1 || l.m < 1 || l.r < 1) return MDBF_EINVAL;
    if (!row_dtype(l.y_dtype)) return MDBF_EDTYPE;
    if (l.r > 256) return MDBF_EUNSUPPORTED;
  }
  return tile_room > (1ll << 30) ? MDBF_EUNSUPPORTED : MDBF_OK;
}
static size_t adapter_ws_bytes(int count, const mdbf_adapter_t* list, int T) {
  size_t n = 0;
  for (int i = 0; i < count; ++i) n += ((size_t)T * list[i].r * 4 + 255) / 256 * 256;
  return n;
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
  *bytes_out = adapter_ws_bytes(count, list, T);
  return MDBF_OK;
}

int mdbf_adapters(int count, const mdbf_adapter_t* list, int dtype, int adapters, int T, const int32_t* rows_dev,
                  const int32_t* tiles_dev, int64_t tile_room, void* workspace_dev, size_t workspace_bytes, void* stream) {
  const int st = check_adapters(count, list, dtype, adapters, T, tile_room);
  if (st) return st;
  if (!rows_dev || !tiles_dev || !workspace_dev) return MDBF_EINVAL;
  if (!ptr_aligned(rows_dev, 4) || !ptr_aligned(tiles_dev, 16) || !ptr_aligned(workspace_dev, 16)) return MDBF_EALIGN;
  AdapterArgs a = {};
  char* ws = (char*)workspace_dev;
  for (int i = 0; i < count; ++i) {
    const mdbf_adapter_t& l = list[i];
    if (!l.A_dev || !l.B_dev || !l.X_dev || !l.Y_dev || l.ldx < l.n || l.ldy < l.m) return MDBF_EINVAL;
    const void* ptrs[] = {l.A_dev, l.B_dev, l.X_dev, l.Y_dev};
    for (const void* p : ptrs)
      if (!ptr_aligned(p, 16)) return MDBF_EALIGN;
    if (!ptr_aligned(l.scale_dev, 4)) return MDBF_EALIGN;
    for (int j = 0; j < i; ++j)
      if (list[j].Y_dev == l.Y_dev) return MDBF_EINVAL;
    a.p[i] = {l.A_dev, l.B_dev, l.X_dev, l.Y_dev, l.scale_dev, (float*)ws, l.ldx, l.ldy, l.n, l.m, l.r, l.y_dtype};
    ws += ((size_t)T * l.r * 4 + 255) / 256 * 256;
  }
  if (workspace_bytes < adapter_ws_bytes(count, list, T)) return MDBF_EWORKSPACE;
  a.rows = rows_dev, a.tiles = tiles_dev, a.adapters = adapters, a.T = T;
  const dim3 grid((unsigned)tile_room, count);
  if (dtype == MDBF_F16) {
    adapter_in_kernel<MDBF_F16><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    adapter_out_kernel<MDBF_F16><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  } else {
    adapter_in_kernel<MDBF_BF16><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    adapter_out_kernel<MDBF_BF16><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  }
  return hip_fail((int)hipGetLastError());
}

}  // extern "C"
