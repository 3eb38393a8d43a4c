// Low-rank adapters of many requests beside a shared projection: y = x W + scale_a (x A_a^T) B_a for the adapter a of
// every token, and its gradients.
#include "gemm_split.h"

namespace {

constexpr int kMostRank = 1024, kMostAdapters = 4096;

inline bool shape_ok(const lz_adapter_shape* s) {
  if (!s || s->T < 0 || s->d_in < 1 || s->d_out < 1 || s->rank < 1 || s->rank > kMostRank) return false;
  if (s->n < 1 || s->n > kMostAdapters || (s->dtype != LZ_F32 && s->dtype != LZ_BF16)) return false;
  const long long d = s->d_in > s->d_out ? s->d_in : s->d_out;
  return s->T <= (1 << 30) && s->T * d < (1ll << 40) && d <= (1 << 22);
}

// Tokens are ordered by adapter with a stable counting sort, those without one last: chunks of consecutive tokens are counted, a
// wave each, the counts summed in order, the tokens placed.  The order is fixed, and with it that of every sum over an adapter's tokens.
constexpr int kChunk = 512;
inline int chunk_tokens(int T) {  // at most 256 chunks of whole waves
  const int even = (T / 256 + 63) / 64 * 64;
  return even > kChunk ? even : kChunk;
}
inline int chunks_of(int T) { return (T + chunk_tokens(T) - 1) / chunk_tokens(T); }

struct AdapterWorkspace {
  int32_t* ids;      // [T], -1: none
  int32_t* counts;   // [chunks, n + 1], then where a chunk's tokens of an adapter go, from the adapter's first row on
  int32_t* first;    // [n + 2]: first row of every adapter, of the tokens without one, T
  int32_t* order;    // [T] row -> token
  int32_t* row_of;   // [T] token -> row
  int32_t* all;      // {0, T}
  void *tiles, *tiles_split;          // row tiles of the adapters' rows
  void *all_tiles, *all_tiles_split;  // of all rows as one slot
  void *xs, *dys;    // x, dy by rows
  float* low;        // [T, rank] before the scale
  void* dh;          // [T, rank]
  float* sum;        // [T, max(d_in, d_out)]
  size_t bytes;
};

AdapterWorkspace carve(void* ws, const lz_adapter_shape* s) {
  AdapterWorkspace w{};
  char* p = (char*)ws;
  auto take = [&](size_t bytes) {
    char* r = p;
    p += lz::align256(bytes);
    return r;
  };
  const size_t T = s->T, eb = lz::elem_bytes(s->dtype), d = s->d_in > s->d_out ? s->d_in : s->d_out;
  w.ids = (int32_t*)take(4 * T);
  w.counts = (int32_t*)take(4 * (size_t)chunks_of(s->T) * (s->n + 1));
  w.first = (int32_t*)take(4 * (s->n + 2));
  w.order = (int32_t*)take(4 * T);
  w.row_of = (int32_t*)take(4 * T);
  w.all = (int32_t*)take(8);
  w.tiles = take(tile_table_bytes(s->T, s->n, kF32Rows));
  w.tiles_split = take(tile_table_bytes(s->T, s->n, kSplitRows));
  w.all_tiles = take(tile_table_bytes(s->T, 1, kF32Rows));
  w.all_tiles_split = take(tile_table_bytes(s->T, 1, kSplitRows));
  w.xs = take(eb * T * s->d_in);
  w.dys = take(eb * T * s->d_out);
  w.low = (float*)take(4 * T * s->rank);
  w.dh = take(eb * T * s->rank);
  w.sum = (float*)take(4 * T * d);
  w.bytes = size_t(p - (char*)ws);
  return w;
}

__global__ __launch_bounds__(64) void count_ids_kernel(const int32_t* __restrict__ ids, int T, int n, int chunk, int32_t* __restrict__ clean,
                                                       int32_t* __restrict__ counts, int32_t* __restrict__ status) {
  extern __shared__ int32_t count[];
  const int lane = threadIdx.x, t0 = blockIdx.x * chunk;
  for (int a = lane; a <= n; a += 64) count[a] = 0;
  __syncthreads();
  bool bad = false;
  for (int t = t0 + lane; t < t0 + chunk && t < T; t += 64) {
    int id = ids[t];
    bad |= id < -1 || id >= n;
    id = id >= 0 && id < n ? id : -1;
    clean[t] = id;
    atomicAdd(&count[id < 0 ? n : id], 1);
  }
  __syncthreads();
  for (int a = lane; a <= n; a += 64) counts[(size_t)blockIdx.x * (n + 1) + a] = count[a];
  if (status != nullptr && bad) atomicOr(status, LZ_ADAPTER_BAD_ID);
}

__global__ void clear_status_kernel(int32_t* status) { *status = 0; }

// One workgroup: counts -> where each chunk's tokens of an adapter start within the adapter's rows, and the adapters' first rows.
__global__ __launch_bounds__(1024) void scan_ids_kernel(int32_t* __restrict__ counts, int chunks, int n, int T, int32_t* __restrict__ first,
                                                        int32_t* __restrict__ all) {
  __shared__ int32_t waves[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base = 0;
  for (int a0 = 0; a0 <= n; a0 += 1024) {
    const int a = a0 + tid;
    int total = 0;
    for (int c = 0; a <= n && c < chunks; ++c) {
      int32_t& at = counts[(size_t)c * (n + 1) + a];
      const int here = at;
      at = total;
      total += here;
    }
    const int incl = lz::wave_scan(total, [](int x, int y) { return x + y; });
    if (lane == 63) waves[wave] = incl;
    __syncthreads();
    int before = base;
    for (int w = 0; w < wave; ++w) before += waves[w];
    if (a <= n) first[a] = before + incl - total;
    for (int w = 0; w < 16; ++w) base += waves[w];
    __syncthreads();
  }
  if (tid == 0) {
    first[n + 1] = T;
    all[0] = 0;
    all[1] = T;
  }
}

__global__ __launch_bounds__(64) void place_ids_kernel(const int32_t* __restrict__ clean, int T, int n, int chunk,
                                                       const int32_t* __restrict__ counts, const int32_t* __restrict__ first,
                                                       int32_t* __restrict__ order, int32_t* __restrict__ row_of) {
  extern __shared__ int32_t next[];
  const int lane = threadIdx.x, t0 = blockIdx.x * chunk;
  for (int a = lane; a <= n; a += 64) next[a] = first[a] + counts[(size_t)blockIdx.x * (n + 1) + a];
  __syncthreads();
  for (int t1 = t0; t1 < t0 + chunk && t1 < T; t1 += 64) {
    const int t = t1 + lane;
    int id = t < T ? clean[t] : -2;
    if (id == -1) id = n;
    unsigned long long left = __ballot(id >= 0);
    while (left != 0) {  // the tokens of one adapter, in order
      const int leader = __ffsll((long long)left) - 1, a = __shfl(id, leader);
      const unsigned long long same = __ballot(id == a);
      if (id == a) {
        const int row = next[a] + __popcll(same & ((1ull << lane) - 1));
        order[row] = t;
        row_of[t] = row;
      }
      __syncthreads();  // (one wave) read before it is written
      if (lane == leader) next[a] += __popcll(same);
      __syncthreads();
      left &= ~same;
    }
  }
}

// to[r] = from[map[r]], rounded to To; rows of `cols`
template <typename From, typename To>
__global__ __launch_bounds__(256) void move_rows_kernel(const From* __restrict__ from, const int32_t* __restrict__ map, long long rows, int cols,
                                                        To* __restrict__ to) {
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const From* const src = from + (size_t)map[r] * cols;
    for (int c = threadIdx.x; c < cols; c += 256) store_elem<To>(to + (size_t)r * cols + c, load_elem<From>(src + c));
  }
}
template <typename From, typename To>
int32_t move_rows(const From* from, const int32_t* map, long long rows, int cols, To* to, hipStream_t st) {
  hipLaunchKernelGGL((move_rows_kernel<From, To>), dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(256), 0, st, from, map, rows, cols, to);
  return lz::launch_status();
}

template <typename Elem>
__global__ __launch_bounds__(256) void clear_kernel(Elem* __restrict__ p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = Elem(0);
}

// h[r] = scale of the row's adapter times low[r], rounded once; zero for rows without one
template <typename Elem>
__global__ __launch_bounds__(256) void scale_rows_kernel(const float* __restrict__ low, const float* __restrict__ scale,
                                                         const int32_t* __restrict__ order, const int32_t* __restrict__ ids, long long T, int rank,
                                                         Elem* __restrict__ h) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < T * rank; i += (long long)gridDim.x * 256) {
    const int id = ids[order[i / rank]];
    store_elem<Elem>(h + i, id >= 0 ? scale[id] * low[i] : 0.f);
  }
}

inline unsigned blocks_of(size_t n) {
  const size_t b = (n + 255) / 256;
  return (unsigned)(b < 4096 ? (b > 0 ? b : 1) : 4096);
}

// out (fp32) = A W, or added to it, over all rows or the adapters'
template <typename Elem, bool WKM>
int32_t product(const AdapterWorkspace& w, const lz_adapter_shape* s, bool by_adapter, const void* A, int K, const void* W, int n_out,
                float* out, bool add, hipStream_t st) {
  F32Args a{};
  a.A = A;
  a.W = W;
  a.C = out;
  a.Cacc = out;
  a.K = a.lda = K;
  a.ldw = WKM ? n_out : K;
  a.ldc = a.n_out = n_out;
  const int S = by_adapter ? s->n : 1;
  a.w_slot = by_adapter ? (long long)K * n_out : 0;
  a.t = carve_tiles(by_adapter ? w.tiles : w.all_tiles, s->T, S, kF32Rows);
  a.t_split = carve_tiles(by_adapter ? w.tiles_split : w.all_tiles_split, s->T, S, kSplitRows);
  if constexpr (sizeof(Elem) == 4) {
    if (!add) return launch_f32_rows<Elem, EPI_NONE, WKM>(a, S, s->T, st);
  } else if (!add) {  // bf16 results would be rounded here
    const size_t n = (size_t)s->T * n_out;
    hipLaunchKernelGGL(clear_kernel<float>, dim3(blocks_of(n)), dim3(256), 0, st, out, n);
  }
  return launch_f32_rows<Elem, EPI_ACCUM, WKM>(a, S, s->T, st);
}

// The low-rank part of either direction: h = scale (rows A^T), rounded
template <typename Elem>
int32_t low_rank(const AdapterWorkspace& w, const lz_adapter_shape* s, const void* rows, int d, const void* A, const float* scale, void* h,
                 hipStream_t st) {
  const size_t n = (size_t)s->T * s->rank;
  hipLaunchKernelGGL(clear_kernel<float>, dim3(blocks_of(n)), dim3(256), 0, st, w.low, n);  // rows without an adapter too
  const int32_t rc = product<Elem, false>(w, s, true, rows, d, A, s->rank, w.low, true, st);
  if (rc != LZ_OK) return rc;
  hipLaunchKernelGGL((scale_rows_kernel<Elem>), dim3(blocks_of(n)), dim3(256), 0, st, w.low, scale, w.order, w.ids, (long long)s->T, s->rank,
                     (Elem*)h);
  return lz::launch_status();
}

template <typename Elem>
int32_t forward(const AdapterWorkspace& w, const lz_adapter_shape* s, const void* x, const void* W, const void* a, const void* b,
                const float* scale, void* h, void* y, hipStream_t st) {
  int32_t rc = move_rows<Elem, Elem>((const Elem*)x, w.order, s->T, s->d_in, (Elem*)w.xs, st);
  if (rc == LZ_OK) rc = low_rank<Elem>(w, s, w.xs, s->d_in, a, scale, h, st);
  if (rc == LZ_OK) rc = product<Elem, true>(w, s, false, w.xs, s->d_in, W, s->d_out, w.sum, false, st);
  if (rc == LZ_OK) rc = product<Elem, true>(w, s, true, h, s->rank, b, s->d_out, w.sum, true, st);
  if (rc == LZ_OK) rc = move_rows<float, Elem>(w.sum, w.row_of, s->T, s->d_out, (Elem*)y, st);
  return rc;
}

template <typename Elem>
int32_t backward(const AdapterWorkspace& w, const lz_adapter_shape* s, const void* dy, const void* x, const void* h, const void* W,
                 const void* a, const void* b, const float* scale, void* dx, void* da, void* db, hipStream_t st) {
  int32_t rc = move_rows<Elem, Elem>((const Elem*)x, w.order, s->T, s->d_in, (Elem*)w.xs, st);
  if (rc == LZ_OK) rc = move_rows<Elem, Elem>((const Elem*)dy, w.order, s->T, s->d_out, (Elem*)w.dys, st);
  if (rc == LZ_OK) rc = low_rank<Elem>(w, s, w.dys, s->d_out, b, scale, w.dh, st);
  if (rc == LZ_OK) rc = product<Elem, false>(w, s, false, w.dys, s->d_out, W, s->d_in, w.sum, false, st);
  if (rc == LZ_OK) rc = product<Elem, true>(w, s, true, w.dh, s->rank, a, s->d_in, w.sum, true, st);
  if (rc == LZ_OK) rc = move_rows<float, Elem>(w.sum, w.row_of, s->T, s->d_in, (Elem*)dx, st);
  if (rc == LZ_OK) rc = launch_f32_wgrad<Elem, EPI_NONE>(f32_wgrad<Elem>(w.dh, s->rank, w.xs, s->d_in, w.first, s->n, s->T, da, nullptr), st);
  if (rc == LZ_OK) rc = launch_f32_wgrad<Elem, EPI_NONE>(f32_wgrad<Elem>(h, s->rank, w.dys, s->d_out, w.first, s->n, s->T, db, nullptr), st);
  return rc;
}

int32_t check(const lz_adapter_shape* s, void* ws, size_t ws_bytes, AdapterWorkspace* w) {
  if (!shape_ok(s)) return LZ_ESHAPE;
  *w = carve(ws, s);
  if (!ws || (uintptr_t)ws % 256 != 0 || ws_bytes < w->bytes) return LZ_EWORKSPACE;
  return LZ_OK;
}

}  // namespace

extern "C" size_t lz_adapter_workspace_bytes(const lz_adapter_shape* shape) {
  return shape_ok(shape) ? carve(nullptr, shape).bytes : 0;
}

extern "C" int32_t lz_adapter_plan(const int32_t* ids, const lz_adapter_shape* shape, int32_t* status_opt, void* ws, size_t ws_bytes,
                                   void* stream) {
  AdapterWorkspace w;
  int32_t rc = check(shape, ws, ws_bytes, &w);
  if (rc != LZ_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (shape->T > 0 && !ids) return LZ_EINVAL;
  if (status_opt) hipLaunchKernelGGL(clear_status_kernel, dim3(1), dim3(1), 0, st, status_opt);
  if (shape->T == 0) return lz::launch_status();
  const int T = shape->T, n = shape->n, chunk = chunk_tokens(T), chunks = chunks_of(T);
  const size_t lds = 4 * (size_t)(n + 1);
  hipLaunchKernelGGL(count_ids_kernel, dim3(chunks), dim3(64), lds, st, ids, T, n, chunk, w.ids, w.counts, status_opt);
  hipLaunchKernelGGL(scan_ids_kernel, dim3(1), dim3(1024), 0, st, w.counts, chunks, n, T, w.first, w.all);
  hipLaunchKernelGGL(place_ids_kernel, dim3(chunks), dim3(64), lds, st, w.ids, T, n, chunk, w.counts, w.first, w.order, w.row_of);
  rc = lz::launch_status();
  if (rc != LZ_OK) return rc;
  auto tables = [&](const int32_t* offsets, int S, void* rows, void* split) {
    TileSpecs specs{};
    add_rows(specs, kF32Rows, T, carve_tiles(rows, T, S, kF32Rows));
    add_rows(specs, kSplitRows, T, carve_tiles(split, T, S, kSplitRows));
    return launch_build_tiles(offsets, S, specs, st);
  };
  rc = tables(w.first, n, w.tiles, w.tiles_split);
  return rc == LZ_OK ? tables(w.all, 1, w.all_tiles, w.all_tiles_split) : rc;
}

extern "C" int32_t lz_adapter_forward(const void* x, const void* w, const void* a, const void* b, const float* scale,
                                      const lz_adapter_shape* shape, void* h, void* y, void* ws, size_t ws_bytes, void* stream) {
  AdapterWorkspace m;
  const int32_t rc = check(shape, ws, ws_bytes, &m);
  if (rc != LZ_OK || shape->T == 0) return rc;
  if (!x || !w || !a || !b || !scale || !h || !y) return LZ_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  return shape->dtype == LZ_F32 ? forward<float>(m, shape, x, w, a, b, scale, h, y, st)
                                : forward<uint16_t>(m, shape, x, w, a, b, scale, h, y, st);
}

extern "C" int32_t lz_adapter_backward(const void* dy, const void* x, const void* h, const void* w, const void* a, const void* b,
                                       const float* scale, const lz_adapter_shape* shape, void* dx, void* da, void* db, void* ws,
                                       size_t ws_bytes, void* stream) {
  AdapterWorkspace m;
  const int32_t rc = check(shape, ws, ws_bytes, &m);
  if (rc != LZ_OK) return rc;
  if (!da || !db) return LZ_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  if (shape->T == 0) {  // no tokens, no gradients
    auto clear = [&](void* p, int d) {
      const size_t elems = (size_t)shape->n * shape->rank * d;
      if (shape->dtype == LZ_F32) hipLaunchKernelGGL(clear_kernel<float>, dim3(blocks_of(elems)), dim3(256), 0, st, (float*)p, elems);
      else hipLaunchKernelGGL(clear_kernel<uint16_t>, dim3(blocks_of(elems)), dim3(256), 0, st, (uint16_t*)p, elems);
    };
    clear(da, shape->d_in);
    clear(db, shape->d_out);
    return lz::launch_status();
  }
  if (!dy || !x || !h || !w || !a || !b || !scale || !dx) return LZ_EINVAL;
  return shape->dtype == LZ_F32 ? backward<float>(m, shape, dy, x, h, w, a, b, scale, dx, da, db, st)
                                : backward<uint16_t>(m, shape, dy, x, h, w, a, b, scale, dx, da, db, st);
}
