// Low-rank adapters on the bf16 matrix cores of gfx950: which adapters a tile's tokens use, the low-rank products h, the
// projection on narrow tiles, the factors' gradients.  The projection on wide tiles is gemm_mfma.h's, EPI_ADAPTER.
// Device code of adapter.hip, not part of the C ABI.
//
// The projection takes a tile of tokens in their own order, whatever adapters they use: the low-rank part is more K steps of the same
// sum, one or more for every adapter that occurs in the tile, in which the rows of h that use another one read as zeros.  A batch of
// requests with some hundred tokens each has one or two adapters in a tile; at worst (every token another one) the steps are those of a
// dense product over all adapters.  Sorting tokens by adapter instead would cost x and y a gather and a scatter.
#pragma once
#include "gemm_narrow.h"

namespace {

// Which adapters the tokens of 256 and of 64 consecutive rows use, and where in that list each row's stands (255: none).
struct AdapterLists {
  int32_t *count256, *list256;
  uint8_t* local256;  // permuted, see AdapterSteps
  int32_t *count64, *list64;
  uint8_t* local64;
};

__global__ __launch_bounds__(256) void adapter_lists_kernel(const int32_t* __restrict__ ids, int T, int n, int32_t* __restrict__ clean,
                                                            AdapterLists out, int32_t* status) {
  extern __shared__ int32_t first[];  // [n]: the first row of an adapter, then its place in the list
  __shared__ int32_t counts[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t = blockIdx.x * 256 + tid;
  for (int a = tid; a < n; a += 256) first[a] = 256;
  int id = t < T ? ids[t] : -1;
  const bool bad = id < -1 || id >= n;
  if (bad) id = -1;
  if (t < T) clean[t] = id;
  if (status != nullptr) {
    if (gridDim.x == 1) {
      const int any = __syncthreads_or(bad);
      if (tid == 0) *status = any ? LZ_ADAPTER_BAD_ID : 0;
    } else if (bad) {
      atomicOr(status, LZ_ADAPTER_BAD_ID);
    }
  }
  // 64 rows, one wave: adapters in the order in which they occur
  const int block = blockIdx.x * 4 + wave;
  int place = 255, n64 = 0;
  for (unsigned long long left = __ballot(id >= 0); left != 0; ++n64) {
    const int a = __shfl(id, __ffsll((long long)left) - 1);
    const unsigned long long same = __ballot(id == a);
    if (id == a) place = n64;
    if (lane == 0) out.list64[(size_t)block * 64 + n64] = a;
    left &= ~same;
  }
  out.local64[(size_t)block * 64 + lane] = (uint8_t)place;
  if (lane == 0) out.count64[block] = n64;
  // 256 rows
  __syncthreads();
  if (id >= 0) atomicMin(&first[id], tid);
  __syncthreads();
  const bool leads = id >= 0 && first[id] == tid;
  const unsigned long long leaders = __ballot(leads);
  if (lane == 0) counts[wave] = __popcll(leaders);
  __syncthreads();
  int at = __popcll(leaders & ((1ull << lane) - 1));
  for (int w = 0; w < wave; ++w) at += counts[w];
  if (leads) {
    out.list256[(size_t)blockIdx.x * 256 + at] = id;
    first[id] = at;
  }
  if (tid == 0) out.count256[blockIdx.x] = counts[0] + counts[1] + counts[2] + counts[3];
  __syncthreads();
  const int r = tid;
  out.local256[(size_t)blockIdx.x * 256 + 8 * (8 * ((r >> 3) & 3) + (r & 7)) + (r >> 5)] = id >= 0 ? (uint8_t)first[id] : 255;
}

// ---- h[t] = scale x[t] A^T of the token's adapter, rounded once; zeros without one.

struct LowRankArgs {
  const uint16_t* x;  // [T, d]
  const uint16_t* a;  // [n, rank, d]
  const float* scale;
  const int32_t* ids;
  const int32_t *count64, *list64;
  const uint8_t* local64;
  uint16_t* h;  // [T, rank]
  int T, d, rank;
};

__device__ __forceinline__ bf16x8 load_bf16x8(const uint16_t* p) { return *(const bf16x8*)p; }

// Few tokens: a wave per token and row of its factor.
__global__ __launch_bounds__(256) void low_rank_token_kernel(LowRankArgs a) {
  const int t = blockIdx.x, r = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.rank) return;
  const int id = __builtin_amdgcn_readfirstlane(a.ids[t]);
  float sum = 0.f;
  if (id >= 0) {
    const uint16_t* const x = a.x + (size_t)t * a.d;
    const uint16_t* const w = a.a + ((size_t)id * a.rank + r) * a.d;
#pragma unroll 4
    for (int k = lane * 8; k < a.d; k += 512) {
      const bf16x8 u = load_bf16x8(x + k), v = load_bf16x8(w + k);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf((float)u[j], (float)v[j], sum);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    sum *= a.scale[id];
  }
  if (lane == 0) a.h[(size_t)t * a.rank + r] = lz::f32_to_bf16(sum);
}

// 16 RT tokens a workgroup, 64 columns of h at a time, for every adapter among the tokens.  Eight waves take every eighth 64 k of
// the sum each, from global memory to the registers (nothing is used twice but by the other fragments of the wave), and add up
// through LDS.  Bound by reading x once.
template <int RT>
__global__ __launch_bounds__(512) void low_rank_kernel(LowRankArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kRows = 16 * RT;
  __shared__ float part[8][kRows][64 + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * kRows, block = t0 / 64, frag = lane & 15, quad = lane >> 4;
  const int mine = lane < kRows ? a.local64[(size_t)t0 + lane] : 255;  // (rows past T: 255)
  for (int i = threadIdx.x; i < kRows * a.rank; i += 512)
    if (a.local64[(size_t)t0 + i / a.rank] == 255 && t0 + i / a.rank < a.T) a.h[(size_t)t0 * a.rank + i] = 0;
  const uint16_t* xrow[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const int t = t0 + j * 16 + frag;
    xrow[j] = a.x + (size_t)(t < a.T ? t : a.T - 1) * a.d;
  }
  const bf16x8 none = {};
  const int count = a.count64[block];
  for (int e = 0; e < count; ++e) {
    if (__ballot(mine == e) == 0) continue;  // the same in every wave
    const int id = __builtin_amdgcn_readfirstlane(a.list64[(size_t)block * 64 + e]);
    const float scale = a.scale[id];
    for (int r0 = 0; r0 < a.rank; r0 += 64) {
      const int frags = (a.rank - r0 + 15) / 16 < 4 ? (a.rank - r0 + 15) / 16 : 4;
      f32x4 acc[4][RT] = {};
      auto sum = [&](auto n_frags) {
        constexpr int NF = decltype(n_frags)::value;
        const uint16_t* arow[NF];
        bool in[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          in[f] = r0 + f * 16 + frag < a.rank;
          arow[f] = a.a + ((size_t)id * a.rank + (in[f] ? r0 + f * 16 + frag : r0)) * a.d;
        }
#pragma clang loop unroll_count(2)
        for (int k = wave * 64; k < a.d; k += 512) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int at = k + half * 32 + quad * 8;
            const bool ok = at < a.d;
            bf16x8 x[RT], w[NF];
#pragma unroll
            for (int j = 0; j < RT; ++j) x[j] = ok ? load_bf16x8(xrow[j] + at) : none;
#pragma unroll
            for (int f = 0; f < NF; ++f) w[f] = ok && in[f] ? load_bf16x8(arow[f] + at) : none;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
              for (int j = 0; j < RT; ++j) acc[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], x[j], acc[f][j], 0, 0, 0);
          }
        }
      };
      if (frags == 1) sum(std::integral_constant<int, 1>{});
      else if (frags == 2) sum(std::integral_constant<int, 2>{});
      else sum(std::integral_constant<int, 4>{});
#pragma unroll
      for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int j = 0; j < RT; ++j)
          if (f < frags) *(f32x4*)&part[wave][j * 16 + frag][f * 16 + 4 * quad] = acc[f][j];
      __syncthreads();
      const int cols = frags * 16;
      for (int i = threadIdx.x; i < kRows * cols; i += 512) {
        const int r = i / cols, c = i - r * cols;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w][r][c];
        if (a.local64[(size_t)t0 + r] == e && r0 + c < a.rank) a.h[(size_t)(t0 + r) * a.rank + r0 + c] = lz::f32_to_bf16(scale * s);
      }
      __syncthreads();
    }
  }
#endif
}

// ---- the projection on 64 x 64 tiles, the sum over K split among workgroups where tiles are few

struct AdapterNarrowArgs {
  const uint16_t* A;  // [T, K]
  const uint16_t* W;  // MODE_NN: [K, n_out], MODE_NT: [n_out, K]
  uint16_t* C;        // [T, n_out]
  float* part;        // [splits, T, n_out]
  const uint16_t* h;  // [T, rank]
  const uint16_t* b;  // MODE_NN: [n, rank, n_out], MODE_NT: [n, n_out, rank]
  const int32_t *count64, *list64;
  const uint8_t* local64;
  int T, K, n_out, rank, n, n_tiles, splits;
};

// As gemm_narrow.h's kernel: a ring of K steps for both operands.  The steps behind the base's take 64 k of h, those of 64 / rank
// adapters of the tile's list or a part of one's.  blockIdx.x = row tile x split x column tile, columns fastest.
template <int MODE, bool KTAIL>
__global__ __launch_bounds__(256, 2) void adapter_narrow_kernel(AdapterNarrowArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool TB = MODE == MODE_NN;
  constexpr int NS = kNarrowStages, kLoads = 4;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ int32_t list[64];
  const int col_tile = blockIdx.x % a.n_tiles, rest = blockIdx.x / a.n_tiles, split = rest % a.splits, row_tile = rest / a.splits;
  const int row0 = row_tile * kNarrow, n0 = col_tile * kNarrow, K = a.K, rank = a.rank;
  const int n_rows = a.T - row0 < kNarrow ? a.T - row0 : kNarrow;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int count = __builtin_amdgcn_readfirstlane(a.count64[row_tile]);
  if (threadIdx.x < 64) list[threadIdx.x] = (int)threadIdx.x < count ? a.list64[(size_t)row_tile * 64 + threadIdx.x] : 0;

  const int ldw = TB ? a.n_out : K;
  const i32x4 wordsA = rsrc_words(a.A + (size_t)row0 * K, (uint32_t)n_rows * (uint32_t)K * 2u);
  const i32x4 wordsW = rsrc_words(a.W, (uint32_t)((unsigned long long)K * (unsigned)a.n_out * 2ull));
  const i32x4 wordsH = rsrc_words(a.h + (size_t)row0 * rank, (uint32_t)n_rows * (uint32_t)rank * 2u);
  const i32x4 wordsB = rsrc_words(a.b, (uint32_t)((unsigned long long)a.n * (unsigned)rank * (unsigned)a.n_out * 2ull));
  const i32x4 wordsNull = rsrc_words(a.A, 0);
  const int stepW = TB ? BK * ldw * 2 : BK * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // low-rank steps: k of the step -> adapter in the list from the step's first on, place in its factor
  const int per = rank <= 64 ? 64 / rank : 1, steps_each = rank <= 64 ? 1 : (rank + 63) / 64;
  int voffX[2], voffW[2], row[2], local[2], chunk[2], kr[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (wave * 2 + i) * 8 + (lane >> 3);
    row[i] = r;
    chunk[i] = ((lane & 7) ^ swz(r)) * 8;
    local[i] = r < n_rows ? a.local64[(size_t)row0 + r] : 255;
    voffX[i] = (int)(((uint32_t)r * (uint32_t)K + (uint32_t)chunk[i]) * 2u);  // rows past the end lie beyond the descriptor: zeros
    if constexpr (TB) {
      kr[i] = r;
      voffW[i] = (int)(((uint32_t)r * (uint32_t)ldw + (uint32_t)(n0 + ((lane & 7) ^ swz_narrow(r)) * 8)) * 2u);
    } else {
      kr[i] = chunk[i];
      voffW[i] = (int)(((uint32_t)(n0 + r) * (uint32_t)K + (uint32_t)chunk[i]) * 2u);
    }
  }
  [[maybe_unused]] int tail_or[2] = {0, 0};
  const int base_steps = (K + BK - 1) / BK;
  if constexpr (KTAIL) {
    const int k_left = K - (base_steps - 1) * BK;
#pragma unroll
    for (int i = 0; i < 2; ++i) tail_or[i] = chunk[i] >= k_left ? (int)0x80000000 : 0;
  }
  const int all_steps = base_steps + (count + per - 1) / per * steps_each;
  const int begin = (int)((long long)all_steps * split / a.splits), end = (int)((long long)all_steps * (split + 1) / a.splits);
  __syncthreads();  // the list
  auto issue = [&](int step, int stage) {  // a step past the end writes zeros, without memory traffic
    const uint32_t lds = lds0 + stage * kNarrowStage;
    if (step >= base_steps && step < end) {
      const int q = step - base_steps, e0 = q / steps_each * per, k0 = q % steps_each * 64;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int in = rank <= 64 ? kr[i] / rank : 0, k = k0 + kr[i] - in * rank, e = e0 + in;
        const bool ok = in < per && e < count && k < rank;
        const int id = list[ok ? e : 0];
        int voff;
        if constexpr (TB) voff = ((id * rank + k) * a.n_out + n0 + ((lane & 7) ^ swz_narrow(row[i])) * 8) * 2;
        else voff = ((id * a.n_out + n0 + row[i]) * rank + k) * 2;
        // (columns past n_out fetch what lies behind: never stored)
        load16_to_lds(wordsB, lds + kNarrowOperand + (wave * 2 + i) * 1024, ok ? voff : (int)0x80000000, 0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int in = rank <= 64 ? chunk[i] / rank : 0, k = k0 + chunk[i] - in * rank, e = e0 + in;
        const bool ok = in < per && e < count && k < rank && local[i] == e;
        load16_to_lds(wordsH, lds + (wave * 2 + i) * 1024, ok ? (row[i] * rank + k) * 2 : (int)0x80000000, 0);
      }
      return;
    }
    const bool real = step < end;
    const i32x4 wa = real ? wordsA : wordsNull, ww = real ? wordsW : wordsNull;
    const int tail = step == base_steps - 1 ? -1 : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int voff = voffW[i];
      if constexpr (KTAIL && !TB) voff |= tail_or[i] & tail;
      load16_to_lds(ww, lds + kNarrowOperand + (wave * 2 + i) * 1024, voff, real ? step * stepW : 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int voff = voffX[i];
      if constexpr (KTAIL) voff |= tail_or[i] & tail;
      load16_to_lds(wa, lds + (wave * 2 + i) * 1024, voff, real ? step * BK * 2 : 0);
    }
  };
  int fragoff[2], woff[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int r = lane & 15;
    fragoff[ks] = r * kRowBytes + (((ks * 4 + (lane >> 4)) ^ swz(r)) << 4);
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if constexpr (TB) {
      const int q = lane & 15, k_row = 8 * (lane >> 4) + (q >> 2);
      woff[c] = k_row * kRowBytes + ((q & 1) << 3) + (((((2 * wn + c) << 1) | ((q >> 1) & 1)) ^ swz_narrow(k_row)) << 4);
    } else {
      woff[c] = (2 * wn + c) * 16 * kRowBytes;
    }
  }
  auto read_x = [&](const char* st, int ks, int j) { return *(const bf16x8*)(st + (2 * wm + j) * 16 * kRowBytes + fragoff[ks]); };
  auto read_w = [&](const char* st, int ks, int c) {
    if constexpr (TB) {
      const char* p = st + kNarrowOperand + woff[c] + ks * 32 * kRowBytes;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + 4 * kRowBytes));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(const bf16x8*)(st + kNarrowOperand + woff[c] + fragoff[ks]);
    }
  };
  f32x4 acc[2][2] = {};
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue(begin + s, s);
  int stage = 0;
  for (int kt = begin; kt < end; ++kt) {
    constexpr int kAhead = (NS - 2) * kLoads;
    __builtin_amdgcn_s_waitcnt(0x0F70 | (kAhead & 15) | ((kAhead >> 4) << 14));  // this wave's loads of step kt are in LDS
    __syncthreads();  // ... everyone's are; and nobody reads the stage of step kt - 1 any more
    issue(kt + NS - 1, stage == 0 ? NS - 1 : stage - 1);
    const char* const st = smem + stage * kNarrowStage;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 x[2], w[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) w[c] = read_w(st, ks, c);
#pragma unroll
      for (int j = 0; j < 2; ++j) x[j] = read_x(st, ks, j);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c], x[j], acc[c][j], 0, 0, 0);
    }
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
  // the trailing loads still write zeros into stages: drained by every wave before the tile overwrites them
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  constexpr int kPitch = kNarrow + 4;
  float* const tile = (float*)smem;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *(f32x4*)(tile + (32 * wm + 16 * j + (lane & 15)) * kPitch + 32 * wn + 16 * c + 4 * (lane >> 4)) = acc[c][j];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = threadIdx.x + 256 * i, r = p >> 3, c = (p & 7) * 8;
    if (r >= n_rows || n0 + c >= a.n_out) continue;  // row lengths are multiples of 8
    const f32x4 v0 = *(const f32x4*)(tile + r * kPitch + c), v1 = *(const f32x4*)(tile + r * kPitch + c + 4);
    const size_t at = (size_t)(row0 + r) * a.n_out + n0 + c;
    if (a.splits > 1) {
      float* const to = a.part + (size_t)split * a.T * a.n_out + at;
      *(f32x4*)to = v0;
      *(f32x4*)(to + 4) = v1;
    } else {
      *(u32x4_t*)(a.C + at) = u32x4_t{pack_bf16x2(v0[0], v0[1]), pack_bf16x2(v0[2], v0[3]), pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3])};
    }
  }
#endif
}

// The splits' sums, in their order.
__global__ __launch_bounds__(256) void join_splits_kernel(const float* __restrict__ part, int splits, size_t elems, uint16_t* __restrict__ out) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= elems) return;
  f32x4 v0 = {}, v1 = {};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    v0 += *(const f32x4*)(part + s * elems + i);
    v1 += *(const f32x4*)(part + s * elems + i + 4);
  }
  *(u32x4_t*)(out + i) = u32x4_t{pack_bf16x2(v0[0], v0[1]), pack_bf16x2(v0[2], v0[3]), pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3])};
}

// Lets a kernel have so much dynamic LDS; once per device (idempotent).
template <auto KERNEL>
int32_t allow_lds(int bytes) {
  static std::atomic<bool> ready_on_device[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return LZ_EHIP;
  if (!ready_on_device[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return LZ_EHIP;
    ready_on_device[dev].store(true, std::memory_order_release);
  }
  return LZ_OK;
}

template <int MODE>
int32_t launch_adapter_narrow(AdapterNarrowArgs a, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(a.T, kNarrow) * (long long)a.splits * a.n_tiles);
  const bool tail = a.K % BK != 0;
  const int32_t rc = tail ? allow_lds<adapter_narrow_kernel<MODE, true>>(kNarrowLds) : allow_lds<adapter_narrow_kernel<MODE, false>>(kNarrowLds);
  if (rc != LZ_OK) return rc;
  if (tail) hipLaunchKernelGGL((adapter_narrow_kernel<MODE, true>), dim3(grid), dim3(256), kNarrowLds, st, a);
  else hipLaunchKernelGGL((adapter_narrow_kernel<MODE, false>), dim3(grid), dim3(256), kNarrowLds, st, a);
  if (a.splits > 1) {
    const size_t elems = (size_t)a.T * a.n_out;
    hipLaunchKernelGGL(join_splits_kernel, dim3((unsigned)((elems / 8 + 255) / 256)), dim3(256), 0, st, a.part, a.splits, elems, a.C);
  }
  return lz::launch_status();
}

// ---- the factors' gradients: sums over an adapter's tokens, in chunks of rows of the order by adapter

struct FactorArgs {
  const uint16_t *h, *x;  // [T, rank], [T, d]
  uint16_t* out;          // [n, rank, d]
  float* part;            // [units, rank, d], of adapters of several units
  int d, n_tiles;
};
struct FactorPair {
  FactorArgs f[2];
  const int32_t *first, *order;  // first row of every adapter; row -> token
  const int32_t *unit_first;     // [n + 1] first unit of every adapter
  const int32_t *unit_adapter;   // [units]
  int n, rank, rank_tiles, chunk;
};
constexpr int kFactorCols = 128, kFactorStages = 3;
constexpr int kFactorX = 64 * kFactorCols * 2, kFactorStage = kFactorX + kNarrowOperand;  // 64 tokens of both operands
constexpr int kMostChunk = 2048;
constexpr int kFactorLds = kFactorStages * kFactorStage + kMostChunk * 4;

__device__ __forceinline__ int swz_factor(int kr) { return ((kr & 3) << 1) | (((kr >> 3) & 1) << 3); }

// 64 rows of the factor x 128 columns, four waves of 32 columns; both operands k-major (k: tokens, gathered by the order), through
// transposing reads.  Bound by reading x (dy) once.  blockIdx.x = unit, blockIdx.y = column tile of either gradient x rank tile.
__global__ __launch_bounds__(256, 2) void factor_gradient_kernel(FactorPair a) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int unit = blockIdx.x;
  if (unit >= a.unit_first[a.n]) return;
  const int rank_tile = blockIdx.y % a.rank_tiles, col = blockIdx.y / a.rank_tiles;
  const bool second = col >= a.f[0].n_tiles;
  const FactorArgs f = second ? a.f[1] : a.f[0];
  const int n0 = (second ? col - a.f[0].n_tiles : col) * kFactorCols, m0 = rank_tile * 64;
  const int id = __builtin_amdgcn_readfirstlane(a.unit_adapter[unit]);
  const int nth = unit - __builtin_amdgcn_readfirstlane(a.unit_first[id]);
  const bool alone = a.unit_first[id + 1] - a.unit_first[id] == 1;
  const int row0 = __builtin_amdgcn_readfirstlane(a.first[id]) + nth * a.chunk;
  const int left = __builtin_amdgcn_readfirstlane(a.first[id + 1]) - row0, rows = left < a.chunk ? left : a.chunk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int32_t* const tokens = (int32_t*)(smem + kFactorStages * kFactorStage);
  for (int i = threadIdx.x; i < rows; i += 256) tokens[i] = a.order[row0 + i];
  __syncthreads();
  const i32x4 wordsX = rsrc_words(f.x + n0, 0x80000000u - 1024), wordsH = rsrc_words(f.h + m0, 0x80000000u - 1024);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int steps = (rows + 63) / 64;
  auto issue = [&](int step, int stage) {
    const uint32_t lds = lds0 + stage * kFactorStage;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (wave * 4 + i) * 4 + (lane >> 4), at = step * 64 + r, c = ((lane & 15) ^ swz_factor(r)) * 8;
      const bool ok = at < rows && n0 + c < f.d;
      const int voff = (int)(((uint32_t)tokens[ok ? at : 0] * (uint32_t)f.d + (uint32_t)c) * 2u);
      load16_to_lds(wordsX, lds + (wave * 4 + i) * 1024, ok ? voff : (int)0x80000000, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = (wave * 2 + i) * 8 + (lane >> 3), at = step * 64 + r, c = ((lane & 7) ^ swz_narrow(r)) * 8;
      const bool ok = at < rows && m0 + c < a.rank;
      const int voff = (int)(((uint32_t)tokens[ok ? at : 0] * (uint32_t)a.rank + (uint32_t)c) * 2u);
      load16_to_lds(wordsH, lds + kFactorX + (wave * 2 + i) * 1024, ok ? voff : (int)0x80000000, 0);
    }
  };
  const int q = lane & 15, k_row = 8 * (lane >> 4) + (q >> 2);
  auto read_tr = [&](const char* p, int pitch) {
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + 4 * pitch));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // (k_row + 4 has the key of k_row: both take bits 0, 1 and 3)
  int xoff[2], hoff[4];
#pragma unroll
  for (int c = 0; c < 2; ++c)
    xoff[c] = k_row * 256 + ((q & 1) << 3) + (((((2 * wave + c) << 1) | ((q >> 1) & 1)) ^ swz_factor(k_row)) << 4);
#pragma unroll
  for (int m = 0; m < 4; ++m) hoff[m] = k_row * 128 + ((q & 1) << 3) + ((((m << 1) | ((q >> 1) & 1)) ^ swz_narrow(k_row)) << 4);
  f32x4 acc[2][4] = {};
#pragma unroll
  for (int s = 0; s < kFactorStages - 1; ++s) issue(s, s);
  int stage = 0;
  for (int kt = 0; kt < steps; ++kt) {
    constexpr int kAhead = (kFactorStages - 2) * 6;
    __builtin_amdgcn_s_waitcnt(0x0F70 | kAhead);
    __syncthreads();
    issue(kt + kFactorStages - 1, stage == 0 ? kFactorStages - 1 : stage - 1);
    const char* const st = smem + stage * kFactorStage;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 x[2], h[4];
#pragma unroll
      for (int c = 0; c < 2; ++c) x[c] = read_tr(st + xoff[c] + ks * 32 * 256, 256);
#pragma unroll
      for (int m = 0; m < 4; ++m) h[m] = read_tr(st + kFactorX + hoff[m] + ks * 32 * 128, 128);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[c][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[c], h[m], acc[c][m], 0, 0, 0);
    }
    stage = stage + 1 == kFactorStages ? 0 : stage + 1;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  constexpr int kPitch = kFactorCols + 4;
  float* const tile = (float*)smem;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int m = 0; m < 4; ++m) *(f32x4*)(tile + (16 * m + (lane & 15)) * kPitch + 32 * wave + 16 * c + 4 * (lane >> 4)) = acc[c][m];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = threadIdx.x + 256 * i, r = p >> 4, c = (p & 15) * 8;
    if (m0 + r >= a.rank || n0 + c >= f.d) continue;
    const f32x4 v0 = *(const f32x4*)(tile + r * kPitch + c), v1 = *(const f32x4*)(tile + r * kPitch + c + 4);
    if (alone) {
      *(u32x4_t*)(f.out + ((size_t)id * a.rank + m0 + r) * f.d + n0 + c) =
          u32x4_t{pack_bf16x2(v0[0], v0[1]), pack_bf16x2(v0[2], v0[3]), pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3])};
    } else {
      float* const to = f.part + ((size_t)unit * a.rank + m0 + r) * f.d + n0 + c;
      *(f32x4*)to = v0;
      *(f32x4*)(to + 4) = v1;
    }
  }
#endif
}
static_assert(64 * (kFactorCols + 4) * 4 <= kFactorStages * kFactorStage, "the tile reuses the stages");

// Adapters of several units: their sums in order.  blockIdx.x = adapter, blockIdx.y = which gradient; blockIdx.z strides over it.
__global__ __launch_bounds__(256) void join_factors_kernel(FactorPair a) {
  const int u0 = a.unit_first[blockIdx.x], u1 = a.unit_first[blockIdx.x + 1];
  if (u1 - u0 <= 1) return;
  const FactorArgs f = a.f[blockIdx.y];
  const size_t elems = (size_t)a.rank * f.d;
  for (size_t i = ((size_t)blockIdx.z * 256 + threadIdx.x) * 8; i < elems; i += (size_t)gridDim.z * 2048) {
    f32x4 v0 = {}, v1 = {};
    for (int u = u0; u < u1; ++u) {
      v0 += *(const f32x4*)(f.part + u * elems + i);
      v1 += *(const f32x4*)(f.part + u * elems + i + 4);
    }
    *(u32x4_t*)(f.out + blockIdx.x * elems + i) =
        u32x4_t{pack_bf16x2(v0[0], v0[1]), pack_bf16x2(v0[2], v0[3]), pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3])};
  }
}

}  // namespace
