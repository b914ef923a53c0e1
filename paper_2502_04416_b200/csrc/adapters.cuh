// Low-rank adapters of many requests beside a shared projection, and their gradients.
//
//   forward    z_t = A_a xd_t,  out_t = base_t + s_a B_a z_t             a: the adapter of row t, xd = x or its dropout
//   backward   e_t = s_a B_a^T g_t,  dx_t = dx_base_t + m_t (A_a^T e_t),  dA_a = sum e_t xd_t^T,  dB_a = sum s_a g_t z_t^T
//
// Both directions are the same two products around a narrow middle (the rank, 8 to 64): rows [d_k] -> [r] -> [d_n], with
// the weights of the second direction read in their other orientation.  One kernel does both products for a tile of rows
// of one adapter and never writes the middle to global memory unless it is wanted; a second kernel forms the two
// gradients of the weights, sums over the rows of an adapter.
//
// Bound: HBM (rows read once, outputs written once; 2 r flops an element).  The products here are warp-level MMAs on fragments
// that are loaded straight from global memory, 32 bytes a lane: no staging through shared memory, and a lane's bytes are
// elements that share blocks of the dropout generator, so the mask costs no exchange either.  Where ranks are high and batches
// long, weights and MMAs weigh more than the rows, and tiles of 128 rows on tcgen05 take over (adapters_umma.cuh).
#pragma once

#include "common.cuh"
#include "dropout.cuh"
#include "permute.cuh"
#include "router_cluster.cuh"
#include "router_mma.cuh"
#include "umma_gemm.cuh"

namespace cmoe {

constexpr int kAdMaxRank = 64;
constexpr int kAdMaxAdapters = 1024;
constexpr int kAdThreads = 256, kAdWarps = 8;
constexpr int kAdSmallRows = 256;      // rows whose tiles every cluster finds for itself
constexpr int kAdMaxRows = 1 << 30;

// ---------------------------------------------------------------------------------------------------------------------
// Tiles: up to M rows of one adapter.

struct AdTiles {
  const int32_t* row_adapter;    // null: every row takes adapter 0
  int planned;                   // the lists below are there
  const int32_t *tile_start;     // [n + 2] first tile of every adapter; group n: rows without an adapter
  const int32_t *tile_adapter;   // [tiles]
  const int32_t *row_list;       // [tiles * M] rows of the tiles, in order; -1 behind a group's last row
};

struct AdPlanOut { int32_t *tile_start, *tile_adapter, *row_list; };

__device__ __forceinline__ uint32_t cluster_ctas() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// The tiles of a batch, by one cluster of up to eight blocks: a stable counting sort of the rows by adapter (so sums over an
// adapter's rows have a fixed order).  A warp owns a run of rows; lanes with the same adapter find each other by ballots, so no
// atomics; blocks exchange their counts.  One block is bound by its instructions and by its stores to many lines (16384 rows of
// 16 adapters in random order: 20.6 us).
__global__ void __launch_bounds__(1024)
adapter_plan_kernel(const int32_t* row_adapter, int n_rows, int n, int m, const AdPlanOut o) {
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  rc_cluster_arrive();                       // this block has started
  grid_dep_wait();
  grid_dep_trigger();
  extern __shared__ int32_t sm[];
  const int groups = n + 1;
  int32_t* hist = sm;                        // [32][groups]
  int32_t* totals = hist + 32 * groups;      // [8][groups] rows of every block
  int32_t* count = totals + 8 * groups;      // [groups]
  int32_t* first = count + groups;           // [groups] place of this block's first row
  int32_t* tiles = first + groups;           // [groups]
  int32_t* start = tiles + groups;           // [groups + 1]
  int32_t* sums = start + groups + 1;        // [32]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned lt = (1u << lane) - 1u;
  const long long warps = 32LL * ctas, per = ((n_rows + warps - 1) / warps + 31) / 32 * 32;
  const long long lo = (long long)(rank * 32 + warp) * per, hi = min(lo + per, (long long)n_rows);
  for (int i = threadIdx.x; i < 32 * groups; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  int32_t* mine = hist + warp * groups;
  // lanes with the same group: a ballot a bit of its number (match.any takes a turn for every distinct one: 16384 rows of 16
  // adapters in random order, 22.8 us)
  const int bits = 32 - __clz(n);
  const auto same_group = [&](int g) {
    unsigned same = __ballot_sync(0xffffffffu, g >= 0);
    if (g < 0) same = ~same;
    for (int b = 0; b < bits; ++b) {
      const unsigned set = __ballot_sync(0xffffffffu, g >> b & 1);
      same &= g >> b & 1 ? set : ~set;
    }
    return same;
  };
  // the groups of 32 kBatch rows from r0 on, their loads in flight at once (-1 behind the warp's last row)
  constexpr int kBatch = 4;
  int v[kBatch];
  auto groups_of = [&](long long r0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const long long row = r0 + 32 * i + lane;
      v[i] = row < hi ? __ldcg(row_adapter + row) : -1;
      if (row < hi && (unsigned)v[i] >= (unsigned)n) v[i] = n;
    }
  };
  for (long long r0 = lo; r0 < hi; r0 += 32 * kBatch) {
    groups_of(r0);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (r0 + 32 * i >= hi) break;
      const unsigned same = same_group(v[i]);
      if (v[i] >= 0 && (same & lt) == 0) mine[v[i]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  for (int g = threadIdx.x; g < groups; g += blockDim.x) {
    int run = 0;
#pragma unroll 8
    for (int w = 0; w < 32; ++w) { const int c = hist[w * groups + g]; hist[w * groups + g] = run; run += c; }
    count[g] = run;
  }
  __syncthreads();
  rc_cluster_wait();                         // every peer has started
  for (int g = threadIdx.x; g < groups; g += blockDim.x)
    for (uint32_t c = 0; c < ctas; ++c) rc_push(rc_peer(totals + rank * groups + g, c), count[g]);
  rc_cluster_arrive();
  rc_cluster_wait();
  for (int g = threadIdx.x; g < groups; g += blockDim.x) {
    int all = 0, before = 0;
    for (uint32_t c = 0; c < ctas; ++c) { if (c == rank) before = all; all += totals[c * groups + g]; }
    count[g] = all;
    first[g] = before;
    tiles[g] = (all + m - 1) / m;
  }
  __syncthreads();
  block_scan_groups(tiles, start, groups, sums);
  if (rank == 0)
    for (int g = threadIdx.x; g <= groups; g += blockDim.x) o.tile_start[g] = start[g];
  for (long long r0 = lo; r0 < hi; r0 += 32 * kBatch) {
    if (hi - lo > 32 * kBatch) groups_of(r0);            // a warp's only batch is still there
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (r0 + 32 * i >= hi) break;
      const int g = v[i];
      const unsigned same = same_group(g);
      const int before = g >= 0 ? mine[g] : 0;
      __syncwarp();
      if (g >= 0) {
        o.row_list[(size_t)start[g] * m + first[g] + before + __popc(same & lt)] = (int32_t)(r0 + 32 * i + lane);
        if ((same & lt) == 0) mine[g] = before + __popc(same);
      }
      __syncwarp();
    }
  }
  const int n_tiles = start[groups];
  for (int t = rank * blockDim.x + threadIdx.x; t < n_tiles; t += ctas * blockDim.x) {
    int a = 0, b = groups;                               // start[a] <= t < start[b]
    while (b - a > 1) {
      const int c = (a + b) >> 1;
      if (start[c] <= t) a = c; else b = c;
    }
    o.tile_adapter[t] = a;
    for (int i = max(0, count[a] - (t - start[a]) * m); i < m; ++i) o.row_list[(size_t)t * m + i] = -1;
  }
}
inline size_t adapter_plan_smem(int n) { return (size_t)(44 * (n + 1) + 1 + 32) * sizeof(int32_t); }

// Rows of tile `tile` into rows[M] (-1: none); returns its adapter, n where its rows have none, or -1: nothing to do.
// Every thread of the block calls it, and every block of a cluster gets the same answer.
template <int M>
__device__ __forceinline__ int adapter_tile(const AdTiles& t, int n_rows, int n, int tile, int32_t* rows) {
  if (t.row_adapter == nullptr) {
    for (int i = threadIdx.x; i < M; i += kAdThreads) {
      const long long r = (long long)tile * M + i;
      rows[i] = r < n_rows ? (int32_t)r : -1;
    }
    __syncthreads();
    return 0;
  }
  if (t.planned) {
    if (tile >= __ldcg(t.tile_start + n + 1)) return -1;
    for (int i = threadIdx.x; i < M; i += kAdThreads) rows[i] = __ldcg(t.row_list + (size_t)tile * M + i);
    __syncthreads();
    return __ldcg(t.tile_adapter + tile);
  }
  // A row heads a tile if a multiple of M rows with its adapter come before it; tile t belongs to the t-th such row.
  static_assert(kAdSmallRows == kAdThreads, "one thread a row");
  __shared__ __align__(16) int32_t ids[kAdSmallRows];
  __shared__ uint32_t heads[kAdWarps];
  __shared__ int2 head;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t lt = (1u << lane) - 1u;
  int a = -2;
  if ((int)threadIdx.x < n_rows) {
    a = __ldcg(t.row_adapter + threadIdx.x);
    a = (unsigned)a < (unsigned)n ? a : n;
  }
  ids[threadIdx.x] = a;
  for (int i = threadIdx.x; i < M; i += kAdThreads) rows[i] = -1;
  __syncthreads();
  int rank = __popc(__match_any_sync(0xffffffffu, a) & lt);
  if (a >= 0)
    for (int i = 0; i < 32 * warp; i += 4) {
      const int4 v = *reinterpret_cast<const int4*>(ids + i);
      rank += (v.x == a) + (v.y == a) + (v.z == a) + (v.w == a);
    }
  const bool is_head = a >= 0 && rank % M == 0;
  const uint32_t vote = __ballot_sync(0xffffffffu, is_head);
  if (lane == 0) heads[warp] = vote;
  __syncthreads();
  int at = __popc(vote & lt), n_heads = 0;
  for (int w = 0; w < kAdWarps; ++w) {
    const int c = __popc(heads[w]);
    if (w < warp) at += c;
    n_heads += c;
  }
  if (tile >= n_heads) return -1;
  if (is_head && at == tile) head = make_int2(a, rank);
  __syncthreads();
  const int2 h = head;
  if (a == h.x && rank >= h.y && rank < h.y + M) rows[rank - h.y] = threadIdx.x;
  __syncthreads();
  return h.x;
}

// ---------------------------------------------------------------------------------------------------------------------

template <typename T> struct AdapterArgs {
  const T* x; long long ldx;             // [rows, d_k]
  const T *w1, *w2;                      // forward: A [n][r][d_k], B [n][d_n][r]; backward: B [n][d_k][r], A [n][r][d_n]
  const float* scale;                    // [n] or null: 1
  const T* base; long long ld_base;      // [rows, d_n] or null: 0
  T* out; long long ld_out;              // [rows, d_n]; null: not wanted
  float* z_out;                          // [rows, r] or null: the middle, unscaled (forward)
  const float* z_in;                     // backward: the forward's z, for the operand of dB
  void *u_e, *u_z;                       // backward: s e / (1 - p) and s z in the order of the tiles, or null
  int n_rows, n, r, d_k, d_n;
  int wide_x, wide_n;                    // rows of x and w1's, of base and out, on 32-byte boundaries and of whole 32-byte pieces
  AdTiles tiles;
  Drop drop;
};

// A 32-bit float as two bf16 whose sum has at least 15 of its significant bits, for twice the MMAs of a narrow product: the error, 2^-16
// of the value, is below a bf16 result's rounding unless the terms of a sum cancel to less than about 2^-7 of their size; it is stated with
// the calls.  Neither part is zero unless the value is, and both have its sign, so that a sum that meets an infinity on the
// other side takes no 0 * Inf from a part: the high part is the last step strictly below the value's magnitude, which leaves something
// for the low part.  Of an infinity the low part is one, and of a NaN.  (Values below 2^-103 may lose their low part to the end of the range.)
__device__ __forceinline__ void split_bf16(float v, uint16_t& hi, uint16_t& lo) {
  const uint32_t u = __float_as_uint(v);
  const uint32_t h = ((max(u & 0x7fffffffu, 1u) - 1u) & 0x7fff0000u) | (u & 0x80000000u);
  hi = (uint16_t)(h >> 16);
  lo = __bfloat16_as_ushort(__float2bfloat16_rn(v - __uint_as_float(h)));
}
// Transposes an 8 x 8 matrix of 16-bit elements held by the warp (lane 4 i + j: row i, columns 2 j and 2 j + 1).
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void push4(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t ld4(const void* p) {
  uint32_t r;
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(r) : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
  uint2 r;
  asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}

// Rows without an adapter: base goes to out, z is zero.  The blocks of a cluster share the columns.
template <int THREADS, typename T>
__device__ __forceinline__ void adapter_none(const AdapterArgs<T>& p, const int32_t* rows, int m, uint32_t rank, uint32_t ctas) {
  const bool copy = p.out && !(p.base == p.out && p.ld_base == p.ld_out);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bytes = p.d_n * (int)sizeof(T), pieces = bytes / 16;
  constexpr int kUnroll = 8;                             // loads in flight a lane
  for (int i = warp; i < m; i += THREADS / 32) {
    const int row = rows[i];
    if (row < 0) break;
    if (copy) {
      const uint4* from = reinterpret_cast<const uint4*>(p.base + (size_t)row * p.ld_base);
      uint4* to = reinterpret_cast<uint4*>(p.out + (size_t)row * p.ld_out);
      for (int c = (int)rank * 32 * kUnroll + lane; c < pieces; c += 32 * kUnroll * ctas) {
        uint4 v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) v[u] = p.base && c + 32 * u < pieces ? ld_dep16(from + c + 32 * u) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (c + 32 * u < pieces) to[c + 32 * u] = v[u];
      }
    }
    if (p.z_out && rank == 0)
      for (int k = lane; k < p.r; k += 32) p.z_out[(size_t)row * p.r + k] = 0.0f;
  }
}

// ---- bf16 -------------------------------------------------------------------------------------------------------------
// MT: 16-row MMA tiles of a row tile; RT: 8-wide tiles of the rank (padded); TRANS: backward.
//
// A lane of an 8 x 4 fragment loads 32 neighbouring bytes of its row: four lanes make whole 128-byte lines, and 32 bytes are
// the operands of four k steps (k inside a 64-wide block is permuted alike on both sides, which leaves the sums as they are)
// or eight tiles' results of one lane.  Loads that are 16 bytes wide, or go by way of shared memory, are bound by L1 instead of
// HBM (16384 rows x 4096, rank 16, rows in and out: 106 us through a ring of asynchronous copies, L1 76 % busy).  What is in
// flight is left to the number of resident warps and the tile's height.  At ranks above 16 the warps that share rows split the
// rank, 16 each.  Loads past the end of a row, a column or the rank read the last valid place instead: what they bring meets
// zeros in the other operand, or is not stored.
template <int MT, int RT, bool TRANS> struct AdapterShape {
  static constexpr int kM = 16 * MT, kR = 8 * RT;
  static constexpr int kSplit = RT <= 2 ? 1 : RT / 2, kRtw = RT / kSplit, kGroups = kAdWarps / kSplit;   // warps of a rank's share
  static constexpr int kQuads = MT * RT * 32;
  // elements between the middle's rows: no two of a fragment's lanes meet in a bank
  static constexpr int kStride = TRANS ? (RT == 1 ? 8 : kR + 8) : RT == 8 ? 96 : kR;
  static constexpr int kPart = kGroups / 2 * kQuads * 16, kRecv = kQuads * 16, kMid = 2 * kM * kStride * 2;
  static constexpr int bytes(int ctas) { return kPart + ctas * kRecv + kMid + kM * 4; }
  static constexpr int kMinBlocks = MT == 1 && RT <= 2 ? 3 : 2;
};

// 32 bytes: columns c .. c + 15 of a row of `width`; past its end, the last ones again.  wide: the row starts on a 32-byte
// boundary and is made of whole 32-byte pieces.
template <bool STREAM>
__device__ __forceinline__ void ld32(const bf16* row, int c, int width, bool wide, uint32_t (&r)[8]) {
  if (wide) {
    const bf16* p = row + min(c, width - 16);
    if (STREAM) ld256_stream(p, r);
    else
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p) : "memory");
  } else {
    const uint4 a = ld_dep16(row + min(c, width - 8)), b = ld_dep16(row + min(c + 8, width - 8));
    r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w; r[4] = b.x; r[5] = b.y; r[6] = b.z; r[7] = b.w;
  }
}
// Zeros in what of those columns lies past the end.
__device__ __forceinline__ void clear_tail(uint32_t (&r)[8], int c, int width) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + (i < 4 ? 0 : 8) >= width) r[i] = 0u;
}
__device__ __forceinline__ void drop16(uint32_t (&r)[8], const Drop& d, uint32_t row, uint32_t block) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 w = drop_draws(d, row, block + h);
    r[4 * h] = drop_pair(r[4 * h], w.x, d.thr16);
    r[4 * h + 1] = drop_pair(r[4 * h + 1], w.y, d.thr16);
    r[4 * h + 2] = drop_pair(r[4 * h + 2], w.z, d.thr16);
    r[4 * h + 3] = drop_pair(r[4 * h + 3], w.w, d.thr16);
  }
}
// Asks for `bytes` bytes from p on in L2; both are multiples of 16.
__device__ __forceinline__ void prefetch_l2(const void* p, int bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ const bf16* row_at(const bf16* m, uint32_t row, uint32_t pitch) {
  return reinterpret_cast<const bf16*>(reinterpret_cast<const char*>(m) + (uint64_t)row * pitch);
}

template <int MT, int RT, bool TRANS, bool DROP>
__global__ void __launch_bounds__(kAdThreads, AdapterShape<MT, RT, TRANS>::kMinBlocks)
adapter_kernel(const AdapterArgs<bf16> p) {
  using S = AdapterShape<MT, RT, TRANS>;
  constexpr int M = S::kM, kStride = S::kStride, kQuads = S::kQuads, kRtw = S::kRtw, kGroups = S::kGroups;
  extern __shared__ __align__(16) uint8_t smem[];
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  float4* part = reinterpret_cast<float4*>(smem);                              // [kGroups / 2][MT][RT][lane]
  float4* recv = part + kGroups / 2 * kQuads;                                  // [ctas][MT][RT][lane]
  uint16_t* mid = reinterpret_cast<uint16_t*>(recv + ctas * kQuads);           // [high, low][M][kStride]
  int32_t* rows = reinterpret_cast<int32_t*>(mid + 2 * M * kStride);
  rc_cluster_arrive();                                                         // this block has started
  grid_dep_wait();
  grid_dep_trigger();
  const int tile = blockIdx.x / ctas;
  const int a = adapter_tile<M>(p.tiles, p.n_rows, p.n, tile, rows);
  if (a < 0 || a == p.n) {                                                     // the whole cluster leaves
    if (a == p.n) adapter_none<kAdThreads>(p, rows, M, rank, ctas);
    rc_cluster_wait();
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint32_t row_of[MT][2];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = rows[mt * 16 + 8 * h + g];
      row_of[mt][h] = row < 0 ? rows[0] : row;           // a row's sums are its own: rows past the end repeat the first
    }
  const uint32_t x_pitch = (uint32_t)p.ldx * 2, base_pitch = (uint32_t)p.ld_base * 2, out_pitch = (uint32_t)p.ld_out * 2;
  const bf16* w2 = p.w2 + (size_t)a * p.r * p.d_n;
  const int nb0 = (int)rank * kAdWarps + warp, n_cols = p.out ? p.d_n : 0;
  const int kg = warp / S::kSplit, rt0 = (warp % S::kSplit) * kRtw;
  const bf16* w1 = p.w1 + (size_t)a * p.r * p.d_k;
  if (MT == 1) {
    // Few rows: what each warp will read comes from HBM, and all of it is asked for now, in L2: blocks of [width][r] weights as
    // they lie, the other weights' and the rows' 128-byte lines one a lane.
    const auto line = [](const bf16* row, int c, int width) {
      if (c < width) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + c));
    };
    const int my_row = rows[lane & 15];
    for (int kb = (int)rank * kGroups + kg; kb * 64 < p.d_k; kb += (int)ctas * kGroups) {
      const int c = kb * 64;
      if (TRANS && lane == 0) prefetch_l2(w1 + (size_t)c * p.r, min(64, p.d_k - c) * p.r * 2);
      if (lane < 16) {
        if (my_row >= 0) line(row_at(p.x, my_row, x_pitch), c, p.d_k);
      } else if (!TRANS && rt0 * 8 + lane - 16 < p.r) {
        line(w1 + (size_t)(rt0 * 8 + lane - 16) * p.d_k, c, p.d_k);
      }
    }
    for (int nb = nb0; nb * 64 < n_cols; nb += (int)ctas * kAdWarps) {
      const int c = nb * 64;
      if (!TRANS && lane == 0) prefetch_l2(w2 + (size_t)c * p.r, min(64, n_cols - c) * p.r * 2);
      if (p.base && lane < 16 && my_row >= 0) line(row_at(p.base, my_row, base_pitch), c, n_cols);
      if (TRANS)
        for (int n = lane; n < p.r; n += 32) line(w2 + (size_t)n * p.d_n, c, n_cols);
    }
  }

  // ---- first product: [M, d_k] x [d_k, r], 64-wide blocks of d_k dealt to the warps of the cluster
  float acc[MT][kRtw][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int rt = 0; rt < kRtw; ++rt)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[mt][rt][i] = 0.0f;
  uint32_t x[MT][2][8];
#pragma unroll 1
  for (int kb = (int)rank * kGroups + kg; kb * 64 < p.d_k; kb += (int)ctas * kGroups) {
    const int k = kb * 64 + 16 * q;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) ld32<S::kSplit == 1>(row_at(p.x, row_of[mt][h], x_pitch), k, p.d_k, p.wide_x, x[mt][h]);
    uint32_t w[kRtw][8];
    if (!TRANS) {
#pragma unroll
      for (int rt = 0; rt < kRtw; ++rt)
        ld32<false>(w1 + (size_t)min((rt0 + rt) * 8 + g, p.r - 1) * p.d_k, k, p.d_k, p.wide_x, w[rt]);
    } else {
      // rows of [d_k][r]: matrix i holds k = 16 (g / 2) + 2 i + g % 2, so that transposed it holds a lane's k = 16 q + 2 i, + 1
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bf16* wr = w1 + (size_t)min(kb * 64 + 16 * (g >> 1) + 2 * i + (g & 1), p.d_k - 1) * p.r;
        if (kRtw == 1) {
          w[0][i] = ld4(wr + 2 * q);
        } else {
          const uint2 v = ld8(wr + min(rt0 * 8 + 4 * q, p.r - 4));
          w[0][i] = v.x; w[kRtw - 1][i] = v.y;
        }
      }
#pragma unroll
      for (int rt = 0; rt < kRtw; ++rt)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[rt][i] = transpose8(w[rt][i]);
    }
    if (kb * 64 + 64 > p.d_k)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) clear_tail(x[mt][h], k, p.d_k);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (DROP && !TRANS)
#pragma unroll
        for (int h = 0; h < 2; ++h) drop16(x[mt][h], p.drop, row_of[mt][h], k >> 3);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int rt = 0; rt < kRtw; ++rt)
          mma_bf16_16816(acc[mt][rt], x[mt][0][2 * s], x[mt][1][2 * s], x[mt][0][2 * s + 1], x[mt][1][2 * s + 1], w[rt][2 * s], w[rt][2 * s + 1]);
    }
  }

  // ---- second product's operands, 64 columns a warp at a time
  constexpr bool kEarly = MT == 1;                       // few rows: both halves' weights at once, the first block's before the sums
  uint32_t base[MT][2][8], wh[kEarly ? 2 : 1][4][RT];
  auto load_base = [&](int nb) {
    const int c = nb * 64 + 16 * q;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (p.base) {
          ld32<true>(row_at(p.base, row_of[mt][h], base_pitch), c, p.d_n, p.wide_n, base[mt][h]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) base[mt][h][i] = 0u;
        }
      }
  };
  // half 0: the lanes' columns 16 q .. 16 q + 7 (tiles 0 .. 3), half 1: the other eight (4 .. 7)
  auto load_w = [&](int nb, int half, uint32_t (&w)[4][RT]) {
    if (!TRANS) {
      // tile j's column g stands for column 16 (g / 2) + 2 j + g % 2, so that a lane's results are neighbours
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16* wr = w2 + (size_t)min(nb * 64 + 16 * (g >> 1) + 8 * half + 2 * j + (g & 1), p.d_n - 1) * p.r;
        if (RT == 1) {
          w[j][0] = ld4(wr + 2 * q);
        } else if (RT == 2) {
          const uint2 v = ld8(wr + 4 * q);
          w[j][0] = v.x; w[j][RT - 1] = v.y;
        } else {
#pragma unroll
          for (int h = 0; h < RT / 4; ++h) {
            const uint4 v = ld_dep16(wr + min(32 * h + 8 * q, p.r - 8));
            w[j][(4 * h) % RT] = v.x; w[j][(4 * h + 1) % RT] = v.y; w[j][(4 * h + 2) % RT] = v.z; w[j][(4 * h + 3) % RT] = v.w;
          }
        }
      }
    } else {
      const int c = min(nb * 64 + 16 * q + 8 * half, p.d_n - 8);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const uint4 v = ld_dep16(w2 + (size_t)min(rt * 8 + g, p.r - 1) * p.d_n + c);
        w[0][rt] = v.x; w[1][rt] = v.y; w[2][rt] = v.z; w[3][rt] = v.w;
      }
    }
  };
  auto load_early = [&](int nb) { load_base(nb); load_w(nb, 0, wh[0]); load_w(nb, 1, wh[kEarly ? 1 : 0]); };
  if (kEarly && nb0 * 64 < n_cols) load_early(nb0);

  // ---- the sums of the block's warps, then of the cluster's blocks, each in a fixed order
  auto quad = [&](int mt, int rt) { return (mt * RT + rt0 + rt) * 32 + lane; };
  if (kg >= kGroups / 2)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int rt = 0; rt < kRtw; ++rt)
        part[(kg - kGroups / 2) * kQuads + quad(mt, rt)] = make_float4(acc[mt][rt][0], acc[mt][rt][1], acc[mt][rt][2], acc[mt][rt][3]);
  __syncthreads();
  if (kg < kGroups / 2)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int rt = 0; rt < kRtw; ++rt) {
        float4& s = part[kg * kQuads + quad(mt, rt)];
        s = make_float4(s.x + acc[mt][rt][0], s.y + acc[mt][rt][1], s.z + acc[mt][rt][2], s.w + acc[mt][rt][3]);
      }
  __syncthreads();
  rc_cluster_wait();                                                           // every peer has started
#pragma unroll 1
  for (int i = threadIdx.x; i < kQuads; i += kAdThreads) {
    float4 s = part[i];
#pragma unroll
    for (int w = 1; w < kGroups / 2; ++w) {
      const float4 v = part[w * kQuads + i];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
#pragma unroll 1
    for (uint32_t c = 0; c < ctas; ++c) push4(rc_peer(recv + rank * kQuads + i, c), s);
  }
  rc_cluster_arrive();
  rc_cluster_wait();
  const float scale = p.scale ? __ldcg(p.scale + a) : 1.0f;
  const float drop_inv = DROP ? p.drop.inv : 1.0f;
#pragma unroll 1
  for (int i = threadIdx.x; i < kQuads; i += kAdThreads) {
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
    for (uint32_t c = 0; c < ctas; ++c) {
      const float4 v = recv[c * kQuads + i];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const int l = i & 31, rt = (i >> 5) % RT, mt = (i >> 5) / RT, lg = l >> 2, lq = l & 3;
    // rank of the lane's first column
    const int n0 = TRANS && RT >= 2 ? (rt & ~1) * 8 + 4 * lq + 2 * (rt & 1) : rt * 8 + 2 * lq;
    const float v[2][2] = {{s.x * drop_inv, s.y * drop_inv}, {s.z * drop_inv, s.w * drop_inv}};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int m = mt * 16 + 8 * h + lg, row = rows[m];
      if (p.z_out && row >= 0 && n0 < p.r && (uint32_t)(i >> 5) % ctas == rank)
        *reinterpret_cast<float2*>(p.z_out + (size_t)row * p.r + n0) = make_float2(v[h][0], v[h][1]);
      uint16_t hi[2], lo[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) split_bf16(row >= 0 && n0 < p.r ? v[h][e] * scale : 0.0f, hi[e], lo[e]);
      *reinterpret_cast<uint32_t*>(mid + m * kStride + n0) = hi[0] | (uint32_t)hi[1] << 16;
      *reinterpret_cast<uint32_t*>(mid + (M + m) * kStride + n0) = lo[0] | (uint32_t)lo[1] << 16;
    }
  }
  __syncthreads();

  // ---- backward: the middle and the forward's as MMA fragments for the sums over rows (16 rows x 8 ranks a warp)
  if (TRANS && p.u_e) {
    uint4* ue = reinterpret_cast<uint4*>(p.u_e) + (size_t)tile * kQuads;
    uint4* uz = reinterpret_cast<uint4*>(p.u_z) + (size_t)tile * kQuads;
#pragma unroll 1
    for (int i = threadIdx.x; i < kQuads; i += kAdThreads) {
      if ((uint32_t)(i >> 5) % ctas != rank) continue;
      const int l = i & 31, rt = (i >> 5) % RT, mt = (i >> 5) / RT, nn = rt * 8 + (l >> 2), t0 = mt * 16 + 2 * (l & 3);
      uint16_t eh[4], el[4], zh[4], zl[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = t0 + (j & 1) + 8 * (j >> 1), row = rows[m];
        eh[j] = mid[m * kStride + nn];
        el[j] = mid[(M + m) * kStride + nn];
        split_bf16(row >= 0 && nn < p.r ? __ldcg(p.z_in + (size_t)row * p.r + nn) * scale : 0.0f, zh[j], zl[j]);
      }
      ue[i] = make_uint4(eh[0] | (uint32_t)eh[1] << 16, eh[2] | (uint32_t)eh[3] << 16, el[0] | (uint32_t)el[1] << 16, el[2] | (uint32_t)el[3] << 16);
      uz[i] = make_uint4(zh[0] | (uint32_t)zh[1] << 16, zh[2] | (uint32_t)zh[3] << 16, zl[0] | (uint32_t)zl[1] << 16, zl[2] | (uint32_t)zl[3] << 16);
    }
  }

  // ---- second product: [M, r] x [r, d_n] on top of base
#pragma unroll 1
  for (int nb = nb0; nb * 64 < n_cols; nb += (int)ctas * kAdWarps) {
    const int c = nb * 64 + 16 * q;
    if (!kEarly) load_base(nb);
    else if (nb != nb0) load_early(nb);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t (&w)[4][RT] = wh[kEarly ? half : 0];
      if (!kEarly) load_w(nb, half, w);
      if (TRANS) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) w[j][rt] = transpose8(w[j][rt]);
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float o[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t b = base[mt][h][4 * half + j];
            o[j][2 * h] = DROP && TRANS ? 0.0f : __uint_as_float(b << 16);
            o[j][2 * h + 1] = DROP && TRANS ? 0.0f : __uint_as_float(b & 0xffff0000u);
          }
        const uint16_t* m0 = mid + (mt * 16 + g) * kStride;
        const uint16_t* m1 = m0 + 8 * kStride;
        if (RT == 1) {                               // one MMA: k 0 .. 7 the high part, 8 .. 15 the low part
          const uint32_t a0 = *reinterpret_cast<const uint32_t*>(m0 + 2 * q), a1 = *reinterpret_cast<const uint32_t*>(m1 + 2 * q);
          const uint32_t a2 = *reinterpret_cast<const uint32_t*>(m0 + M * kStride + 2 * q), a3 = *reinterpret_cast<const uint32_t*>(m1 + M * kStride + 2 * q);
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_bf16_16816(o[j], a0, a1, a2, a3, w[j][0], w[j][0]);
        } else {
#pragma unroll
          for (int s = 0; s < RT / 2; ++s)
#pragma unroll
            for (int lo = 1; lo >= 0; --lo) {
              // k of step s: ranks 16 s .. 16 s + 15 as they lie (TRANS), else a lane's own four neighbours
              uint2 u0, u1;
              if (TRANS) {
                const uint16_t *s0 = m0 + lo * M * kStride + 16 * s + 2 * q, *s1 = m1 + lo * M * kStride + 16 * s + 2 * q;
                u0 = make_uint2(*reinterpret_cast<const uint32_t*>(s0), *reinterpret_cast<const uint32_t*>(s0 + 8));
                u1 = make_uint2(*reinterpret_cast<const uint32_t*>(s1), *reinterpret_cast<const uint32_t*>(s1 + 8));
              } else {
                const int at = lo * M * kStride + (RT == 2 ? 4 * q : (s >> 1) * 32 + 8 * q + 4 * (s & 1));
                u0 = *reinterpret_cast<const uint2*>(m0 + at);
                u1 = *reinterpret_cast<const uint2*>(m1 + at);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) mma_bf16_16816(o[j], u0.x, u1.x, u0.y, u1.y, w[j][(2 * s) % RT], w[j][(2 * s + 1) % RT]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) { v[2 * j] = o[j][2 * h]; v[2 * j + 1] = o[j][2 * h + 1]; }
          if (DROP && TRANS) {
            drop8(v, drop_draws(p.drop, row_of[mt][h], (c >> 3) + half), p.drop.thr16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t b = base[mt][h][4 * half + j];
              v[2 * j] += __uint_as_float(b << 16);
              v[2 * j + 1] += __uint_as_float(b & 0xffff0000u);
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) base[mt][h][4 * half + j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t (&b)[8] = base[mt][h];
        bf16* o = const_cast<bf16*>(row_at(p.out, row_of[mt][h], out_pitch)) + c;
        if (rows[mt * 16 + 8 * h + g] < 0 || c >= p.d_n) continue;
        if (p.wide_n) {
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(o), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]),
                       "r"(b[4]), "r"(b[5]), "r"(b[6]), "r"(b[7]) : "memory");
        } else {
          *reinterpret_cast<uint4*>(o) = make_uint4(b[0], b[1], b[2], b[3]);
          if (c + 8 < p.d_n) *reinterpret_cast<uint4*>(o + 8) = make_uint4(b[4], b[5], b[6], b[7]);
        }
      }
  }
}

// ---- the gradients of the weights, bf16 ---------------------------------------------------------------------------------
// G[c][k] = sum over the adapter's rows t of V[t][c] U[t][k]: V = x under its mask with U = s e / (1 - p) for dA, V = g with
// U = s z for dB.  A block owns 256 columns; four warps take 64 of them each, for the first and the second half of a stage's
// 64 rows.  Two more warps keep a ring of stages full: a bulk copy a row (rows of one adapter lie anywhere), one a lane, and
// one for the rows' fragments of U, which the kernel above wrote as the MMA wants them.  The columns become the MMA's rows by
// transposing reads of shared memory, whose rows are 16 bytes apart modulo 128, so that eight of them meet in no bank.
// The blocks of a cluster split the rows further and add their sums through each other's shared memory, in rank order.
// Bound: HBM, and at ranks above 32 the MMAs, twice two for every operand pair since U comes in two parts.  Rows by loads into
// registers had a third of the bytes in flight: 16384 rows x 4096 + 4096, rank 16, 80 us.
struct OuterSide {
  const void* v; long long ldv;
  const void* u;
  void* g;
  int d;
};
struct OuterArgs {
  OuterSide side[2];           // 0: dA [n][r][d], 1: dB [n][d][r]
  int slices[2];               // column slices of either side
  int n_rows, n, r, m;         // m: rows of a tile
  AdTiles tiles;
  Drop drop;
};
// Slices of the two sides take turns (the masks make one side the slower), the longer side's rest follows.
__device__ __forceinline__ void outer_slice(const OuterArgs& p, int i, int& side, int& slice) {
  const int both = 2 * min(p.slices[0], p.slices[1]);
  if (i < both) {
    side = i & 1;
    slice = i >> 1;
  } else {
    side = p.slices[0] > p.slices[1] ? 0 : 1;
    slice = i - both / 2;
  }
}

// Code of a wait for a copy that ran out in a kernel of this file, until cmoe_adapter_status takes it.
static __device__ int32_t g_adapter_error;
// A row of zeros for the places behind a group's last row.
static __device__ __align__(128) uint32_t g_adapter_zeros[128];

constexpr int kOutColWarps = 4, kOutRowWarps = 2, kOutWidth = 64 * kOutColWarps, kOutStageRows = 64;
constexpr int kOutCopyWarps = 2, kOutThreads = 32 * (kOutColWarps * kOutRowWarps + kOutCopyWarps);
constexpr int kOutPitch = kOutWidth * 2 + 16;
static_assert(kOutStageRows == 32 * kOutCopyWarps && kOutStageRows == 32 * kOutRowWarps, "a copying lane a row, two steps of 16 a warp");

template <int RT> struct OuterShape {
  static constexpr int kQuads = kOutColWarps * 4 * RT * 32;
  static constexpr int kV = kOutStageRows * kOutPitch, kU = kOutStageRows / 16 * RT * 512, kStage = kV + kU;
  static constexpr int kBlocks = RT <= 2 ? 2 : 1, kDepth = RT <= 2 ? 3 : 4;
  static constexpr int kSmem = kDepth * kStage;            // afterwards: the second half's sums, and those of the peers
  static_assert(kSmem >= 2 * kQuads * 16 && kBlocks * (kSmem + 2048) <= 227 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <int RT, bool DROP>
__global__ void __launch_bounds__(kOutThreads, OuterShape<RT>::kBlocks)
adapter_outer_kernel(const OuterArgs p) {
  using S = OuterShape<RT>;
  constexpr int kQuads = S::kQuads, kDepth = S::kDepth;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[2 * kDepth];       // full, empty
  __shared__ int32_t stage_rows[kDepth][kOutStageRows];    // the rows of a stage, for their masks
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kDepth;
  if (threadIdx.x == 0) {
    abort_word = 0;
    for (int i = 0; i < kDepth; ++i) { mbar_init(full0 + 8 * i, kOutCopyWarps); mbar_init(empty0 + 8 * i, kOutColWarps * kOutRowWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  grid_dep_wait();
  grid_dep_trigger();
  int side, slice;
  outer_slice(p, blockIdx.x, side, slice);
  const int a = blockIdx.y;
  const OuterSide sd = p.side[side];
  long long lo = 0, hi = p.n_rows;                         // places of the adapter's rows in the order of the tiles
  if (p.tiles.row_adapter) {
    lo = (long long)__ldcg(p.tiles.tile_start + a) * p.m;
    hi = (long long)__ldcg(p.tiles.tile_start + a + 1) * p.m;
  } else if (a > 0) {
    hi = 0;
  }
  const int c_lo = slice * kOutWidth, width = min(kOutWidth, sd.d - c_lo);
  const int n_stages = hi > lo ? (int)((hi - lo + kOutStageRows - 1) / kOutStageRows) : 0;
  const int mine = n_stages > (int)rank ? (n_stages - (int)rank + (int)ctas - 1) / (int)ctas : 0;     // stages rank, rank + ctas, ..
  __syncthreads();
  const bool drop = DROP && side == 0;
  float acc[4][RT][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][rt][e] = 0.0f;
  const int cw = warp % kOutColWarps, rw = warp / kOutColWarps;

  if (warp >= kOutColWarps * kOutRowWarps) {
    // ---- copies: one row a lane; the first warp's first lane also copies U
    const int half = warp - kOutColWarps * kOutRowWarps, at = 32 * half + lane;
    const uint32_t v_pitch = (uint32_t)sd.ldv * 2;
    auto row_of = [&](int n) {
      const long long pos = lo + ((long long)n * ctas + rank) * kOutStageRows + at;
      return n >= mine || pos >= hi ? -1 : p.tiles.row_adapter ? __ldcg(p.tiles.row_list + pos) : (int)pos;
    };
    int row = row_of(0), n = 0;
    for (; n < mine; ++n) {
      const int s = n % kDepth, use = n / kDepth, next = row_of(n + 1);
      if (use > 0 && !mbar_wait_warp(empty0 + 8 * s, (use - 1) & 1, abort_flag, &g_adapter_error, kErrWaitEmpty)) break;
      const uint32_t dst = smem_u32(smem) + s * S::kStage, bar = full0 + 8 * s;
      // 16-row tiles of the stage that U has: the last stage may end early
      const long long t0 = (lo + ((long long)n * ctas + rank) * kOutStageRows) / 16;
      const int u_tiles = min(kOutStageRows / 16, (int)((hi + 15) / 16 - t0));
      stage_rows[s][at] = row;
      __syncwarp();
      if (elect_one()) mbar_expect_tx(bar, 32 * width * 2 + (half == 0 ? u_tiles * RT * 512 : 0));
      __syncwarp();
      const void* src = row < 0 ? (const void*)g_adapter_zeros : row_at((const bf16*)sd.v, row, v_pitch) + c_lo;
      bulk_copy(dst + at * kOutPitch, src, width * 2, bar);
      if (half == 0 && elect_one()) bulk_copy(dst + S::kV, (const uint4*)sd.u + t0 * RT * 32, u_tiles * RT * 512, bar);
      row = next;
    }
    // What is on its way lands before the ring becomes the sums' memory and before the block ends, also where a wait ran out, here or
    // in a warp of the products (otherwise those have waited for it all).
    for (int i = max(0, n - kDepth); i < n; ++i) {
      const long long t = clock64();
      while (!mbar_try_wait(full0 + 8 * (i % kDepth), (i / kDepth) & 1) && clock64() - t < kUmmaWaitCycles) {}
    }
  } else {
    // ---- products: two steps of 16 rows a stage
    for (int n = 0; n < mine; ++n) {
      const int s = n % kDepth, use = n / kDepth;
      if (!mbar_wait_warp(full0 + 8 * s, use & 1, abort_flag, &g_adapter_error, kErrWaitFull)) break;
      const uint32_t stage = smem_u32(smem) + s * S::kStage;
      const long long t0 = (lo + ((long long)n * ctas + rank) * kOutStageRows) / 16;
      const int u_tiles = min(kOutStageRows / 16, (int)((hi + 15) / 16 - t0));
#pragma unroll 1
      for (int k = 0; k < 2; ++k) {
        const int tile = 2 * rw + k;
        if (tile >= u_tiles || cw * 64 >= width) break;
        const uint32_t v = stage + tile * 16 * kOutPitch + cw * 128;
        if (drop) {                                        // the warp's 16 x 64 elements, 16 bytes a lane at a time
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * i + (lane >> 3), at = v + r * kOutPitch + (lane & 7) * 16;
            sts16(at, drop8(lds16(at), drop_draws(p.drop, stage_rows[s][tile * 16 + r], (c_lo >> 3) + cw * 8 + (lane & 7)), p.drop.thr16));
          }
          __syncwarp();
        }
        uint4 u[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) u[rt] = lds16(stage + S::kV + (tile * RT + rt) * 512 + lane * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x[4];
          ldsm4_t(v + ((lane & 7) + 8 * (lane >> 4)) * kOutPitch + (16 * i + 8 * ((lane >> 3) & 1)) * 2, x);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) mma_bf16_16816(acc[i][rt], x[0], x[1], x[2], x[3], u[rt].z, u[rt].w);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) mma_bf16_16816(acc[i][rt], x[0], x[1], x[2], x[3], u[rt].x, u[rt].y);
        }
      }
      if (drop) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the stage was written, and is copied over next
      __syncwarp();
      if (elect_one()) mbar_arrive(empty0 + 8 * s);
    }
  }

  // ---- the two halves of the rows, then the blocks of the cluster; the ring's memory is free
  float4* part = reinterpret_cast<float4*>(smem);
  float4* recv = part + kQuads;                            // [ctas][kQuads / ctas]
  auto quad = [&](int i, int rt) { return ((cw * 4 + i) * RT + rt) * 32 + lane; };
  __syncthreads();
  if (rw == 1)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) part[quad(i, rt)] = make_float4(acc[i][rt][0], acc[i][rt][1], acc[i][rt][2], acc[i][rt][3]);
  rc_cluster_arrive();                                     // this block no longer copies into its ring
  __syncthreads();
  rc_cluster_wait();
  const int own = kQuads / (int)ctas;                      // quads that a block finishes
  if (rw == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int k = quad(i, rt);
        const float4 s = part[k];
        push4(rc_peer(recv + (int)rank * own + k % own, k / own),
              make_float4(s.x + acc[i][rt][0], s.y + acc[i][rt][1], s.z + acc[i][rt][2], s.w + acc[i][rt][3]));
      }
  rc_cluster_arrive();
  rc_cluster_wait();
  bf16* out = (bf16*)sd.g + (size_t)a * p.r * sd.d;
  for (int i = threadIdx.x; i < own; i += kOutThreads) {
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t k = 0; k < ctas; ++k) {
      const float4 w = recv[k * own + i];
      s.x += w.x; s.y += w.y; s.z += w.z; s.w += w.w;
    }
    const int k = (int)rank * own + i, l = k & 31, rt = (k >> 5) % RT, mi = (k >> 5) / RT;   // mi: column warp, tile
    const int n0 = rt * 8 + 2 * (l & 3);
    if (n0 >= p.r) continue;
    const float val[2][2] = {{s.x, s.y}, {s.z, s.w}};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = c_lo + 16 * mi + 8 * h + (l >> 2);
      if (col >= sd.d) continue;
      if (side == 0) {
        out[(size_t)n0 * sd.d + col] = __float2bfloat16_rn(val[h][0]);
        out[(size_t)(n0 + 1) * sd.d + col] = __float2bfloat16_rn(val[h][1]);
      } else {
        *reinterpret_cast<uint32_t*>(out + (size_t)col * p.r + n0) = pack_bf16x2(val[h][0], val[h][1]);
      }
    }
  }
}

// ---- fp32 -------------------------------------------------------------------------------------------------------------
// The same tiles and exchange on the CUDA cores, with fused multiply-adds in full 32 bits.  A lane holds rows g, g + 8, ..
// of the tile and eight neighbouring k (first product) or columns (second product); ranks go by in chunks of 16.
constexpr int kSimtM = 32, kSimtRc = 16, kSimtBatch = 2;
struct AdapterSimtSmem {
  static constexpr int kStride = kAdMaxRank + 4;
  static constexpr int bytes(int ctas) {
    return (kAdWarps * kSimtM * kSimtRc + kSimtM * kAdMaxRank + ctas * kSimtM * kAdMaxRank + kSimtM * kStride) * 4 + kSimtM * 4;
  }
};

template <bool TRANS, bool DROP>
__global__ void __launch_bounds__(kAdThreads, 2)
adapter_simt_kernel(const AdapterArgs<float> p) {
  constexpr int M = kSimtM, kStride = AdapterSimtSmem::kStride;
  extern __shared__ __align__(16) uint8_t smem[];
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  float* part = reinterpret_cast<float*>(smem);                      // [warp][M][kSimtRc]
  float* zpart = part + kAdWarps * M * kSimtRc;                      // [M][kAdMaxRank]
  float* recv = zpart + M * kAdMaxRank;                              // [ctas][M][kAdMaxRank]
  float* mid = recv + ctas * M * kAdMaxRank;                         // [M][kStride]
  int32_t* rows = reinterpret_cast<int32_t*>(mid + M * kStride);
  rc_cluster_arrive();
  grid_dep_wait();
  grid_dep_trigger();
  const int tile = blockIdx.x / ctas;
  const int a = adapter_tile<M>(p.tiles, p.n_rows, p.n, tile, rows);
  if (a < 0 || a == p.n) {
    if (a == p.n) adapter_none<kAdThreads>(p, rows, M, rank, ctas);
    rc_cluster_wait();
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int wi = (int)rank * kAdWarps + warp, nw = (int)ctas * kAdWarps;
  int row_of[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) row_of[m] = rows[8 * m + g] < 0 ? rows[0] : rows[8 * m + g];
  const float* w1 = p.w1 + (size_t)a * p.r * p.d_k;
  const int kb_end = (p.d_k + 31) >> 5;
#pragma unroll 1
  for (int rc = 0; rc < p.r; rc += kSimtRc) {
    float acc[4][kSimtRc];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int j = 0; j < kSimtRc; ++j) acc[m][j] = 0.0f;
#pragma unroll 1
    for (int kb = wi; kb < kb_end; kb += nw) {
      const int k = kb * 32 + 8 * q;
      if (k < p.d_k) {                                               // d_k is a multiple of 8
        float x[4][8];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          load8(p.x + (size_t)row_of[m] * p.ldx + k, x[m]);
          if (DROP && !TRANS) drop8(x[m], drop_draws(p.drop, row_of[m], k >> 3), p.drop.thr16);
        }
        if (!TRANS) {
          // ranks come in eights; a few at a time, so that their loads are in flight together
#pragma unroll
          for (int h = 0; h < kSimtRc / 8; ++h)
            if (rc + 8 * h < p.r) {
#pragma unroll
              for (int j0 = 8 * h; j0 < 8 * h + 8; j0 += kSimtBatch) {
                float w[kSimtBatch][8];
#pragma unroll
                for (int j = 0; j < kSimtBatch; ++j) load8(w1 + (size_t)(rc + j0 + j) * p.d_k + k, w[j]);
#pragma unroll
                for (int j = 0; j < kSimtBatch; ++j)
#pragma unroll
                  for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[m][j0 + j] = fmaf(x[m][i], w[j][i], acc[m][j0 + j]);
              }
            }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int h = 0; h < kSimtRc / 8; ++h)
              if (rc + 8 * h < p.r) {
                float w[8];
                load8(w1 + (size_t)(k + i) * p.r + rc + 8 * h, w);
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                  for (int j = 0; j < 8; ++j) acc[m][8 * h + j] = fmaf(x[m][i], w[j], acc[m][8 * h + j]);
              }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int j = 0; j < kSimtRc; ++j) {
        float s = acc[m][j];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        if ((j >> 2) == q) part[(warp * M + 8 * m + g) * kSimtRc + j] = s;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < M * kSimtRc; i += kAdThreads) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kAdWarps; ++w) s += part[w * M * kSimtRc + i];
      zpart[(i / kSimtRc) * kAdMaxRank + rc + i % kSimtRc] = s;
    }
    __syncthreads();
  }
  rc_cluster_wait();
  for (int i = threadIdx.x; i < M * (p.r / 4); i += kAdThreads) {
    const int m = i / (p.r / 4), c = 4 * (i % (p.r / 4));
    const float4 v = *reinterpret_cast<const float4*>(zpart + m * kAdMaxRank + c);
    for (uint32_t k = 0; k < ctas; ++k) push4(rc_peer(recv + (rank * M + m) * kAdMaxRank + c, k), v);
  }
  rc_cluster_arrive();
  rc_cluster_wait();
  const float scale = p.scale ? __ldcg(p.scale + a) : 1.0f;
  const float drop_inv = DROP ? p.drop.inv : 1.0f;
  for (int i = threadIdx.x; i < M * p.r; i += kAdThreads) {
    const int m = i / p.r, c = i - m * p.r, row = rows[m];
    float s = 0.0f;
    for (uint32_t k = 0; k < ctas; ++k) s += recv[(k * M + m) * kAdMaxRank + c];
    s *= drop_inv;
    const bool mine = (uint32_t)m % ctas == rank;
    if (p.z_out && row >= 0 && mine) p.z_out[(size_t)row * p.r + c] = s;
    s = row >= 0 ? s * scale : 0.0f;
    mid[m * kStride + c] = s;
    if (TRANS && p.u_e && mine) {
      const size_t at = ((size_t)tile * M + m) * p.r + c;
      reinterpret_cast<float*>(p.u_e)[at] = s;
      reinterpret_cast<float*>(p.u_z)[at] = row >= 0 ? __ldcg(p.z_in + (size_t)row * p.r + c) * scale : 0.0f;
    }
  }
  __syncthreads();
  const float* w2 = p.w2 + (size_t)a * p.r * p.d_n;
  const int nb_end = p.out ? (p.d_n + 31) >> 5 : 0;
#pragma unroll 1
  for (int nb = wi; nb < nb_end; nb += nw) {
    const int c = nb * 32 + 8 * q;
    if (c >= p.d_n) continue;
    float o[4][8];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int j = 0; j < 8; ++j) o[m][j] = 0.0f;
#pragma unroll 1
    for (int k = 0; k < p.r; k += 4) {
      float4 z[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) z[m] = *reinterpret_cast<const float4*>(mid + (8 * m + g) * kStride + k);
      if (!TRANS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint4 w = ld_dep16(w2 + (size_t)(c + j) * p.r + k);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            o[m][j] = fmaf(z[m].x, __uint_as_float(w.x), o[m][j]);
            o[m][j] = fmaf(z[m].y, __uint_as_float(w.y), o[m][j]);
            o[m][j] = fmaf(z[m].z, __uint_as_float(w.z), o[m][j]);
            o[m][j] = fmaf(z[m].w, __uint_as_float(w.w), o[m][j]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float w[8];
          load8(w2 + (size_t)(k + i) * p.d_n + c, w);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float zz = i == 0 ? z[m].x : i == 1 ? z[m].y : i == 2 ? z[m].z : z[m].w;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[m][j] = fmaf(zz, w[j], o[m][j]);
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int row = rows[8 * m + g];
      if (row < 0) continue;
      if (DROP && TRANS) drop8(o[m], drop_draws(p.drop, row, c >> 3), p.drop.thr16);
      if (p.base) {
        float b[8];
        load8(p.base + (size_t)row * p.ld_base + c, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[m][j] += b[j];
      }
      store8(p.out + (size_t)row * p.ld_out + c, o[m]);
    }
  }
}

// Gradients of the weights in fp32: a block owns 128 columns and 16 ranks (four columns a lane: with two, the loads of the narrow
// operand took as long as the products; 8192 rows x 4096 + 4096, rank 64, 910 us), its warps and the blocks of its cluster split
// the rows.  The masks of four rows come from two generator blocks a lane, by shuffles.
constexpr int kSimtOutCols = 128;

template <bool DROP>
__global__ void __launch_bounds__(kAdThreads, 2)
adapter_outer_simt_kernel(const OuterArgs p) {
  __shared__ __align__(16) float part[kAdWarps / 2][kSimtRc][kSimtOutCols];
  __shared__ __align__(16) float recv[kSimtRc * kSimtOutCols];       // [ctas][kSimtRc * kSimtOutCols / ctas]
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  rc_cluster_arrive();
  grid_dep_wait();
  grid_dep_trigger();
  const int chunks = (p.r + kSimtRc - 1) / kSimtRc;
  int side, slice;
  outer_slice(p, blockIdx.x, side, slice);
  const int a = blockIdx.y / chunks, rc = (blockIdx.y % chunks) * kSimtRc;
  const OuterSide sd = p.side[side];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int lo = 0, hi = p.n_rows;                                         // positions in the order of the tiles
  if (p.tiles.row_adapter) {
    lo = __ldcg(p.tiles.tile_start + a) * p.m;
    hi = __ldcg(p.tiles.tile_start + a + 1) * p.m;
  } else if (a > 0) {
    hi = 0;
  }
  const float* v = (const float*)sd.v;
  const float* u = (const float*)sd.u;
  const int c = slice * kSimtOutCols + 4 * lane;         // widths are multiples of 8: four columns are in or out together
  const bool in = c < sd.d, drop = DROP && side == 0;
  float acc[4][kSimtRc];
#pragma unroll
  for (int j = 0; j < kSimtRc; ++j) acc[0][j] = acc[1][j] = acc[2][j] = acc[3][j] = 0.0f;
  const int stride = (int)ctas * kAdWarps * 4;
#pragma unroll 1
  for (int t = lo + ((int)rank * kAdWarps + warp) * 4; t < hi; t += stride) {
    int row[4];
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      row[i] = t + i < hi ? (p.tiles.row_adapter ? __ldcg(p.tiles.row_list + t + i) : t + i) : -1;
      x[i] = row[i] >= 0 && in ? ld_dep16(v + (size_t)row[i] * sd.ldv + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    uint32_t bits[2] = {0u, 0u};                                     // of rows lane / 16 and 2 + lane / 16, block lane % 16
    if (drop)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        bits[h] = keep_bits(drop_draws(p.drop, lane < 16 ? row[2 * h] : row[2 * h + 1], (slice * kSimtOutCols >> 3) + (lane & 15)), p.drop.thr16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (drop) {
        const uint32_t b = __shfl_sync(0xffffffffu, bits[i >> 1], 16 * (i & 1) + (lane >> 1)) >> (4 * (lane & 1));
        if (!(b & 1u)) x[i].x = 0u;
        if (!(b & 2u)) x[i].y = 0u;
        if (!(b & 4u)) x[i].z = 0u;
        if (!(b & 8u)) x[i].w = 0u;
      }
      if (row[i] < 0) continue;
      const float xs[4] = {__uint_as_float(x[i].x), __uint_as_float(x[i].y), __uint_as_float(x[i].z), __uint_as_float(x[i].w)};
#pragma unroll
      for (int h = 0; h < kSimtRc / 8; ++h)
        if (rc + 8 * h < p.r) {
          float w[8];
          load8(u + (size_t)(t + i) * p.r + rc + 8 * h, w);
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e][8 * h + j] = fmaf(xs[e], w[j], acc[e][8 * h + j]);
        }
    }
  }
  // the second half of the warps, then the first on top
#pragma unroll
  for (int turn = 1; turn >= 0; --turn) {
    if (warp / (kAdWarps / 2) == turn)
#pragma unroll
      for (int j = 0; j < kSimtRc; ++j) {
        float4& s = *reinterpret_cast<float4*>(&part[warp % (kAdWarps / 2)][j][4 * lane]);
        float4 f = make_float4(acc[0][j], acc[1][j], acc[2][j], acc[3][j]);
        if (turn == 0) { f.x += s.x; f.y += s.y; f.z += s.z; f.w += s.w; }
        s = f;
      }
    __syncthreads();
  }
  rc_cluster_wait();
  constexpr int kAll = kSimtRc * kSimtOutCols;
  const int own = kAll / (int)ctas;
  const float* flat = &part[0][0][0];
  for (int i = 4 * threadIdx.x; i < kAll; i += 4 * kAdThreads) {
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kAdWarps / 2; ++w) {
      const float4 f = *reinterpret_cast<const float4*>(flat + w * kAll + i);
      s.x += f.x; s.y += f.y; s.z += f.z; s.w += f.w;
    }
    push4(rc_peer(recv + (int)rank * own + i % own, i / own), s);
  }
  rc_cluster_arrive();
  rc_cluster_wait();
  float* out = (float*)sd.g + (size_t)a * p.r * sd.d;
  for (int i = threadIdx.x; i < own; i += kAdThreads) {
    float s = 0.0f;
    for (uint32_t k = 0; k < ctas; ++k) s += recv[k * own + i];
    const int at = (int)rank * own + i, j = rc + at / kSimtOutCols, col = slice * kSimtOutCols + at % kSimtOutCols;
    if (j < p.r && col < sd.d) out[side == 0 ? (size_t)j * sd.d + col : (size_t)col * p.r + j] = s;
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------

inline int adapter_rank_tiles(int r) { return r <= 8 ? 1 : r <= 16 ? 2 : r <= 32 ? 4 : 8; }

// 16-row MMA tiles of a row tile: two read the weights half as often; one where the blocks find their tiles themselves (most
// adapters of such a batch have a row or two) and where the batch would not fill the SMs with eight blocks a tile otherwise.
inline int adapter_mt(int n_rows, bool small, int n_sms) { return small || n_rows < 4 * n_sms ? 1 : 2; }
inline bool adapter_small(const int32_t* row_adapter, int n_rows, bool backward) { return row_adapter && n_rows <= kAdSmallRows && !backward; }
// Tiles of 128 rows on tcgen05 (adapters_umma.cuh) where ranks make the weights heavy and tiles are filled.  Both sides, us, all
// kernels of a call, 4096 + 4096 columns (rows x adapters, rank): forward 1024 x 1, 64: 19 against 23; 512 x 1, 64: 20, 16;
// 2048 x 64, 64: 53, 67; 8192 x 16, 64: 54, 109; 8192 x 16, 32: 53, 77; 4096 x 64, 32: 52, 66; 2048 x 1, 32: 26, 21; 8192 x 8, 16:
// 53, 51.  Gradients 8192 x 16, 64: 104, 191; 1024 x 16, 64: 69, 87; 2048 x 1, 64: 53, 52; 8192 x 16, 32: 118, 146; 2048 x 64, 32: 183, 150.
// The rule does not ask for the widths.  Narrow layers are small either way and lose some microseconds to the exchange: 1024 + 1024 columns
// (rows x adapters, rank) forward 1024 x 1, 64: 11.3, 9.8; 8192 x 1, 64: 15.7, 22.1; 4096 x 64, 32: 23.6, 16.4; gradients 1024 x 16, 64: 33, 29;
// 16384 x 64, 64: 75, 124; 256 + 256 columns forward 1024 x 1, 64: 10.1, 7.0; 8192 x 16, 32: 16.5, 13.2; 16384 x 64, 64: 17.7, 25.6.
constexpr int kAdTallRows = 128;
inline bool adapter_tall(bool bf, int n_rows, int n, int r, bool small) {
  return bf && !small && (r > 32 ? n_rows >= 1024 && n_rows >= 32 * n : r > 16 && n_rows >= 4096 && n_rows >= 64 * n);
}
inline int adapter_tile_rows(bool bf, int n_rows, bool small, bool tall, int n_sms) {
  return tall ? kAdTallRows : bf ? 16 * adapter_mt(n_rows, small, n_sms) : kSimtM;
}
inline long long adapter_max_tiles(long long n_rows, int n, int m, bool one) {
  return one ? (n_rows + m - 1) / m : n_rows / m + std::min<long long>(n + 1, n_rows);
}

// A scratch for some rows serves any fewer, whatever tiles those take: room for as many tiles as the lowest have, and for the places of
// the highest that the batch can take (a longer batch never has fewer of them).
struct AdapterScratch { size_t tile_start, tile_adapter, row_list, u_e, u_z, total; };
inline AdapterScratch adapter_scratch(bool bf, int n_rows, int n, int r, bool backward, bool one, bool tall) {
  AdapterScratch s{};
  const int m_lo = bf ? 16 : kSimtM, m_hi = tall ? kAdTallRows : kSimtM;
  const size_t tiles = (size_t)adapter_max_tiles(n_rows, n, m_lo, one), places = (size_t)adapter_max_tiles(n_rows, n, m_hi, one) * m_hi;
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) / 256 * 256; return p; };
  if (!one) {
    s.tile_start = take((size_t)(n + 2) * 4);
    s.tile_adapter = take(tiles * 4);
    s.row_list = take(places * 4);
  }
  if (backward) {
    const size_t u = places * (bf ? (size_t)adapter_rank_tiles(r) * 32 : (size_t)r * 4);
    s.u_e = take(u);
    s.u_z = take(u);
  }
  s.total = at;
  return s;
}

constexpr int kAdSmemPerSm = 220 * 1024;
constexpr size_t kAdPlainSmem = 46 * 1024;    // dynamic shared memory that needs no attribute next to the kernels' static variables

// Clusters of c blocks that run at once with per_sm blocks an SM.  Those of four and eight leave places of the processing
// clusters over: a B200's 148 SMs hold 148, 74, 33, 15 of 1, 2, 4, 8 blocks at one an SM, 296, 148, 71, 33 at two, as the runtime
// says; one cluster more is another round.
inline long long clusters_at_once(int n_sms, int c, int per_sm) {
  const long long places = (long long)n_sms * per_sm;
  return std::max<long long>(1, c <= 2 ? places / c : per_sm == 1 ? (c == 4 ? places * 9 / 40 : places * 13 / 128) : (c == 4 ? places * 24 / 100 : places * 9 / 80));
}

// Blocks of a cluster for `tiles` tiles: as many as run at once, two an SM; no more than have a `block` wide piece of either
// product for each warp, and no more than shared memory for their sums allows.
inline int adapter_ctas(long long tiles, int n_sms, int widest, int block, int smem_limit_ctas) {
  int c = 1;
  while (c < 8 && tiles * c <= n_sms && c * 2 * kAdWarps <= std::max(kAdWarps, (widest + block - 1) / block) && c * 2 <= smem_limit_ctas) c *= 2;
  return c;
}

// most: the most that any launch of the kernel asks for.  The limit belongs to the kernel and the device, so all host threads share
// it: it is always set to the same number, and no launch of one thread lowers what another has just asked for.
template <typename K> inline cudaError_t allow_most_smem(K kernel, size_t smem, size_t most) {
  return smem > kAdPlainSmem ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) : cudaSuccess;
}
template <typename P>
inline cudaError_t launch_cluster(bool dep, void (*kernel)(P), dim3 grid, dim3 cluster, size_t smem, size_t most, cudaStream_t st, const P& args, int threads = kAdThreads) {
  const cudaError_t e = allow_most_smem(kernel, smem, most);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  unsigned n = 0;
  at[n].id = cudaLaunchAttributeClusterDimension;
  at[n].val.clusterDim.x = cluster.x; at[n].val.clusterDim.y = cluster.y; at[n].val.clusterDim.z = cluster.z;
  ++n;
  if (dep) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = at; cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, args);
}

template <int MT, int RT, bool TRANS>
inline cudaError_t launch_adapter_tile(const AdapterArgs<bf16>& a, long long tiles, int n_sms, bool dep, cudaStream_t st) {
  using S = AdapterShape<MT, RT, TRANS>;
  const int room = std::max(1, (kAdSmemPerSm / S::kMinBlocks - S::bytes(0)) / S::kRecv);
  const int ctas = adapter_ctas(tiles, n_sms, std::max(a.d_k, a.d_n), 64, room);
  const size_t smem = S::bytes(ctas), most = S::bytes(std::min(room, 8));
  const dim3 grid((unsigned)(tiles * ctas)), cl(ctas);
  return a.drop.thr16 ? launch_cluster(dep, adapter_kernel<MT, RT, TRANS, true>, grid, cl, smem, most, st, a)
                      : launch_cluster(dep, adapter_kernel<MT, RT, TRANS, false>, grid, cl, smem, most, st, a);
}

template <int MT, bool TRANS>
inline cudaError_t launch_adapter_mt(const AdapterArgs<bf16>& a, long long tiles, int n_sms, bool dep, cudaStream_t st) {
  switch (adapter_rank_tiles(a.r)) {
    case 1: return launch_adapter_tile<MT, 1, TRANS>(a, tiles, n_sms, dep, st);
    case 2: return launch_adapter_tile<MT, 2, TRANS>(a, tiles, n_sms, dep, st);
    case 4: return launch_adapter_tile<MT, 4, TRANS>(a, tiles, n_sms, dep, st);
    default: return launch_adapter_tile<MT, 8, TRANS>(a, tiles, n_sms, dep, st);
  }
}
// m: rows of a tile
template <bool TRANS>
inline cudaError_t launch_adapter(const AdapterArgs<bf16>& a, int m, long long tiles, int n_sms, bool dep, cudaStream_t st) {
  return m == 16 ? launch_adapter_mt<1, TRANS>(a, tiles, n_sms, dep, st) : launch_adapter_mt<2, TRANS>(a, tiles, n_sms, dep, st);
}
template <bool TRANS>
inline cudaError_t launch_adapter(const AdapterArgs<float>& a, int, long long tiles, int n_sms, bool dep, cudaStream_t st) {
  const int ctas = adapter_ctas(tiles, n_sms, std::max(a.d_k, a.d_n), 32, 8);
  const size_t smem = AdapterSimtSmem::bytes(ctas), most = AdapterSimtSmem::bytes(8);
  const dim3 grid((unsigned)(tiles * ctas)), cl(ctas);
  return a.drop.thr16 ? launch_cluster(dep, adapter_simt_kernel<TRANS, true>, grid, cl, smem, most, st, a)
                      : launch_cluster(dep, adapter_simt_kernel<TRANS, false>, grid, cl, smem, most, st, a);
}

template <typename T>
inline cudaError_t launch_adapter_plan(const AdapterArgs<T>& a, int m, const AdPlanOut& o, cudaStream_t st) {
  const size_t smem = adapter_plan_smem(a.n);
  const cudaError_t e = allow_most_smem(adapter_plan_kernel, smem, adapter_plan_smem(kAdMaxAdapters));
  if (e != cudaSuccess) return e;
  int blocks = 1;                              // a batch of 32 rows or two for every warp
  while (blocks < 8 && a.n_rows > blocks * 1024) blocks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(1024); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = blocks; at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, adapter_plan_kernel, a.tiles.row_adapter, a.n_rows, a.n, m, o);
}

// Blocks that share an adapter's rows: the split with the least rounds of the SMs times steps a block, where a block's start
// and the sums between blocks cost about twelve steps (16384 rows of four adapters of rank 64 over 5120 + 5120 columns, by one, two,
// four, eight blocks: 179, 140, 161, 209 us; 4096 rows of one of rank 32 over 4096 + 4096: 84, 46, 27, 45; of rank 8 under a
// mask: 120, 63, 36, 30).
inline int outer_ctas(long long blocks, int n_sms, int per_sm, long long steps) {
  int best = 1;
  long long least = 0;
  for (int c = 1; c <= 8; c *= 2) {
    const long long at_once = clusters_at_once(n_sms, c, per_sm);
    const long long cost = (blocks + at_once - 1) / at_once * ((steps + c - 1) / c + 12);
    if (c == 1 || cost < least) { best = c; least = cost; }
  }
  return best;
}

template <int RT> inline cudaError_t launch_outer_rt(OuterArgs p, int n_sms, bool dep, cudaStream_t st) {
  using S = OuterShape<RT>;
  for (int i = 0; i < 2; ++i) p.slices[i] = (p.side[i].d + kOutWidth - 1) / kOutWidth;
  const int slices = p.slices[0] + p.slices[1];
  const int ctas = outer_ctas((long long)slices * p.n, n_sms, S::kBlocks, (long long)p.n_rows / p.n / kOutStageRows);
  const dim3 grid(slices, p.n, ctas), cl(1, 1, ctas);
  return p.drop.thr16 ? launch_cluster(dep, adapter_outer_kernel<RT, true>, grid, cl, S::kSmem, S::kSmem, st, p, kOutThreads)
                      : launch_cluster(dep, adapter_outer_kernel<RT, false>, grid, cl, S::kSmem, S::kSmem, st, p, kOutThreads);
}
inline cudaError_t launch_outer(bool bf, const OuterArgs& a, int n_sms, bool dep, cudaStream_t st) {
  if (bf) switch (adapter_rank_tiles(a.r)) {
      case 1: return launch_outer_rt<1>(a, n_sms, dep, st);
      case 2: return launch_outer_rt<2>(a, n_sms, dep, st);
      case 4: return launch_outer_rt<4>(a, n_sms, dep, st);
      default: return launch_outer_rt<8>(a, n_sms, dep, st);
    }
  OuterArgs p = a;
  for (int i = 0; i < 2; ++i) p.slices[i] = (p.side[i].d + kSimtOutCols - 1) / kSimtOutCols;
  const int slices = p.slices[0] + p.slices[1], chunks = (p.r + kSimtRc - 1) / kSimtRc;
  const int ctas = outer_ctas((long long)slices * p.n * chunks, n_sms, 2, (long long)p.n_rows / p.n / (4 * kAdWarps));
  const dim3 grid(slices, p.n * chunks, ctas), cl(1, 1, ctas);
  return p.drop.thr16 ? launch_cluster(dep, adapter_outer_simt_kernel<true>, grid, cl, 0, 0, st, p)
                      : launch_cluster(dep, adapter_outer_simt_kernel<false>, grid, cl, 0, 0, st, p);
}

}  // namespace cmoe
