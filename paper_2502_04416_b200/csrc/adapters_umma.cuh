// Both products of an adapter (adapters.cuh) for tiles of 128 rows on tcgen05: batches with many rows of each adapter.
//
// A tile of 32 rows reads an adapter's weights once for 32 rows, which at a rank of 64 is more than the rows themselves, and
// warp-level MMAs of the two-part middle take as long as HBM does.  Here 128 rows share the weights and the tensor cores
// read everything from shared memory: X [128 x 64] and W1 [64 x r] give the middle in tensor memory, its two bf16 parts go
// back to shared memory as the A operand, and blocks of 64 output columns meet the rows' base in the epilogue.
// Bound: HBM latency at the start and the end of a block (9 us with nothing in between), then HBM: 16384 rows of four adapters, rank
// 64, 5120 + 5120 columns 101 us, 5 TB/s; by tiles of 32 rows 266 us.
// Blocks of a cluster share the columns of both products and exchange the middle's sums, 1 / ctas of the rows each, in rank order.
//
// Every operand comes by 16-byte cp.async into 128-byte rows with the 128-byte swizzle: rows of one adapter lie anywhere, widths
// end inside a block (zeros from there on).  The forward's dropout masks a block of x in shared memory, by the warps that have the
// epilogue later.  One ring serves both products: blocks of base follow the blocks of x without a gap.
//
// A kernel that follows may allocate tensor memory before it waits for these (a layer's first kernel does, chained to whatever precedes
// it).  It becomes resident only once every block here has let it, which a block does when it has its own: otherwise the two could wait
// for each other, the one for tensor memory and the other for the end of this grid.
#pragma once

#include "adapters.cuh"

namespace cmoe {

constexpr int kAuRows = 128;
constexpr int kAuStages = 6;
constexpr int kAuXBytes = 128 * 128, kAuWBytes = 64 * 128, kAuStage = kAuXBytes + kAuWBytes, kAuRing = kAuStages * kAuStage;
constexpr int kAgLeastRank = 32;                            // ranks above take adapter_outer_umma_kernel
constexpr int kAuEpiWarps = 8, kAuLoadWarps = 4, kAuThreads = 32 * (kAuEpiWarps + kAuLoadWarps + 1);
constexpr int kAuMid = 2 * kAuXBytes, kAuRecv = 128 * 64 * 4;
constexpr int kAuTmem = 256;                                 // the middle: 64 columns; two blocks of output: 2 x 64
constexpr int kAuSmem = 1024 + kAuRing + kAuMid + kAuRecv + kAuRows * 4 + 256;
static_assert(kAuSmem <= 227 * 1024, "shared memory of an SM");

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool have) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16u : 0u) : "memory");
}
// Arrives on `bar` when this thread's copies so far have landed.  (Waiting for them here and arriving once a warp leaves fewer in
// flight: 105 us -> 129 us for the sums over 16384 rows x 5120 + 5120, rank 64; a proxy fence here would wait for all of them.
// The warp that issues the MMAs has the fence.)
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
// Arrives on a barrier of another block of the cluster (address by mapa); what came before is visible to who waits there.
__device__ __forceinline__ void mbar_arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t peer_address(uint32_t a, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
// mbar_wait_warp for barriers that peers arrive on.
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* err, int code) {
  if (!mbar_wait_warp(bar, parity, abort_flag, err, code)) return false;
  asm volatile("fence.acq_rel.cluster;" ::: "memory");
  return true;
}
// B operand that lies [k][64] (64 neighbouring columns a 128-byte row): 8-row groups along k 1024 bytes apart.
__device__ __forceinline__ uint32_t umma_idesc_bt(int n) { return umma_idesc(n) | 1u << 16; }

template <bool TRANS, bool DROP>
__global__ void __launch_bounds__(kAuThreads, 1)
adapter_umma_kernel(const AdapterArgs<bf16> p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base0 = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base0 - raw);
  const uint32_t mid = base0 + kAuRing, recv = mid + kAuMid;
  int32_t* rows = reinterpret_cast<int32_t*>(gen + kAuRing + kAuMid + kAuRecv);
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(rows + kAuRows);
  const uint32_t full0 = smem_u32(bar_mem), empty0 = full0 + 8 * kAuStages, d1_full = empty0 + 8 * kAuStages, d2_full = d1_full + 8,
                 d2_empty = d2_full + 16, sums_here = d2_empty + 16, mid_here = sums_here + 8, done = mid_here + 8, masked0 = done + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_mem + 3 * kAuStages + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  const int warp = warp_index(), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kAuStages; ++s) { mbar_init(full0 + 8 * s, 32 * kAuLoadWarps); mbar_init(empty0 + 8 * s, 4); mbar_init(masked0 + 8 * s, kAuEpiWarps); }
    mbar_init(d1_full, 1);
    mbar_init(done, 1);
    for (int b = 0; b < 2; ++b) { mbar_init(d2_full + 8 * b, 1); mbar_init(d2_empty + 8 * b, 4); }
    mbar_init(sums_here, ctas * kAuEpiWarps);
    mbar_init(mid_here, ctas * kAuEpiWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  grid_dep_wait();
  const int tile = blockIdx.x / ctas;
  int a = 0;
  if (p.tiles.row_adapter) {
    if (tile >= __ldcg(p.tiles.tile_start + p.n + 1)) return;                  // the whole cluster leaves
    a = __ldcg(p.tiles.tile_adapter + tile);
  }
  if (threadIdx.x < kAuRows) {
    const long long at = (long long)tile * kAuRows + threadIdx.x;
    rows[threadIdx.x] = p.tiles.row_adapter ? __ldcg(p.tiles.row_list + at) : at < p.n_rows ? (int32_t)at : -1;
  }
  if (a == p.n) {
    __syncthreads();
    adapter_none<kAuThreads>(p, rows, kAuRows, rank, ctas);
    return;
  }
  if (warp == kAuEpiWarps + kAuLoadWarps) {
    tmem_alloc(smem_u32(tmem_slot), kAuTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  grid_dep_trigger();                                                          // this block has its tensor memory (see the top of the file)
  rc_cluster_arrive();
  rc_cluster_wait();                                                           // every peer's barriers are there
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int kb_all = (p.d_k + 63) >> 6, nb_all = p.out ? (p.d_n + 63) >> 6 : 0;
  const int n1 = kb_all > (int)rank ? (kb_all - (int)rank + (int)ctas - 1) / (int)ctas : 0;       // blocks rank, rank + ctas, ..
  const int n2 = nb_all > (int)rank ? (nb_all - (int)rank + (int)ctas - 1) / (int)ctas : 0;
  const int r16 = (p.r + 15) & ~15;
  const float scale = p.scale ? __ldcg(p.scale + a) : 1.0f;                    // now: later it would come back behind the copies
  const bf16* w1 = p.w1 + (size_t)a * p.r * p.d_k;
  const bf16* w2 = p.w2 + (size_t)a * p.r * p.d_n;

  if (warp >= kAuEpiWarps && warp < kAuEpiWarps + kAuLoadWarps) {
    // ---- loads: chunk `ch` (16 bytes) of rows at + 16 i of a block
    const int t = threadIdx.x - 32 * kAuEpiWarps, at = t >> 3, ch = t & 7;
    const uint32_t dst0 = at * 128 + ((ch ^ (at & 7)) << 4);
    int row_of[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row_of[i] = rows[at + 16 * i];
    const uint32_t x_pitch = (uint32_t)p.ldx * 2, base_pitch = (uint32_t)p.ld_base * 2;
    const auto load_rows = [&](int i) {
      const uint32_t dst = base0 + (i % kAuStages) * kAuStage + dst0;
      if (i < n1) {
        const int k = ((int)rank + i * (int)ctas) * 64 + 8 * ch;
        const bool in = k < p.d_k;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool have = in && row_of[j] >= 0;
          cp_async16(dst + j * 2048, have ? row_at(p.x, row_of[j], x_pitch) + k : p.x, have);
        }
      } else {
        const int c = ((int)rank + (i - n1) * (int)ctas) * 64 + 8 * ch;
        if (p.base && c < p.d_n)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (row_of[j] >= 0) cp_async16(dst + j * 2048, row_at(p.base, row_of[j], base_pitch) + c, true);
      }
    };
    const auto load_weights = [&](int i) {
      const uint32_t dst = base0 + (i % kAuStages) * kAuStage + kAuXBytes + dst0;
      if (i < n1) {
        const int k0 = ((int)rank + i * (int)ctas) * 64, k = k0 + 8 * ch;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int m = at + 16 * j;
          if (!TRANS) {                                      // rows past the rank are columns of the middle that nobody reads
            if (m < p.r) cp_async16(dst + j * 2048, k < p.d_k ? w1 + (size_t)m * p.d_k + k : w1, k < p.d_k);
          } else if (8 * ch < p.r) {
            const bool have = k0 + m < p.d_k;
            cp_async16(dst + j * 2048, have ? w1 + (size_t)(k0 + m) * p.r + 8 * ch : w1, have);
          }
        }
      } else {
        const int c0 = ((int)rank + (i - n1) * (int)ctas) * 64, c = c0 + 8 * ch;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int m = at + 16 * j;
          if (!TRANS) {                                      // ranks up to the next multiple of 16 are zero
            if (c0 + m < p.d_n && 8 * ch < r16) cp_async16(dst + j * 2048, 8 * ch < p.r ? w2 + (size_t)(c0 + m) * p.r + 8 * ch : w2, 8 * ch < p.r);
          } else if (m < r16 && c < p.d_n) {
            cp_async16(dst + j * 2048, m < p.r ? w2 + (size_t)m * p.d_n + c : w2, m < p.r);
          }
        }
      }
    };
    for (int i = 0; i < n1 + n2; ++i) {
      const int st = i % kAuStages, use = i / kAuStages;
      if (use > 0 && !mbar_wait_warp(empty0 + 8 * st, (use - 1) & 1, abort_flag, &g_adapter_error, kErrWaitEmpty)) break;
      load_rows(i);
      load_weights(i);
      cp_async_arrive(full0 + 8 * st);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kAuEpiWarps + kAuLoadWarps) {
    // ---- products
    const uint32_t idesc_k = umma_idesc(64), idesc_t = umma_idesc_bt(64);
    bool ok = true;
    for (int i = 0; ok && i < n1; ++i) {
      const int s = i % kAuStages;
      if (!(ok = mbar_wait_warp((DROP && !TRANS ? masked0 : full0) + 8 * s, (i / kAuStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull))) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_after();
      const uint32_t x = base0 + s * kAuStage, w = x + kAuXBytes;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma_bf16(tmem, umma_smem_desc(x + 32 * k), umma_smem_desc(w + (TRANS ? 2048 : 32) * k), TRANS ? idesc_t : idesc_k, i > 0 || k > 0);
        umma_commit(empty0 + 8 * s);
        mbar_arrive_n(empty0 + 8 * s, 3);                    // a stage of the second product is freed by four warps
      }
      __syncwarp();
    }
    if (elect_one()) umma_commit(d1_full);
    __syncwarp();
    if (ok) ok = mbar_wait_cluster(mid_here, 0, abort_flag, &g_adapter_error, kErrWaitFull);
    asm volatile("fence.proxy.async;" ::: "memory");
    for (int j = 0; ok && j < n2; ++j) {
      const int i = n1 + j, s = i % kAuStages, b = j & 1;
      if (!mbar_wait_warp(full0 + 8 * s, (i / kAuStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull)) break;
      if (j >= 2 && !mbar_wait_warp(d2_empty + 8 * b, ((j >> 1) - 1) & 1, abort_flag, &g_adapter_error, kErrWaitAccEmpty)) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_after();
      const uint32_t w = base0 + s * kAuStage + kAuXBytes;
      if (elect_one()) {
        for (int lo = 1; lo >= 0; --lo)
          for (int k = 0; k < r16 / 16; ++k)
            umma_bf16(tmem + 64 + 64 * b, umma_smem_desc(mid + lo * kAuXBytes + 32 * k), umma_smem_desc(w + (TRANS ? 2048 : 32) * k),
                      TRANS ? idesc_t : idesc_k, lo == 0 || k > 0);
        umma_commit(d2_full + 8 * b);
      }
      __syncwarp();
    }
  } else {
    // ---- the middle's sums: lane = row, a warpgroup takes half of the ranks
    const int quad = warp & 3, half = warp >> 2, m = 32 * quad + lane, share = kAuRows / (int)ctas;
    const uint32_t my_tmem = tmem + ((uint32_t)(32 * quad) << 16);
    bool ok = true;
    if (DROP && !TRANS) {                                    // the masks of x, while there is nothing else to do
      const int at = threadIdx.x >> 3, ch = threadIdx.x & 7;
      for (int i = 0; ok && i < n1; ++i) {
        const int s = i % kAuStages, k = ((int)rank + i * (int)ctas) * 64 + 8 * ch;
        const uint32_t dst = base0 + s * kAuStage + at * 128 + ((ch ^ (at & 7)) << 4);
        uint4 draws[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) draws[j] = drop_draws(p.drop, rows[at + 32 * j], k >> 3);
        if (!(ok = mbar_wait_warp(full0 + 8 * s, (i / kAuStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull))) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) sts16(dst + j * 4096, drop8(lds16(dst + j * 4096), draws[j], p.drop.thr16));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(masked0 + 8 * s);
      }
    }
    ok = ok && mbar_wait_warp(d1_full, 0, abort_flag, &g_adapter_error, kErrWaitAccFull);
    if (ok) {
      tc_fence_after();
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = 0.0f;
      if (n1 > 0) {
        tmem_ld16(my_tmem + 32 * half, v);
        tmem_ld16(my_tmem + 32 * half + 16, v + 16);
        tmem_ld_wait();
      }
      const float drop_inv = DROP ? p.drop.inv : 1.0f;
      // eight ranks from n0 on of row mm: the forward's z, and both parts of the scaled middle into this block's or every block's operand
      const auto finish = [&](int mm, int n0, float (&t)[8]) {
        const int row = rows[mm];
        const bool have = row >= 0 && n0 < p.r;
        uint16_t hi[8], lo[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[e] *= drop_inv;
          split_bf16(have ? t[e] * scale : 0.0f, hi[e], lo[e]);
        }
        if (p.z_out && have) {
          float2* z = reinterpret_cast<float2*>(p.z_out + (size_t)row * p.r + n0);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = make_float2(t[2 * e], t[2 * e + 1]);
        }
        const uint32_t at = mid + mm * 128 + (((n0 >> 3) ^ (mm & 7)) << 4);
        const auto pack = [](const uint16_t (&v)[8]) { return make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16); };
        const uint4 h = pack(hi), l = pack(lo);
        if (ctas == 1) {
          sts16(at, h);
          sts16(at + kAuXBytes, l);
        } else {
          for (uint32_t c = 0; c < ctas; ++c) {
            const uint32_t d = peer_address(at, c);
            push4(d, make_float4(__uint_as_float(h.x), __uint_as_float(h.y), __uint_as_float(h.z), __uint_as_float(h.w)));
            push4(d + kAuXBytes, make_float4(__uint_as_float(l.x), __uint_as_float(l.y), __uint_as_float(l.z), __uint_as_float(l.w)));
          }
        }
      };
      if (ctas == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) finish(m, 32 * half + 8 * i, *reinterpret_cast<float (*)[8]>(v + 8 * i));
      } else {
        const uint32_t dst = peer_address(recv, (uint32_t)(m / share)) + ((int)rank * share + m % share) * 256;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          push4(dst + (((8 * half + i) ^ (m & 15)) << 4), make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
        __syncwarp();
        if (lane < (int)ctas) mbar_arrive_peer(peer_address(sums_here, lane));
        ok = mbar_wait_cluster(sums_here, 0, abort_flag, &g_adapter_error, kErrWaitFull);
        const float4* got = reinterpret_cast<const float4*>(gen + kAuRing + kAuMid);
        for (int i = threadIdx.x; ok && i < share * 8; i += 32 * kAuEpiWarps) {
          const int mr = i >> 3, mm = (int)rank * share + mr, q = 2 * (i & 7);
          float t[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] = 0.0f;
          for (uint32_t c = 0; c < ctas; ++c) {
            const float4 x = got[((int)c * share + mr) * 16 + (q ^ (mm & 15))], y = got[((int)c * share + mr) * 16 + ((q + 1) ^ (mm & 15))];
            t[0] += x.x; t[1] += x.y; t[2] += x.z; t[3] += x.w; t[4] += y.x; t[5] += y.y; t[6] += y.z; t[7] += y.w;
          }
          finish(mm, 4 * q, t);
        }
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      __syncwarp();
      if (ok && lane < (int)ctas) mbar_arrive_peer(peer_address(mid_here, lane));
      ok = ok && mbar_wait_cluster(mid_here, 0, abort_flag, &g_adapter_error, kErrWaitFull);
      if (TRANS && p.u_e && ok && p.r <= kAgLeastRank) {
        // operands of adapter_outer_kernel: MMA fragments, 16 rows x 8 ranks a warp; this block's share of the rows
        const int rt_n = p.r <= 8 ? 1 : p.r <= 16 ? 2 : 4, groups = 8 / (int)ctas;
        for (int i = threadIdx.x; i < groups * rt_n * 32; i += 32 * kAuEpiWarps) {
          const int l = i & 31, rt = (i >> 5) % rt_n, mt = (int)rank * groups + (i >> 5) / rt_n, nn = rt * 8 + (l >> 2), t0 = mt * 16 + 2 * (l & 3);
          uint16_t e[2][4], z[2][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int mm = t0 + (j & 1) + 8 * (j >> 1), z_row = rows[mm], at = mm * 64 + (((nn >> 3) ^ (mm & 7)) << 3) + (nn & 7);
            const uint16_t* mids = reinterpret_cast<const uint16_t*>(gen + kAuRing);
            e[0][j] = mids[at];
            e[1][j] = mids[kAuXBytes / 2 + at];
            split_bf16(z_row >= 0 && nn < p.r ? __ldcg(p.z_in + (size_t)z_row * p.r + nn) * scale : 0.0f, z[0][j], z[1][j]);
          }
          const size_t at = (((size_t)tile * 8 + mt) * rt_n + rt) * 32 + l;
          const auto pack = [](const uint16_t (&v)[2][4]) { return make_uint4(v[0][0] | (uint32_t)v[0][1] << 16, v[0][2] | (uint32_t)v[0][3] << 16, v[1][0] | (uint32_t)v[1][1] << 16, v[1][2] | (uint32_t)v[1][3] << 16); };
          reinterpret_cast<uint4*>(p.u_e)[at] = pack(e);
          reinterpret_cast<uint4*>(p.u_z)[at] = pack(z);
        }
      } else if (TRANS && p.u_e && ok) {
        // operands of the sums over rows: a tile's 128 rows as they lie here, high parts, then low parts; this block's share
        uint4* ue = reinterpret_cast<uint4*>(p.u_e) + (size_t)tile * (kAuMid / 16);
        uint4* uz = reinterpret_cast<uint4*>(p.u_z) + (size_t)tile * (kAuMid / 16);
        for (int i = threadIdx.x; i < share * 8; i += 32 * kAuEpiWarps) {
          const int mm = (int)rank * share + (i >> 3), ch = i & 7, at = mm * 8 + (ch ^ (mm & 7)), z_row = rows[mm];
          ue[at] = lds16(mid + at * 16);
          ue[kAuXBytes / 16 + at] = lds16(mid + kAuXBytes + at * 16);
          uint16_t zh[8], zl[8];
          const bool have = z_row >= 0 && 8 * ch < p.r;
#pragma unroll
          for (int e = 0; e < 8; ++e) split_bf16(have ? __ldcg(p.z_in + (size_t)z_row * p.r + 8 * ch + e) * scale : 0.0f, zh[e], zl[e]);
          uz[at] = make_uint4(zh[0] | (uint32_t)zh[1] << 16, zh[2] | (uint32_t)zh[3] << 16, zh[4] | (uint32_t)zh[5] << 16, zh[6] | (uint32_t)zh[7] << 16);
          uz[kAuXBytes / 16 + at] = make_uint4(zl[0] | (uint32_t)zl[1] << 16, zl[2] | (uint32_t)zl[3] << 16, zl[4] | (uint32_t)zl[5] << 16, zl[6] | (uint32_t)zl[7] << 16);
        }
      }
    }
    // ---- the second product's epilogue: a warpgroup takes every other block of 64 columns, lane = row
    const int row = rows[m];
    const uint32_t out_pitch = (uint32_t)p.ld_out * 2;
    for (int j = half; ok && j < n2; j += 2) {
      const int i = n1 + j, s = i % kAuStages, c0 = ((int)rank + j * (int)ctas) * 64;
      if (!mbar_wait_warp(full0 + 8 * s, (i / kAuStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull)) break;
      if (!mbar_wait_warp(d2_full + 8 * half, (j >> 1) & 1, abort_flag, &g_adapter_error, kErrWaitAccFull)) break;
      tc_fence_after();
      float v[64];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_ld16(my_tmem + 64 + 64 * half + 16 * q, v + 16 * q);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(d2_empty + 8 * half);
      const uint32_t x = base0 + s * kAuStage, mine = x + m * 128;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const uint32_t at = mine + ((q ^ (m & 7)) << 4);
        float (&o)[8] = *reinterpret_cast<float (*)[8]>(v + 8 * q);
        if (DROP && TRANS) drop8(o, drop_draws(p.drop, row, (c0 >> 3) + q), p.drop.thr16);
        if (p.base) {
          const uint4 b = lds16(at);
          const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) { o[2 * e] += __uint_as_float(w[e] << 16); o[2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u); }
        }
        sts16(at, make_uint4(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]), pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7])));
      }
      __syncwarp();
      const int ch = lane & 7, c = c0 + 8 * ch;              // whole 128-byte lines of four rows at a time
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int mm = 32 * quad + 4 * q + (lane >> 3), to = __shfl_sync(0xffffffffu, row, 4 * q + (lane >> 3));
        const uint4 o = lds16(x + mm * 128 + ((ch ^ (mm & 7)) << 4));
        if (to >= 0 && c < p.d_n) *reinterpret_cast<uint4*>(const_cast<bf16*>(row_at(p.out, to, out_pitch)) + c) = o;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty0 + 8 * s);
    }
  }
  // ---- no peer writes here any more, and none of the MMAs that the epilogue did not see is left
  __syncwarp();
  if (warp == kAuEpiWarps + kAuLoadWarps) {
    if (elect_one()) umma_commit(done);
    __syncwarp();
  }
  tc_fence_before();
  rc_cluster_arrive();
  rc_cluster_wait();
  __syncthreads();
  if (warp == kAuEpiWarps + kAuLoadWarps) {
    mbar_wait_warp(done, 0, abort_flag, &g_adapter_error, kErrWaitAccFull);
    tc_fence_after();
    tmem_dealloc(tmem, kAuTmem);
  }
}

// ---- the gradients of the weights ---------------------------------------------------------------------------------------
// G[k][c] = sum over the adapter's rows t of U[t][k] V[t][c], as adapter_outer_kernel, for the tiles above: U's rows [32 x 64],
// high and low parts, are 128 rows of the product, V's [32 x 256] its columns; both as they lie in memory (the sum runs along
// their rows: operands whose columns are neighbours).  Two MMAs of 256 columns a step; with V as the rows and U as 64 columns they
// were eight.  U was written in the swizzled order and comes by bulk copies.  Two blocks an SM, so that one's start and end (13 us
// with a cluster) are the other's time.  Blocks of a cluster split the rows and add their sums through shared memory, in rank order.
// Bound: the bytes a block has in flight, 4 steps of 24 KB at a loaded latency of 2 to 3 us; DRAM at 44 %, the tensor pipe at 24 %
// (8192 rows of four adapters, rank 64, 4096 + 4096 columns, 39 us).
constexpr int kAgCols = 256, kAgRows = 32, kAgStages = 4, kAgAtom = kAgRows * 128;      // 64 columns of a stage's rows
constexpr int kAgVBytes = kAgCols / 64 * kAgAtom, kAgUBytes = 2 * kAgAtom, kAgStage = kAgVBytes + kAgUBytes;
constexpr int kAgTmem = 256;
static_assert(kAgRows == 32, "eight rows a loading warp, four a masking one");
constexpr int kAgSmem = 1024 + kAgStages * kAgStage + 256;
static_assert(2 * (kAgSmem + 1024) <= 227 * 1024 && kAgStages * kAgStage >= kAgCols * 64 * 4 + 128 * 64 * 4, "shared memory of an SM; the sums' exchange in the ring");

// An operand that lies [k][columns], 64 columns a 128-byte row: the next 64 columns a block of a stage's rows on.
__device__ __forceinline__ uint64_t umma_smem_desc_at(uint32_t addr) { return umma_smem_desc(addr) - ((uint64_t)1 << 16) + ((uint64_t)(kAgAtom >> 4) << 16); }

template <bool DROP>
__global__ void __launch_bounds__(kAuThreads, 2)
adapter_outer_umma_kernel(const OuterArgs p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base0 = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base0 - raw);
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(gen + kAgStages * kAgStage);
  const uint32_t full0 = smem_u32(bar_mem), empty0 = full0 + 8 * kAgStages, masked0 = empty0 + 8 * kAgStages, done = masked0 + 8 * kAgStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_mem + 3 * kAgStages + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t ctas = cluster_ctas(), rank = cluster_rank();
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kAgStages; ++s) {
      mbar_init(full0 + 8 * s, 32 * kAuLoadWarps + 1);
      mbar_init(empty0 + 8 * s, 1);
      mbar_init(masked0 + 8 * s, kAuEpiWarps);
    }
    mbar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  grid_dep_wait();                                         // before the allocation: a block that waits holds no tensor memory
  if (warp == kAuEpiWarps + kAuLoadWarps) {
    tmem_alloc(smem_u32(tmem_slot), kAgTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  grid_dep_trigger();                                      // this block has its tensor memory
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
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
  const int c_lo = slice * kAgCols;
  const int n_stages = hi > lo ? (int)((hi - lo + kAgRows - 1) / kAgRows) : 0;
  const int mine = n_stages > (int)rank ? (n_stages - (int)rank + (int)ctas - 1) / (int)ctas : 0;     // stages rank, rank + ctas, ..
  const bool drop = DROP && side == 0;
  const auto place = [&](int i) { return lo + ((long long)i * ctas + rank) * kAgRows; };

  if (warp >= kAuEpiWarps && warp < kAuEpiWarps + kAuLoadWarps) {
    // ---- loads: a warp takes rows lw, lw + 4, .. of a stage, a lane 16 bytes of each
    const int lw = warp - kAuEpiWarps;
    const uint32_t v_pitch = (uint32_t)sd.ldv * 2;
    const bool in = c_lo + 8 * lane < sd.d;
    // A warp's rows of four stages, eight a stage, one a lane; asked for eight stages ahead, since a load comes back behind the
    // copies that went before it.
    const auto rows_of = [&](int i) {
      const long long pos = place(i + (lane >> 3)) + lw + 4 * (lane & 7);
      return i + (lane >> 3) >= mine || pos >= hi ? -1 : p.tiles.row_adapter ? __ldcg(p.tiles.row_list + pos) : (int)pos;
    };
    int row = -1, next = rows_of(0), next2 = rows_of(4);
    for (int i = 0; i < mine; ++i) {
      const int s = i % kAgStages, use = i / kAgStages;
      if (i % 4 == 0) { row = next; next = next2; next2 = rows_of(i + 8); }
      if (use > 0 && !mbar_wait_warp(empty0 + 8 * s, (use - 1) & 1, abort_flag, &g_adapter_error, kErrWaitEmpty)) break;
      const uint32_t v = base0 + s * kAgStage, bar = full0 + 8 * s;
      if (lw == 0 && elect_one()) {
        const uint4* u = (const uint4*)sd.u + place(i) / kAuRows * (kAuMid / 16) + place(i) % kAuRows * 8;
        mbar_expect_tx(bar, kAgUBytes);
        bulk_copy(v + kAgVBytes, u, kAgUBytes / 2, bar);
        bulk_copy(v + kAgVBytes + kAgUBytes / 2, u + kAuXBytes / 16, kAgUBytes / 2, bar);
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kAgRows / 4; ++j) {
        const int r = __shfl_sync(0xffffffffu, row, 8 * (i % 4) + j), m = lw + 4 * j;
        if (in) cp_async16(v + (lane >> 3) * kAgAtom + m * 128 + (((lane & 7) ^ (m & 7)) << 4), r >= 0 ? row_at((const bf16*)sd.v, r, v_pitch) + c_lo + 8 * lane : sd.v, r >= 0);
      }
      cp_async_arrive(bar);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kAuEpiWarps + kAuLoadWarps) {
    // ---- products
    const uint32_t idesc = umma_idesc_bt(kAgCols) | 1u << 15;
    int i = 0;
    for (; i < mine; ++i) {
      const int s = i % kAgStages;
      if (!mbar_wait_warp((drop ? masked0 : full0) + 8 * s, (i / kAgStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull)) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_after();
      const uint32_t v = base0 + s * kAgStage, u = v + kAgVBytes;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kAgRows / 16; ++k) umma_bf16(tmem, umma_smem_desc_at(u + 2048 * k), umma_smem_desc_at(v + 2048 * k), idesc, i > 0 || k > 0);
        umma_commit(empty0 + 8 * s);
      }
      __syncwarp();
    }
    if (i < mine)                                          // a wait ran out: what is on its way lands before the block ends
      for (int j = max(0, i - kAgStages); j < min(mine, i + kAgStages); ++j) {
        const long long t = clock64();
        while (!mbar_try_wait(full0 + 8 * (j % kAgStages), (j / kAgStages) & 1) && clock64() - t < kUmmaWaitCycles / 8) {}
      }
    if (elect_one()) umma_commit(done);
    __syncwarp();
  } else if (drop) {
    // ---- the masks of x: a warp takes rows warp, warp + 8, .. of a stage, a lane 16 bytes of each
    const auto rows_of = [&](int i) {                      // of eight stages, four a stage, one a lane
      const long long pos = place(i + (lane >> 2)) + warp + 8 * (lane & 3);
      return i + (lane >> 2) >= mine || pos >= hi ? 0 : p.tiles.row_adapter ? __ldcg(p.tiles.row_list + pos) : (int)pos;
    };
    int row = 0, next = rows_of(0);
    for (int i = 0; i < mine; ++i) {
      const int s = i % kAgStages;
      if (i % 8 == 0) { row = next; next = rows_of(i + 8); }
      uint4 draws[kAgRows / 8];
#pragma unroll
      for (int j = 0; j < kAgRows / 8; ++j) draws[j] = drop_draws(p.drop, __shfl_sync(0xffffffffu, row, 4 * (i % 8) + j), (c_lo >> 3) + lane);
      if (!mbar_wait_warp(full0 + 8 * s, (i / kAgStages) & 1, abort_flag, &g_adapter_error, kErrWaitFull)) break;
#pragma unroll
      for (int j = 0; j < kAgRows / 8; ++j) {
        const int m = warp + 8 * j;
        const uint32_t at = base0 + s * kAgStage + (lane >> 3) * kAgAtom + m * 128 + (((lane & 7) ^ (m & 7)) << 4);
        sts16(at, drop8(lds16(at), draws[j], p.drop.thr16));
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(masked0 + 8 * s);
    }
  }
  // ---- the sums: lanes 0 .. 63 of tensor memory have the high parts' of 64 ranks, 64 .. 127 the low parts'.  Half of the columns
  // at a time: low parts by way of shared memory to the high ones' warps, those to the block of the cluster that has the column.
  const bool have = warp < kAuEpiWarps && mbar_wait_warp(done, 0, abort_flag, &g_adapter_error, kErrWaitAccFull) && mine > 0;
  tc_fence_after();
  const int share = kAgCols / (int)ctas, n = 32 * (warp & 1) + lane;
  // 16 bytes are four columns of a rank; they are turned by the rank, so that eight ranks meet in no bank
  float4* got = reinterpret_cast<float4*>(gen);            // [ctas][64][share / 4]
  float4* low = got + kAgCols / 4 * 64;                    // [64][128 / 4]
  __syncthreads();
  rc_cluster_arrive();                                     // no block copies into its ring any more
  rc_cluster_wait();
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    const int c0 = 64 * (warp >> 2);
    const bool is_low = warp & 2;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
      if (warp < kAuEpiWarps && is_low == (turn == 0)) {
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          float v[16];
          if (have) {
            tmem_ld16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 128 * h + c0 + 16 * q, v);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
          }
          const int c = c0 + 16 * q, col = 128 * h + c;    // 16 neighbours, all of one block's share
          const uint32_t dst = peer_address(base0, (uint32_t)(col / share)) + ((int)rank * 64 + n) * share * 4;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float4& l = low[n * 32 + ((c / 4 + i) ^ (n & 7))];
            const float4 x = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            if (is_low) l = x;
            else push4(dst + (((col % share / 4 + i) ^ (n & 7)) << 4), make_float4(x.x + l.x, x.y + l.y, x.z + l.z, x.w + l.w));
          }
        }
      }
      __syncthreads();
    }
  }
  rc_cluster_arrive();
  rc_cluster_wait();
  {
    bf16* out = (bf16*)sd.g + (size_t)a * p.r * sd.d;
    const int first = c_lo + (int)rank * share, quads = share / 4;
    if (side == 0) {
      for (int i = threadIdx.x; i < quads * p.r; i += kAuThreads) {
        const int k = i / quads, c = i % quads;            // widths are multiples of 8: four columns are in or out together
        if (first + 4 * c >= sd.d) continue;
        float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (uint32_t b = 0; b < ctas; ++b) {
          const float4 w = got[((int)b * 64 + k) * quads + (c ^ (k & 7))];
          t.x += w.x; t.y += w.y; t.z += w.z; t.w += w.w;
        }
        *reinterpret_cast<uint2*>(out + (size_t)k * sd.d + first + 4 * c) = make_uint2(pack_bf16x2(t.x, t.y), pack_bf16x2(t.z, t.w));
      }
    } else {
      const float* flat = reinterpret_cast<const float*>(got);
      for (int i = threadIdx.x; i < share * (p.r / 8); i += kAuThreads) {
        const int c = i % share, k = i / share * 8;
        if (first + c >= sd.d) continue;
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = 0.0f;
        for (uint32_t b = 0; b < ctas; ++b)
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] += flat[(((int)b * 64 + k + e) * quads + ((c / 4) ^ e)) * 4 + c % 4];
        *reinterpret_cast<uint4*>(out + (size_t)(first + c) * p.r + k) =
            make_uint4(pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3]), pack_bf16x2(t[4], t[5]), pack_bf16x2(t[6], t[7]));
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kAuEpiWarps + kAuLoadWarps) {
    mbar_wait_warp(done, 0, abort_flag, &g_adapter_error, kErrWaitAccFull);
    tc_fence_after();
    tmem_dealloc(tmem, kAgTmem);
  }
}

// Blocks of a cluster for `tiles` tiles: the split with the least rounds of the SMs times blocks of 64 columns a block, where
// a block's start and the exchange cost about as much as kAuFixed of them.
constexpr int kAuFixed = 16;
inline int adapter_umma_ctas(long long tiles, int n_sms, int blocks) {
  int best = 1;
  long long least = 0;
  for (int c = 1; c <= 8; c *= 2) {
    const long long at_once = clusters_at_once(n_sms, c, 1);
    const long long cost = (tiles + at_once - 1) / at_once * ((blocks + c - 1) / c + kAuFixed);
    if (c == 1 || cost < least) { best = c; least = cost; }
  }
  return best;
}
// tiles: the most there can be.  The split does not ask whether the second product is wanted: the middle keeps its bits.
template <bool TRANS>
inline cudaError_t launch_adapter_umma(const AdapterArgs<bf16>& a, long long tiles, int n_sms, bool dep, cudaStream_t st) {
  const long long likely = std::min<long long>(tiles, ((long long)a.n_rows + 64LL * (a.n + 1)) / kAuRows + 1);
  const int ctas = adapter_umma_ctas(a.tiles.row_adapter ? likely : tiles, n_sms, (a.d_k + 63) / 64 + (a.d_n + 63) / 64);
  const dim3 grid((unsigned)(tiles * ctas)), cl(ctas);
  return a.drop.thr16 ? launch_cluster(dep, adapter_umma_kernel<TRANS, true>, grid, cl, kAuSmem, kAuSmem, st, a, kAuThreads)
                      : launch_cluster(dep, adapter_umma_kernel<TRANS, false>, grid, cl, kAuSmem, kAuSmem, st, a, kAuThreads);
}

inline cudaError_t launch_outer_umma(OuterArgs p, int n_sms, bool dep, cudaStream_t st) {
  for (int i = 0; i < 2; ++i) p.slices[i] = (p.side[i].d + kAgCols - 1) / kAgCols;
  const int slices = p.slices[0] + p.slices[1];
  // Blocks that share an adapter's rows: until there are one and a half an SM, with four steps of 64 rows or more each (16384
  // rows of four adapters of rank 64 over 5120 + 5120 columns, by 1, 2, 4, 8 blocks: 185, 105, 101, 145 us; 8192 rows of one over
  // 4096 + 4096: 173, 93, 54, 40 us; 1024 rows of one over 5120 + 5120: 40, 27, 22, 33 us).
  int ctas = 1;
  while (ctas < 8 && (long long)slices * p.n * ctas * 2 < 3LL * n_sms && p.n_rows / p.n >= 512 * ctas) ctas *= 2;
  // Rows of several adapters are seldom shared evenly: two adapters that have nearly all of them should fill the SMs as well, where
  // there are enough of them to pay for more blocks.  The whole gradient by the split above and by twice as many blocks, us, for even shares,
  // random ones and 90 % of the rows with one adapter (rank 64, 5120 + 5120 columns / 4096 + 4096).  From 2048 rows a block on:
  //   16384 x 4   210, 209; 206, 193; 253, 192 / 146, 161; 189, 164; 236, 172
  //   24000 x 4   315, 305; 309, 294; 381, 292 / 222, 239; 263, 248; 356, 262
  //   16384 x 8   212, 205; 211, 191; 384, 253 / 148, 160; 193, 163; 368, 235
  //   32768 x 16  367, 372; 389, 379; 750, 485 / 288, 314; 328, 321; 718, 452
  // and below, where the split stays as it is:
  //   12000 x 4   192, 198; 189, 185; 219, 177 / 132, 148; 159, 150; 197, 152
  //    8192 x 8   129, 132; 136, 130; 211, 146 /  92, 105; 122, 113; 202, 136
  //   16384 x 16  208, 220; 203, 212; 387, 258 / 163, 184; 170, 180; 372, 240
  // A doubling costs even shares up to 10 % above and 16 % below (two of them 20 %: 32768 x 8, 4096 + 4096 columns, 268, 321); random ones
  // gain 2 to 16 % above, and below between 8 % and -6 %.
  while (p.n > 1 && ctas < 8 && 4LL * slices * ctas < 3LL * n_sms && p.n_rows / p.n >= 2048 * ctas) ctas *= 2;
  const dim3 grid(slices, p.n, ctas), cl(1, 1, ctas);
  return p.drop.thr16 ? launch_cluster(dep, adapter_outer_umma_kernel<true>, grid, cl, kAgSmem, kAgSmem, st, p, kAuThreads)
                      : launch_cluster(dep, adapter_outer_umma_kernel<false>, grid, cl, kAgSmem, kAgSmem, st, p, kAuThreads);
}

}  // namespace cmoe
