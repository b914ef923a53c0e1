// Dropout whose keep mask is a function of (seed, offset, row, column) and is never stored.
//
// Eight neighbouring elements of a row (columns 8c .. 8c + 7) share one block of the counter-based generator Philox 4x32
// with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) on the counter
// (c, row, offset low, offset high) under the key (seed low, seed high); column 8c + j takes the j-th of the block's
// eight 16-bit halves, the low half of a word first, and is kept where that draw is at least thr = round(65536 p).
// Sixteen bits an element hold p to 1 / 65536 (kept elements are scaled by 65536 / (65536 - thr), so the mean is exact)
// and make a block the 16 bytes of a bf16 vector; 32 bits would double the generator's work, which would then bound the pass.
#pragma once

#include "common.cuh"

namespace cmoe {

struct Drop {
  uint32_t thr16 = 0;        // thr << 16; 0: nothing is dropped
  float inv = 1.0f;          // 65536 / (65536 - thr)
  uint32_t k[10][2] = {};    // keys of the generator's rounds: seed + round * Weyl constants
  uint32_t off0 = 0, off1 = 0;
  uint32_t row0 = 0;         // row of the mask that the matrix's first row takes
};

// The eight draws of columns 8 * block .. 8 * block + 7, two a word.  The rounds' keys are kernel arguments, read as constants
// by the exclusive ors: added up on the way they would be a fifth of the instructions.
__device__ __forceinline__ uint4 drop_draws(const Drop& d, uint32_t row, uint32_t block) {
  uint32_t c0 = block, c1 = d.row0 + row, c2 = d.off0, c3 = d.off1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ d.k[i][0], n2 = (uint32_t)(p0 >> 32) ^ c3 ^ d.k[i][1];
    c0 = n0; c1 = (uint32_t)p1; c2 = n2; c3 = (uint32_t)p0;
  }
  return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ bool keep_lo(uint32_t w, uint32_t thr16) { return (w << 16) >= thr16; }
__device__ __forceinline__ bool keep_hi(uint32_t w, uint32_t thr16) { return w >= thr16; }   // thr16's low half is zero: w's does not matter

// Dropped elements of eight become zero (a NaN or an infinity too); the scale is the caller's.
__device__ __forceinline__ uint32_t drop_pair(uint32_t v, uint32_t w, uint32_t thr16) {
  if (!keep_lo(w, thr16)) v &= 0xffff0000u;
  if (!keep_hi(w, thr16)) v &= 0x0000ffffu;
  return v;
}
__device__ __forceinline__ uint4 drop8(uint4 v, uint4 w, uint32_t thr16) {
  return make_uint4(drop_pair(v.x, w.x, thr16), drop_pair(v.y, w.y, thr16), drop_pair(v.z, w.z, thr16), drop_pair(v.w, w.w, thr16));
}
__device__ __forceinline__ void drop8(float (&v)[8], uint4 w, uint32_t thr16) {
  const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!keep_lo(r[i], thr16)) v[2 * i] = 0.0f;
    if (!keep_hi(r[i], thr16)) v[2 * i + 1] = 0.0f;
  }
}
__device__ __forceinline__ uint32_t keep_bits(uint4 w, uint32_t thr16) {
  const uint32_t r[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= (keep_lo(r[i], thr16) ? 1u : 0u) << (2 * i) | (keep_hi(r[i], thr16) ? 2u : 0u) << (2 * i);
  return m;
}

constexpr int kDropThreads = 256;

template <typename T> struct DropoutArgs {
  const T *x, *residual;     // residual: may be null
  T* out;                    // may be x or residual
  long long ldx, ld_res, ld_out;
  int rows, cols;
  Drop drop;
};

// out = residual + keep * x / (1 - p).  Bound: HBM (two or three matrices) with the generator close behind: ten rounds
// of two 32 x 32 -> 64 bit products for 16 bytes of bf16.  A thread takes whole blocks of eight columns with 16-byte
// accesses where every row starts on a 16-byte boundary; row and block advance by additions, without a division.
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const DropoutArgs<T> p) {
  const unsigned nb = ((unsigned)p.cols + 7u) >> 3;
  const unsigned long long total = (unsigned long long)p.rows * nb;
  const unsigned long long stride = (unsigned long long)gridDim.x * kDropThreads;
  unsigned long long i = (unsigned long long)blockIdx.x * kDropThreads + threadIdx.x;
  if (i >= total) return;
  unsigned row = (unsigned)(i / nb), b = (unsigned)(i - (unsigned long long)row * nb);
  const unsigned d_row = (unsigned)(stride / nb), d_b = (unsigned)(stride - (unsigned long long)d_row * nb);
  for (; i < total; i += stride) {
    const T* xp = p.x + (size_t)row * p.ldx + 8 * b;
    const T* rp = p.residual ? p.residual + (size_t)row * p.ld_res + 8 * b : nullptr;
    T* op = p.out + (size_t)row * p.ld_out + 8 * b;
    const int have = min(8, p.cols - 8 * (int)b);
    float v[8], r[8];
    if (have == 8) {
      load8(xp, v);
      if (rp) load8(rp, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = j < have ? to_float(xp[j]) : 0.0f;
        if (rp) r[j] = j < have ? to_float(rp[j]) : 0.0f;
      }
    }
    drop8(v, drop_draws(p.drop, row, b), p.drop.thr16);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = rp ? fmaf(v[j], p.drop.inv, r[j]) : v[j] * p.drop.inv;
    if (have == 8) {
      store8(op, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < have) op[j] = from_float<T>(v[j]);
    }
    row += d_row; b += d_b;
    if (b >= nb) { b -= nb; ++row; }
  }
}

// The same for a contiguous matrix whose width is no multiple of eight: its elements as one array in vectors of eight, which start
// at column s past a block's first in a whole row.  A lane draws for the block that its vector starts in and has the keep bits of
// the next one from the next lane, which starts there, or in the next row's first block; only where both a row's last, short block
// and the next row's first lie in one vector does it draw twice.  A warp's last lane draws for its neighbour alone.
// cols >= 16, so that a vector meets two rows at most.
__device__ __forceinline__ float raw_element(const uint4 (&r)[1], int j) {
  const uint32_t w = j < 2 ? r[0].x : j < 4 ? r[0].y : j < 6 ? r[0].z : r[0].w;
  return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
}
__device__ __forceinline__ float raw_element(const uint4 (&r)[2], int j) {
  const uint4& h = r[j >> 2];
  return __uint_as_float((j & 3) == 0 ? h.x : (j & 3) == 1 ? h.y : (j & 3) == 2 ? h.z : h.w);
}

template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_flat_kernel(const DropoutArgs<T> p) {
  constexpr int kRaw = sizeof(T) / 2;                                      // 16-byte pieces of a vector
  const unsigned lane = threadIdx.x & 31, cols = (unsigned)p.cols;
  const unsigned long long n = (unsigned long long)p.rows * cols, vecs = n >> 3;
  if (blockIdx.x == 0 && threadIdx.x < (n & 7)) {                          // what no vector takes, of the last row
    const unsigned long long e = 8 * vecs + threadIdx.x;
    const unsigned row = (unsigned)p.rows - 1, col = (unsigned)(e - (unsigned long long)row * cols);
    const bool keep = keep_bits(drop_draws(p.drop, row, col >> 3), p.drop.thr16) >> (col & 7) & 1u;
    const float x = keep ? to_float(p.x[e]) : 0.0f;
    p.out[e] = from_float<T>(p.residual ? fmaf(x, p.drop.inv, to_float(p.residual[e])) : x * p.drop.inv);
  }
  const unsigned long long warp = ((unsigned long long)blockIdx.x * kDropThreads + threadIdx.x) >> 5;
  const unsigned long long stride = (unsigned long long)gridDim.x * (kDropThreads / 32) * 31;
  unsigned long long v = warp * 31 + lane;
  const unsigned long long row0 = 8 * v / cols, d_row0 = 8 * stride / cols;
  unsigned row = (unsigned)row0, col = (unsigned)(8 * v - row0 * cols);
  const unsigned d_row = (unsigned)d_row0, d_col = (unsigned)(8 * stride - d_row0 * cols);
  for (; v - lane < vecs; v += stride) {
    const bool in = lane < 31 && v < vecs;
    uint4 x[kRaw], r[kRaw];
#pragma unroll
    for (int i = 0; i < kRaw; ++i) {
      x[i] = r[i] = make_uint4(0u, 0u, 0u, 0u);
      if (in) {
        x[i] = ld_dep16(reinterpret_cast<const uint4*>(p.x) + v * kRaw + i);
        if (p.residual) r[i] = ld_dep16(reinterpret_cast<const uint4*>(p.residual) + v * kRaw + i);
      }
    }
    const unsigned b = col >> 3, s = col & 7, left = cols - col;          // left: of the vector's first row
    const uint32_t mine = keep_bits(drop_draws(p.drop, row, b), p.drop.thr16);
    const uint32_t next = __shfl_down_sync(0xffffffffu, mine, 1);
    uint32_t bits = mine >> s;
    if (left > 8) {                                                        // the next lane goes on in this row
      bits |= next << (8 - s);
    } else {
      if (8 * b + 8 < cols) bits |= keep_bits(drop_draws(p.drop, row, b + 1), p.drop.thr16) << (8 - s);
      bits = (bits & ((1u << left) - 1u)) | next << left;
    }
    if (in) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float kept = bits >> j & 1u ? raw_element(x, j) : 0.0f;
        o[j] = p.residual ? fmaf(kept, p.drop.inv, raw_element(r, j)) : kept * p.drop.inv;
      }
      store8(p.out + 8 * v, o);
    }
    row += d_row; col += d_col;
    if (col >= cols) { col -= cols; ++row; }
  }
}

// The same where rows start anywhere: a warp draws for 32 consecutive blocks and walks their 256 elements 32 at a time,
// one element a lane, so that accesses stay side by side; the blocks' keep bits and places come by shuffles.
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_ragged_kernel(const DropoutArgs<T> p) {
  const unsigned nb = ((unsigned)p.cols + 7u) >> 3;
  const unsigned long long total = (unsigned long long)p.rows * nb;
  const unsigned long long stride = (unsigned long long)gridDim.x * kDropThreads;
  const unsigned lane = threadIdx.x & 31;
  // a warp's lanes stay together: those past the end draw for block (0, 0) and store nothing
  for (unsigned long long i = (unsigned long long)blockIdx.x * kDropThreads + threadIdx.x; i - lane < total; i += stride) {
    const bool in = i < total;
    const unsigned row = in ? (unsigned)(i / nb) : 0u, b = in ? (unsigned)(i - (unsigned long long)row * nb) : 0u;
    const uint32_t valid = in ? (0xffu >> (8 - min(8, p.cols - 8 * (int)b))) : 0u;
    const uint32_t bits = keep_bits(drop_draws(p.drop, row, b), p.drop.thr16) | valid << 8;
    float v[8], r[8];
    unsigned at_row[8];
    int at_col[8];
    uint32_t st[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int src = 4 * j + (int)(lane >> 3);
      st[j] = __shfl_sync(0xffffffffu, bits, src) >> (lane & 7);
      at_row[j] = __shfl_sync(0xffffffffu, row, src);
      at_col[j] = 8 * (int)__shfl_sync(0xffffffffu, b, src) + (int)(lane & 7);
      const bool on = st[j] >> 8 & 1u;
      v[j] = on ? to_float(p.x[(size_t)at_row[j] * p.ldx + at_col[j]]) : 0.0f;
      r[j] = on && p.residual ? to_float(p.residual[(size_t)at_row[j] * p.ld_res + at_col[j]]) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float kept = (st[j] & 1u) ? v[j] : 0.0f;
      if (st[j] >> 8 & 1u)
        p.out[(size_t)at_row[j] * p.ld_out + at_col[j]] = from_float<T>(p.residual ? fmaf(kept, p.drop.inv, r[j]) : kept * p.drop.inv);
    }
  }
}

inline int drop_grid(unsigned long long blocks8, int n_sms) {
  const unsigned long long g = (blocks8 + kDropThreads - 1) / kDropThreads;
  return (int)(g < (unsigned long long)n_sms * 16 ? g : (unsigned long long)n_sms * 16);
}

template <typename T> inline cudaError_t launch_dropout(const DropoutArgs<T>& a, int n_sms, cudaStream_t st) {
  const int grid = drop_grid((unsigned long long)a.rows * (((unsigned)a.cols + 7u) / 8), n_sms);
  const auto on16 = [](const void* q, long long ld) { return ((uintptr_t)q & 15) == 0 && (ld * sizeof(T)) % 16 == 0; };
  if (on16(a.x, a.ldx) && on16(a.out, a.ld_out) && (!a.residual || on16(a.residual, a.ld_res)))
    return launch_kernel(false, dropout_kernel<T>, dim3(grid), dim3(kDropThreads), 0, st, a);
  const auto flat = [&](const void* q, long long ld) { return ((uintptr_t)q & 15) == 0 && (ld == a.cols || a.rows == 1); };
  // 4099 x 1377, bf16, one matrix in and out: 20.0 us by the kernel below, 10.6 by this one (device time)
  if (a.cols >= 16 && flat(a.x, a.ldx) && flat(a.out, a.ld_out) && (!a.residual || flat(a.residual, a.ld_res)))
    return launch_kernel(false, dropout_flat_kernel<T>, dim3(drop_grid((unsigned long long)a.rows * a.cols / 8 * 32 / 31 + 1, n_sms)), dim3(kDropThreads), 0, st, a);
  return launch_kernel(false, dropout_ragged_kernel<T>, dim3(grid), dim3(kDropThreads), 0, st, a);
}

}  // namespace cmoe
