// The 8-bit paged key/value cache: rows in, rows out.
//
// A block holds block_size tokens of every head, [head][token][head_dim] bytes, with one fp32 scale for each head of it (keys and
// values apart): value = number * scale.  A scale for a whole block of a head costs 4 bytes in block_size * head_dim, and the
// numbers of a block can enter an integer-valued matrix product as they are, the scale coming in once per product.
#pragma once
#include <cuda_fp16.h>

#include "ptx.cuh"

namespace eas {

enum : uint32_t { DEV_ERR_CACHE_RANGE = 3 };     // a block number or a place outside the cache
constexpr float kCacheMinScale = 7.888609052210118e-31f;   // 2^-100: blocks of zeros, and no division by a subnormal scale

// Tables, lengths, starts and scales are read by ordinary loads: an earlier kernel may still be writing them when this one starts, and a load of the
// read-only path promises that nobody does while the kernel runs, so that nothing keeps it behind the wait for that kernel.
struct CacheView {
  int8_t *k, *v;
  float *k_scale, *v_scale;
  int n_blocks, n_kv, bs_log2;
};
struct CacheSeqs {
  const int32_t *table, *cu, *start;
  long long ld_table;
  int n_seqs, max_blocks;
};

__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t code) { atomicCAS(status, DEV_OK, code); }

template <typename T> struct Pair16;
template <> struct Pair16<bf16> {
  static __device__ __forceinline__ float lo(uint32_t w) { return bf16_lo(w); }
  static __device__ __forceinline__ float hi(uint32_t w) { return bf16_hi(w); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
};
template <> struct Pair16<__half> {
  static __device__ __forceinline__ float lo(uint32_t w) { return __half2float(__ushort_as_half(static_cast<unsigned short>(w & 0xFFFFu))); }
  static __device__ __forceinline__ float hi(uint32_t w) { return __half2float(__ushort_as_half(static_cast<unsigned short>(w >> 16))); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
__device__ __forceinline__ float load16(uint16_t x, bool fp16) {
  return fp16 ? __half2float(__ushort_as_half(x)) : __uint_as_float(static_cast<uint32_t>(x) << 16);
}

// ------------------------------------------------------------------------------------------------ store, load
struct CacheRowsParams {
  CacheView c;
  CacheSeqs s;
  void *k, *v;            // [n_rows][n_kv * head_dim] (store: read, load: written)
  long long ld_k, ld_v;
  int n_rows;
  long long units;        // store: pair numbers x heads x {keys, values}
  uint32_t* status;
  int early_launch;
};

// Storing walks (sequence, block) pairs.  How many blocks a sequence touches is only known on the device, so a pair has a number that the
// host can bound: sequence s owns the numbers from floor(cu[s] / bs) + 2 s on.  A run of n tokens touches at most
// floor(n / bs) + 2 blocks and floor(a / bs) + floor(n / bs) <= floor((a + n) / bs), so the ranges never overlap, and
// all numbers are below floor(n_rows / bs) + 2 n_seqs.
struct CacheRun {         // the part of a sequence's rows that lies in one block
  int block;              // -1: none
  int lo, hi;             // places in the block
  int row;                // row of place lo
};
__device__ __forceinline__ CacheRun cache_run(const CacheRowsParams& p, int pair, bool report) {
  CacheRun r;
  r.block = -1;
  auto cu = [&](int i) { return min(max(p.s.cu[i], 0), p.n_rows); };
  int lo = 0, hi = p.s.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((cu(mid) >> p.c.bs_log2) + 2 * mid <= pair) lo = mid; else hi = mid - 1;
  }
  const int c0 = cu(lo), len = cu(lo + 1) - c0, j = pair - ((c0 >> p.c.bs_log2) + 2 * lo);
  if (len <= 0 || j < 0) return r;
  const long long at = p.s.start[lo], end = at + len;
  if (at < 0) {
    if (report && j == 0) raise_status(p.status, DEV_ERR_CACHE_RANGE);
    return r;
  }
  const long long b = (at >> p.c.bs_log2) + j, b0 = b << p.c.bs_log2;
  if (b0 >= end) return r;
  int block = -1;
  if (b < p.s.max_blocks) block = p.s.table[lo * p.s.ld_table + b];
  if (block < 0 || block >= p.c.n_blocks) {
    if (report) raise_status(p.status, DEV_ERR_CACHE_RANGE);
    return r;
  }
  r.block = block;
  r.lo = static_cast<int>(max(at - b0, 0LL));
  r.hi = static_cast<int>(min(end - b0, 1LL << p.c.bs_log2));
  r.row = c0 + static_cast<int>(b0 + r.lo - at);
  return r;
}

// The nearest integer to x / s (ties to even) in the low byte.  x * inv is off by a few 2^-24 relative, so its floor k is right or one
// off where x / s lies next to an integer, and in both cases the answer is k or k + 1; which, says the sign of
// x - (k + 1/2) s, and one fma gives that sign exactly (k + 1/2 has 8 bits; the difference, if not 0, is far above the subnormals for s >= 2^-100).
__device__ __forceinline__ uint32_t quantise(float x, float s, float inv) {
  const float k = floorf(x * inv);
  const float d = fmaf(-(k + 0.5f), s, x);
  const uint32_t kb = __float_as_uint(k + 12582912.0f);          // 1.5 * 2^23: k in the low bits, two's complement
  return kb + ((d > 0.0f || (d == 0.0f && (kb & 1u))) ? 1u : 0u);
}
// Eight values (four words of two) to eight numbers.  The rounded product is the answer wherever it is not within 2^-15 of a tie (it is off by
// less than 127 * 2^-22); only then the exact test above decides.
template <typename T>
__device__ __forceinline__ uint2 quantise8(const uint4& x, float s, float inv) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const uint64_t inv2 = pack2(inv, inv), magic = pack2(12582912.0f, 12582912.0f), less = pack2(-12582912.0f, -12582912.0f), minus = pack2(-1.0f, -1.0f);
  uint32_t q[8];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t r = fmul2(pack2(Pair16<T>::lo(w[i]), Pair16<T>::hi(w[i])), inv2);
    const uint64_t t = fadd2(r, magic);                          // the nearest integer in the low bits
    float a, b, d0, d1;
    unpack2(t, a, b);
    unpack2(ffma2(fadd2(t, less), minus, r), d0, d1);
    off = fmax3(off, fabsf(d0), fabsf(d1));
    q[2 * i] = __float_as_uint(a);
    q[2 * i + 1] = __float_as_uint(b);
  }
  if (__builtin_expect(off > 0.5f - 3.0517578125e-05f, 0)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[2 * i] = quantise(Pair16<T>::lo(w[i]), s, inv);
      q[2 * i + 1] = quantise(Pair16<T>::hi(w[i]), s, inv);
    }
  }
  return make_uint2(__byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410));
}
// The same for a number that is in the block already: number * old / s.  The product has too many bits for one fma, so what comes
// within 2^-10 of a tie is decided in fp64 (31 by 24 bits: the rounded quotient is a tie exactly where the true one is).
__device__ __forceinline__ uint32_t requantise(int q, float old, float s, float ratio) {
  const float r = static_cast<float>(q) * ratio;
  float n = rintf(r);
  if (fabsf(fabsf(r - n) - 0.5f) < 0.0009765625f) n = static_cast<float>(rint(static_cast<double>(q) * old / s));
  return __float_as_uint(n + 12582912.0f);
}

// GT threads per (sequence, block, head, keys or values): the largest magnitude of the new rows, the scale, the numbers.  Memory-bound: 2 bytes
// read and 1 written per value.  A thread holds all of its values, at most 8 loads of 16 bytes (GT = block_size * head_dim / 64): they are all
// in flight at once, 64 KB an SM, and are read once.  6227 tokens of 8 heads of 128 into blocks of 64 take 12 us, 16384 32 (half the copy rate: a group
// goes from one unit to the next in series).  (One warp per block, reading the rows twice in four trips each: 6227 tokens in and out again 46 instead of 25.)
template <int HD, int GT, typename T>
__global__ void __launch_bounds__(512, 1) cache_store_kernel(const __grid_constant__ CacheRowsParams p) {
  __shared__ uint32_t group_max[32];
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  constexpr int kChunks = HD / 8, kRows = GT / kChunks, kSteps = 8;      // threads per row (8 values each), rows per step, steps of the largest block
  const int tid = threadIdx.x % GT, group = threadIdx.x / GT, lane = threadIdx.x & 31;
  const int chunk = tid % kChunks, sub = tid / kChunks;
  const long long groups = static_cast<long long>(gridDim.x) * (blockDim.x / GT);
  for (long long u = static_cast<long long>(blockIdx.x) * (blockDim.x / GT) + group; u < p.units; u += groups) {
    const bool values = u & 1;
    const int pair_head = static_cast<int>(u >> 1), head = pair_head % p.c.n_kv;
    const CacheRun r = cache_run(p, pair_head / p.c.n_kv, tid == 0 && head == 0 && !values);
    if (r.block < 0) continue;
    const long long ld = values ? p.ld_v : p.ld_k;
    const T* src = static_cast<const T*>(values ? p.v : p.k) + static_cast<long long>(r.row) * ld + head * HD + chunk * 8;
    const long long at = static_cast<long long>(r.block) * p.c.n_kv + head;
    float* scale = (values ? p.c.v_scale : p.c.k_scale) + at;
    int8_t* dst = (values ? p.c.v : p.c.k) + ((at << p.c.bs_log2) * HD);
    const int n = r.hi - r.lo;
    uint4 x[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (sub + i * kRows < n) x[i] = *reinterpret_cast<const uint4*>(src + (sub + i * kRows) * ld);
    }
    const float old = r.lo > 0 ? *scale : 0.0f;
    // magnitudes compare as integers, with Inf above every number and NaN above Inf
    uint32_t m2 = 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu), __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu)));
    uint32_t m = __reduce_max_sync(0xffffffffu, max(m2 & 0xFFFFu, m2 >> 16));
    if constexpr (GT > 32) {
      if (lane == 0) group_max[threadIdx.x >> 5] = m;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GT) : "memory");
      m = group_max[(group * GT >> 5) + (lane & (GT / 32 - 1))];
      m = __reduce_max_sync(0xffffffffu, m);
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GT) : "memory");      // read by all (and the old scale, before it is overwritten)
    } else {
      __syncwarp();
    }
    float s = __fdiv_rn(Pair16<T>::lo(m), 127.0f);
    if (s < kCacheMinScale) s = kCacheMinScale;
    if (!(s * 0.0f == 0.0f)) s = __uint_as_float(0x7FFFFFFFu);     // Inf or NaN among the values: the block and head reads as NaN
    if (r.lo > 0) {
      if (!(s <= old) && old == old) {                           // the scale grows (or stops being a number)
        const float ratio = __fdiv_rn(old, s);
        constexpr int kLanes = HD / 16;
        for (int t = tid / kLanes; t < r.lo; t += GT / kLanes) {
          uint4* w = reinterpret_cast<uint4*>(dst + t * HD + (tid % kLanes) * 16);
          const uint4 y = *w;
          uint32_t yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t z = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b)
              z |= (requantise(static_cast<int8_t>(yw[i] >> (8 * b)), old, s, ratio) & 0xFFu) << (8 * b);
            yw[i] = z;
          }
          *w = make_uint4(yw[0], yw[1], yw[2], yw[3]);
        }
      } else {
        s = old;
      }
    }
    const float inv = __fdiv_rn(1.0f, s);
    int8_t* out = dst + (r.lo + sub) * HD + chunk * 8;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (sub + i * kRows < n) *reinterpret_cast<uint2*>(out + i * kRows * HD) = quantise8<T>(x[i], s, inv);
    }
    if (tid == 0) *scale = s;
  }
}

// Four numbers (bytes of x, two's complement) times the scale, rounded to the data type.  0x4B000000 | (byte ^ 0x80) is 2^23 + 128 + number as
// fp32, so the number is exact and the product the one fp32 rounding of number * scale.
template <typename T>
__device__ __forceinline__ uint2 dequantise4(uint32_t x, uint64_t scale2) {
  x ^= 0x80808080u;
  const uint64_t less = pack2(-8388736.0f, -8388736.0f);
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint64_t raw = pack2(__uint_as_float(__byte_perm(x, 0x4B000000u, 0x7440 | i)), __uint_as_float(__byte_perm(x, 0x4B000000u, 0x7441 | i)));
    unpack2(fmul2(fadd2(raw, less), scale2), f[i], f[i + 1]);
  }
  return make_uint2(Pair16<T>::pack(f[0], f[1]), Pair16<T>::pack(f[2], f[3]));
}

// A warp takes a stretch of neighbouring rows of k and of v, and of it the runs that lie in one block each.  Memory-bound: 1 byte read and 2
// written per value; rows are written whole, and two rows of keys and values are in flight (16 loads of 8 values a lane).  (One warp per
// block and head: 43 us instead of 23 for 19993 tokens of 8 heads of 128.)
template <int HD, typename T>
__global__ void __launch_bounds__(512, 1) cache_load_kernel(const __grid_constant__ CacheRowsParams p) {
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  constexpr int kChunks = HD / 8, kBatch = 4;                    // 8 values each; 128 chunks of a row at a time
  const int lane = threadIdx.x & 31, row_chunks = p.c.n_kv * kChunks;
  const int warps = gridDim.x * (blockDim.x >> 5), me = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  auto cu = [&](int i) { return min(max(p.s.cu[i], 0), p.n_rows); };
  const int begin = static_cast<int>(static_cast<long long>(p.n_rows) * me / warps);
  const int end = static_cast<int>(static_cast<long long>(p.n_rows) * (me + 1) / warps);
  if (begin >= end) return;
  int s = 0, hi = p.s.n_seqs - 1;
  while (s < hi) {                                               // the last sequence that begins at or before the first row
    const int mid = (s + hi + 1) >> 1;
    if (cu(mid) <= begin) s = mid; else hi = mid - 1;
  }
  for (int row = begin; row < end;) {
    while (row >= cu(s + 1) && s + 1 < p.s.n_seqs) ++s;
    const int first = cu(s), next = min(cu(s + 1), end);
    if (row < first || row >= next) {                            // a row of no sequence
      ++row;
      continue;
    }
    const long long at = p.s.start[s] + static_cast<long long>(row - first), b = at >> p.c.bs_log2;
    const int place = static_cast<int>(at) & ((1 << p.c.bs_log2) - 1), n = min(next - row, (1 << p.c.bs_log2) - place);
    int block = -1;
    if (at >= 0 && b < p.s.max_blocks) block = p.s.table[s * p.s.ld_table + b];
    if (block < 0 || block >= p.c.n_blocks) {
      if (lane == 0) raise_status(p.status, DEV_ERR_CACHE_RANGE);
      row += n;
      continue;
    }
    const long long block0 = static_cast<long long>(block) * p.c.n_kv;
    for (int base = lane; base < row_chunks; base += 32 * kBatch) {
      const int8_t *k[kBatch], *v[kBatch];
      uint64_t ks[kBatch], vs[kBatch];
      bool there[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int c = base + 32 * i, head = c / kChunks;
        there[i] = c < row_chunks;
        const long long from = (((block0 + head) << p.c.bs_log2) + place) * HD + c % kChunks * 8;
        k[i] = p.c.k + from;
        v[i] = p.c.v + from;
        const float x = there[i] ? p.c.k_scale[block0 + head] : 0.f, y = there[i] ? p.c.v_scale[block0 + head] : 0.f;
        ks[i] = pack2(x, x);
        vs[i] = pack2(y, y);
      }
      T *to_k = static_cast<T*>(p.k) + row * p.ld_k + base * 8, *to_v = static_cast<T*>(p.v) + row * p.ld_v + base * 8;
      auto fetch = [&](int t, uint2 (&x)[2 * kBatch]) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (there[i]) {
            x[i] = *reinterpret_cast<const uint2*>(k[i] + t * HD);
            x[kBatch + i] = *reinterpret_cast<const uint2*>(v[i] + t * HD);
          }
      };
      auto put = [&](const uint2 (&x)[2 * kBatch]) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (there[i]) {
            const uint2 a = dequantise4<T>(x[i].x, ks[i]), b2 = dequantise4<T>(x[i].y, ks[i]);
            *reinterpret_cast<uint4*>(to_k + i * 256) = make_uint4(a.x, a.y, b2.x, b2.y);
            const uint2 c = dequantise4<T>(x[kBatch + i].x, vs[i]), d = dequantise4<T>(x[kBatch + i].y, vs[i]);
            *reinterpret_cast<uint4*>(to_v + i * 256) = make_uint4(c.x, c.y, d.x, d.y);
          }
        to_k += p.ld_k;
        to_v += p.ld_v;
      };
      uint2 x[2 * kBatch], y[2 * kBatch];
      int t = 0;
#pragma unroll 1
      for (; t + 1 < n; t += 2) {
        fetch(t, x);
        fetch(t + 1, y);
        put(x);
        put(y);
      }
      if (t < n) {
        fetch(t, x);
        put(x);
      }
    }
    row += n;
  }
}

}  // namespace eas
