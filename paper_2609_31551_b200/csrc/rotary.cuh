// Rotary positions with several axes, alone and on the way into the 8-bit cache.
//
// Pair i of a head (two dimensions a, b of the first rotary_dim) turns by angle = positions[axis i][token] * inv_freq[i]:
//   a' = scale (a cos - b sin),  b' = scale (b cos + a sin)
// fp32 loses the angles of far positions (a position of 700000 is known to 0.03 rad), fp64 costs 64 times as much.  So angles are whole numbers: with
// F = round(inv_freq / 2 pi * 2^64), position * F mod 2^64 is the angle in turns of 2^-64, exactly but for the rounding of F, which a position below 2^31
// makes 2^-34 turns.  Of those the upper 32 bits count.
#pragma once
#include <type_traits>

#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

constexpr int kRotaryMaxPairs = 64, kRotaryMaxAxes = 4;

struct RotaryTable {                      // (kernel parameter)
  uint32_t f_lo[kRotaryMaxPairs], f_hi[kRotaryMaxPairs];
  uint8_t axis[kRotaryMaxPairs];
  int pairs, neighbours;
  float scale;
};

// A thread's pair: which it works out cosines and sines of, for any number of rows.  (Taken from the parameters once: threads that read different ones go one after the
// other, which for every row was two thirds of the time.)
struct RotaryPair {
  uint32_t f_lo, f_hi;
  int axis;
  int at;                                 // place in a row's table (below); -1: none
  __device__ __forceinline__ RotaryPair(const RotaryTable& t, int pair) {
    const int i = min(pair, t.pairs - 1);
    f_lo = t.f_lo[i];
    f_hi = t.f_hi[i];
    axis = t.axis[i];
    at = pair < t.pairs ? rotary_place(i, t.pairs) : -1;
  }
  __device__ __forceinline__ void put(float* row, float2 turn) const {
    row[at] = turn.x;
    row[at + 2] = turn.y;
  }
  // The table of a row: 8 pairs an item (16 dimensions), as four float4, cosines and sines of two pairs; those of all items side by side, so that threads of
  // neighbouring items read side by side
  static __device__ __forceinline__ int rotary_place(int pair, int pairs) { return ((pair >> 1) & 3) * (pairs >> 1) + (pair >> 3) * 4 + (pair & 1); }
};
// cosine and sine of a pair's angle at a position, times the scale (the sine's is negative where the rotation is taken back).  The turn's upper bits are the nearest
// quarter, the rest an angle within pi / 4, for which the Taylor sums up to x^9 and x^8 are off by less than 2^-29 and 2^-25.
__device__ __forceinline__ float2 rotary_turn(const RotaryPair& f, int position, float scale, float sin_scale) {
  const uint32_t p = static_cast<uint32_t>(position);
  const uint32_t turn = p * f.f_hi + __umulhi(p, f.f_lo) - (position < 0 ? f.f_lo : 0u);      // bits 32 .. 63 of position * F
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(turn - (quarter << 30))) * 1.4629180792671596e-09f;      // 2 pi 2^-32
  const float x2 = x * x;
  float s = fmaf(fmaf(fmaf(2.7557319223985893e-06f, x2, -1.9841269841269841e-04f), x2, 8.3333333333333333e-03f), x2, -1.6666666666666667e-01f);
  s = fmaf(x * x2, s, x);
  const float c = fmaf(fmaf(fmaf(fmaf(2.4801587301587302e-05f, x2, -1.3888888888888889e-03f), x2, 4.1666666666666667e-02f), x2, -0.5f), x2, 1.0f);
  const bool swap = quarter & 1u;
  const float cs = swap ? s : c, sn = swap ? c : s;              // of the angle: quarter 0 (c, s), 1 (-s, c), 2 (-c, -s), 3 (s, -c)
  return make_float2((quarter + 1u) & 2u ? -cs * scale : cs * scale, quarter & 2u ? -sn * sin_scale : sn * sin_scale);
}

struct RotaryRows {
  const void *q, *k;
  void *out_q, *out_k;
  long long ld_q, ld_k, ld_out_q, ld_out_k;
  const int32_t* positions;
  long long ld_positions;
  int n_rows, n_heads, n_kv;
  int inverse;
  int in_place;                           // outputs lie where the inputs do: what is not rotated stays
};

// 16 dimensions of a head, as two words of 8: with halves, item c < pairs / 8 is the first halves 8 c .. of the pairs and the second ones; everything else
// is 16 dimensions side by side.
__device__ __forceinline__ int2 rotary_at(int c, int pairs, int neighbours) {
  return !neighbours && 8 * c < pairs ? make_int2(8 * c, pairs + 8 * c) : make_int2(16 * c, 16 * c + 8);
}
// the 16 values of a rotated item, turned by its 8 pairs' cosines and sines (cs: the item's first two in the row's table of `items` items)
template <typename T>
__device__ __forceinline__ void rotary_turn_16(const uint4& lo, const uint4& hi, const float4* cs, int items, int neighbours, float (&y)[16]) {
  const uint32_t a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {           // two pairs
    const float4 t = cs[i * items];
    const uint64_t cos2 = pack2(t.x, t.y), sin2 = pack2(t.z, t.w), minus2 = pack2(-t.z, -t.w);
    uint64_t u, v;                        // the pairs' first and second values
    if (neighbours) {
      const uint32_t w0 = i < 2 ? a[2 * i] : b[2 * i - 4], w1 = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
      u = pack2(Pair16<T>::lo(w0), Pair16<T>::lo(w1));
      v = pack2(Pair16<T>::hi(w0), Pair16<T>::hi(w1));
    } else {
      u = pack2(Pair16<T>::lo(a[i]), Pair16<T>::hi(a[i]));
      v = pack2(Pair16<T>::lo(b[i]), Pair16<T>::hi(b[i]));
    }
    const uint64_t u_new = ffma2(u, cos2, fmul2(v, minus2)), v_new = ffma2(v, cos2, fmul2(u, sin2));
    if (neighbours) {
      unpack2(u_new, y[4 * i], y[4 * i + 2]);
      unpack2(v_new, y[4 * i + 1], y[4 * i + 3]);
    } else {
      unpack2(u_new, y[2 * i], y[2 * i + 1]);
      unpack2(v_new, y[8 + 2 * i], y[9 + 2 * i]);
    }
  }
}

// One token's heads [head0, head1) of queries and keys side by side (keys behind the queries), by a warp.  cs: the warp's 64 cosines and sines.
template <int HD, int BATCH, typename T>
__device__ __forceinline__ void rotary_row(const RotaryTable& t, const RotaryRows& r, const RotaryPair (&pair)[2], int row, int head0, int head1, const int (&position)[2],
                                           float2* cs) {
  constexpr int ITEMS = HD / 16, LANES = 32 / ITEMS;                     // items a head, heads a warp takes at once (BATCH times that are in flight)
  const int lane = threadIdx.x & 31, item = lane % ITEMS, sub = lane / ITEMS;
  const bool turned = 8 * item < t.pairs;
  const int2 at = rotary_at(item, t.pairs, t.neighbours);
  auto from = [&](int h) {
    return h < r.n_heads ? static_cast<const T*>(r.q) + row * r.ld_q + h * HD : static_cast<const T*>(r.k) + row * r.ld_k + (h - r.n_heads) * HD;
  };
  auto to = [&](int h) {
    return h < r.n_heads ? static_cast<T*>(r.out_q) + row * r.ld_out_q + h * HD : static_cast<T*>(r.out_k) + row * r.ld_out_k + (h - r.n_heads) * HD;
  };
  bool first = true;
  for (int h0 = head0; h0 < head1; h0 += LANES * BATCH) {
    uint4 lo[BATCH], hi[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * LANES + sub;
      lo[i] = hi[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h < head1 && (turned || !r.in_place)) {
        const T* src = from(h);
        lo[i] = *reinterpret_cast<const uint4*>(src + at.x);
        hi[i] = *reinterpret_cast<const uint4*>(src + at.y);
      }
    }
    if (first) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (pair[i].at >= 0) pair[i].put(reinterpret_cast<float*>(cs), rotary_turn(pair[i], position[i], t.scale, r.inverse ? -t.scale : t.scale));
      }
      __syncwarp();
      first = false;
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * LANES + sub;
      if (h >= head1 || (!turned && r.in_place)) continue;
      T* dst = to(h);
      if (turned) {
        float y[16];
        rotary_turn_16<T>(lo[i], hi[i], reinterpret_cast<const float4*>(cs) + item, t.pairs >> 3, t.neighbours, y);
        lo[i] = make_uint4(Pair16<T>::pack(y[0], y[1]), Pair16<T>::pack(y[2], y[3]), Pair16<T>::pack(y[4], y[5]), Pair16<T>::pack(y[6], y[7]));
        hi[i] = make_uint4(Pair16<T>::pack(y[8], y[9]), Pair16<T>::pack(y[10], y[11]), Pair16<T>::pack(y[12], y[13]), Pair16<T>::pack(y[14], y[15]));
      }
      *reinterpret_cast<uint4*>(dst + at.x) = lo[i];
      *reinterpret_cast<uint4*>(dst + at.y) = hi[i];
    }
  }
}

struct RotaryParams {
  RotaryTable t;
  RotaryRows r;
  uint32_t parts;                         // a token's heads in `parts` pieces of part_heads
  int part_heads;
  int early_launch;
};

constexpr int kRotaryThreads = 512, kRotaryBatch = 4;

template <int HD, typename T>
__global__ void __launch_bounds__(kRotaryThreads, 1) rotary_kernel(const __grid_constant__ RotaryParams p) {
  __shared__ __align__(16) float2 table[kRotaryThreads / 32][kRotaryMaxPairs];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const RotaryPair pair[2] = {{p.t, lane}, {p.t, lane + 32}};
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  const uint32_t units = static_cast<uint32_t>(p.r.n_rows) * p.parts, step = gridDim.x * (blockDim.x >> 5);      // (below 2^31)
  const int heads = p.r.n_heads + p.r.n_kv;
  auto position_of = [&](uint32_t u, int (&position)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      position[i] = u < units && pair[i].at >= 0 ? p.r.positions[pair[i].axis * p.r.ld_positions + u / p.parts] : 0;
  };
  int position[2];
  uint32_t u = blockIdx.x * (blockDim.x >> 5) + warp;
  position_of(u, position);
  for (; u < units; u += step) {
    int next[2];
    position_of(u + step, next);
    const int row = static_cast<int>(u / p.parts), head0 = static_cast<int>(u - row * p.parts) * p.part_heads;
    rotary_row<HD, kRotaryBatch, T>(p.t, p.r, pair, row, head0, min(head0 + p.part_heads, heads), position, table[warp]);
    position[0] = next[0];
    position[1] = next[1];
  }
}

// ------------------------------------------------------------------------------------------------ append
struct AppendParams {
  CacheView c;
  CacheSeqs s;
  RotaryTable t;
  RotaryRows r;                           // n_kv: 0 (the keys' rotated form goes to the cache only); positions null: a token's place in its sequence
  const void* v;
  long long ld_v;
  int pairs;                              // numbers of (sequence, block) pairs (see cache_run)
  int pairs_log2;                         // of the next power of two from the rotated pairs on
  int head_parts, part_heads;             // key/value heads of a pair in pieces
  uint32_t q_parts;                       // query heads of a token in pieces
  int q_part_heads;
  uint32_t* status;
  int early_launch;
};

constexpr int kAppendThreads = 256, kAppendCtas = 3, kAppendSteps = 2, kAppendBatch = 2;      // CTAs an SM: one's loads beside the others' arithmetic

// Eight fp32 values to eight numbers, as quantise8 does it
__device__ __forceinline__ uint2 quantise8_fp32(const float* y, float s, float inv) {
  const uint64_t inv2 = pack2(inv, inv), magic = pack2(12582912.0f, 12582912.0f), less = pack2(-12582912.0f, -12582912.0f), minus = pack2(-1.0f, -1.0f);
  uint32_t q[8];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t r = fmul2(pack2(y[i], y[i + 1]), inv2);
    const uint64_t t = fadd2(r, magic);                            // the nearest integer in the low bits
    float a, b, d0, d1;
    unpack2(t, a, b);
    unpack2(ffma2(fadd2(t, less), minus, r), d0, d1);
    off = fmax3(off, fabsf(d0), fabsf(d1));
    q[i] = __float_as_uint(a);
    q[i + 1] = __float_as_uint(b);
  }
  if (__builtin_expect(off > 0.5f - 3.0517578125e-05f, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quantise(y[i], s, inv);
  }
  return make_uint2(__byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410));
}

// An item is the run of one sequence's new rows that lies in one block, and some of its key/value heads: the cosines and sines of the run's rows go to
// shared memory once for all of them.  GT: threads of a head's keys or values, a warp where runs have a few rows (decoding steps, drafts).  Behind those items the queries: a warp takes a token's heads, or some of them.
template <int HD, int GT, typename T>
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas) cache_append_kernel(const __grid_constant__ AppendParams p) {
  extern __shared__ __align__(16) float2 append_turns[];
  __shared__ uint32_t group_max[32];
  constexpr int ITEMS = HD / 16, ROWS = GT / ITEMS, STEPS = kAppendSteps, CAP = STEPS * ROWS;
  const int tid = threadIdx.x % GT, group = threadIdx.x / GT, item = tid % ITEMS, sub = tid / ITEMS;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const RotaryPair q_pair[2] = {{p.t, lane}, {p.t, lane + 32}};
  const int pairs_log2 = p.pairs_log2, my_row = threadIdx.x >> pairs_log2;
  const RotaryPair k_pair(p.t, threadIdx.x & ((1 << pairs_log2) - 1));
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  auto cu = [&](int i) { return min(max(p.s.cu[i], 0), p.r.n_rows); };
  const int pair_items = p.pairs * p.head_parts;
  const uint32_t q_units = static_cast<uint32_t>(p.r.n_heads > 0 ? p.r.n_rows : 0) * p.q_parts;
  const uint32_t items = pair_items + (q_units + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
  for (uint32_t it = blockIdx.x; it < items; it += gridDim.x) {
    if (it >= static_cast<uint32_t>(pair_items)) {
      const uint32_t u = (it - pair_items) * (kAppendThreads / 32) + warp;
      __syncthreads();                                             // (the table in shared memory is no longer read)
      if (u >= q_units) continue;
      const int row = static_cast<int>(u / p.q_parts), head0 = static_cast<int>(u - row * p.q_parts) * p.q_part_heads;
      if (row < cu(0) || row >= cu(p.s.n_seqs)) continue;
      int position[2] = {0, 0};
      if (p.r.positions == nullptr) {
        const int s = last_sequence(p.s.n_seqs, row, cu);
        position[0] = position[1] = static_cast<int>(static_cast<uint32_t>(p.s.start[s]) + static_cast<uint32_t>(row - cu(s)));
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (q_pair[i].at >= 0) position[i] = p.r.positions[q_pair[i].axis * p.r.ld_positions + row];
      }
      rotary_row<HD, kAppendBatch, T>(p.t, p.r, q_pair, row, head0, min(head0 + p.q_part_heads, p.r.n_heads), position, append_turns + warp * kRotaryMaxPairs);
      continue;
    }
    const int pair = static_cast<int>(it) / p.head_parts, part = static_cast<int>(it) - pair * p.head_parts;
    const CacheRun r = cache_run_of(p.c, p.s, last_sequence(p.s.n_seqs, pair, [&](int i) { return (cu(i) >> p.c.bs_log2) + 2 * i; }), p.r.n_rows, pair, p.status,
                                    threadIdx.x == 0 && part == 0);
    if (r.block < 0) continue;
    const int n = r.hi - r.lo;
    // The keys or the values of one head at a time by THREADS threads, 2 rows of 16 dimensions a thread, rotated in fp32 and rounded once, to the number; then the
    // block's scale and numbers as in cache_store_kernel.  (Four rows a thread do not fit the registers of two CTAs an SM.)  A run of more rows than the threads have
    // takes several rounds, and all but the last are read again for their numbers.
    {
      const int units = 2 * min(p.part_heads, p.c.n_kv - part * p.part_heads), rounds = (n + CAP - 1) / CAP;
#pragma unroll 1
      for (int u = group, first = 1; u < units || first; u += kAppendThreads / GT, first = 0) {
        const bool values = u & 1, turned = !values && 8 * item < p.t.pairs;
        const int head = part * p.part_heads + (u >> 1);
        const long long ld = values ? p.ld_v : p.r.ld_k, at = static_cast<long long>(r.block) * p.c.n_kv + head;
        const T* src = static_cast<const T*>(values ? p.v : p.r.k) + static_cast<long long>(r.row + sub) * ld + head * HD;
        const int2 dims = values ? make_int2(16 * item, 16 * item + 8) : rotary_at(item, p.t.pairs, p.t.neighbours);
        float* scale = (values ? p.c.v_scale : p.c.k_scale) + at;
        int8_t* dst = (values ? p.c.v : p.c.k) + ((at << p.c.bs_log2) * HD);
        uint4 x[2 * STEPS];
        float y[STEPS][16];
        auto load = [&](int row0) {                                // rows row0 + sub, ...
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            x[2 * i] = x[2 * i + 1] = make_uint4(0u, 0u, 0u, 0u);
            if (u < units && row0 + sub + i * ROWS < n) {
              x[2 * i] = *reinterpret_cast<const uint4*>(src + (row0 + i * ROWS) * ld + dims.x);
              x[2 * i + 1] = *reinterpret_cast<const uint4*>(src + (row0 + i * ROWS) * ld + dims.y);
            }
          }
        };
        auto turn = [&](int row0) {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            if (turned && row0 + sub + i * ROWS < n) {
              rotary_turn_16<T>(x[2 * i], x[2 * i + 1], reinterpret_cast<const float4*>(append_turns + (row0 + sub + i * ROWS) * p.t.pairs) + item, p.t.pairs >> 3, p.t.neighbours, y[i]);
            } else {
              const uint32_t w[8] = {x[2 * i].x, x[2 * i].y, x[2 * i].z, x[2 * i].w, x[2 * i + 1].x, x[2 * i + 1].y, x[2 * i + 1].z, x[2 * i + 1].w};
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                y[i][2 * e] = Pair16<T>::lo(w[e]);
                y[i][2 * e + 1] = Pair16<T>::hi(w[e]);
              }
            }
          }
        };
        load(0);
        const float old = r.lo > 0 && u < units ? *scale : 0.0f;
        if (first) {                                               // (beside the first loads)
          __syncthreads();                                         // (the last item's table is no longer read)
          if (k_pair.at >= 0)
            for (int j = my_row; j < n; j += kAppendThreads >> pairs_log2) {
              const int position = p.r.positions == nullptr ? r.place + j : p.r.positions[k_pair.axis * p.r.ld_positions + r.row + j];
              k_pair.put(reinterpret_cast<float*>(append_turns + j * p.t.pairs), rotary_turn(k_pair, position, p.t.scale, p.t.scale));
            }
          __syncthreads();
          if (u >= units) break;
        }
        // the largest magnitude: of Inf and NaN by 16-bit integers, which order Inf above every number and NaN above Inf
        uint32_t m2 = 0;
        float largest = 0.f;
#pragma unroll 1
        for (int round = 0; round < rounds; ++round) {
          if (round > 0) load(round * CAP);
#pragma unroll
          for (int i = 0; i < 2 * STEPS; ++i)
            m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu), __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu)));
          turn(round * CAP);
#pragma unroll
          for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 2) largest = fmax3(largest, fabsf(y[i][e]), fabsf(y[i][e + 1]));
        }
        const float whole = Pair16<T>::lo(max(m2 & 0xFFFFu, m2 >> 16));
        uint32_t m = __float_as_uint(whole * 0.f == 0.f ? largest : whole);
        m = __reduce_max_sync(0xffffffffu, m);
        if constexpr (GT > 32) {
          if (lane == 0) group_max[warp] = m;
          asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GT) : "memory");
          m = group_max[(group * GT >> 5) + (lane & (GT / 32 - 1))];
          m = __reduce_max_sync(0xffffffffu, m);
          asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GT) : "memory");      // read by all (and the old scale, before it is overwritten)
        } else {
          __syncwarp();
        }
        bool grows;
        const float s = cache_new_scale(__uint_as_float(m), old, r.lo, grows);
        if (grows) cache_requantise_apart<HD, GT>(old, s, r.lo, dst, tid);
        const float inv = __fdiv_rn(1.0f, s);
        int8_t* out = dst + (r.lo + sub) * HD;
#pragma unroll 1
        for (int round = rounds - 1; round >= 0; --round) {        // (the last round's values are at hand)
          if (round < rounds - 1) {
            load(round * CAP);
            turn(round * CAP);
          }
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            const int j = round * CAP + i * ROWS;
            if (sub + j < n) {
              *reinterpret_cast<uint2*>(out + j * HD + dims.x) = quantise8_fp32(y[i], s, inv);
              *reinterpret_cast<uint2*>(out + j * HD + dims.y) = quantise8_fp32(y[i] + 8, s, inv);
            }
          }
        }
        if (tid == 0) *scale = s;
      }
    }
  }
}

}  // namespace eas
