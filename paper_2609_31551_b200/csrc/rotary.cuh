// Rotary positions with several axes, alone and on the way into the 8-bit cache.
//
// Pair i of a head (two dimensions a, b of the first rotary_dim) turns by angle = positions[axis i][token] * inv_freq[i]:
//   a' = scale (a cos - b sin),  b' = scale (b cos + a sin)
// fp32 loses the angles of far positions (a position of 700000 is known to 0.03 rad), fp64 costs 64 times as much.  So angles are whole numbers: with
// F = round(inv_freq / 2 pi * 2^64), position * F mod 2^64 is the angle in turns of 2^-64, exactly but for the rounding of F, which a position below 2^31
// makes 2^-34 turns.  Of those the upper 32 bits count.
//
// Alone, the rotation is a copy: a warp takes a token's heads, 32 bytes a lane and head, 16 heads of 128 (32 of 64) in flight; cosines and sines are worked out
// once a token (64 pairs, two a lane) into 512 bytes of shared memory.  16384 tokens of 32 and 8 heads of 128 54.6 us, 6.14 TB/s, 94 % of the copy rate; 6
// prompts of 6227 tokens 23.7; 40 tokens 2.3 (one launch).
// On the way into the cache (append), a block's run of new rows has its cosines worked out once for all heads (8 bytes a pair and row of shared memory, 32 KB
// for 64 rows of 64 pairs), is read once, rotated in fp32 and rounded once, to its number; queries go warp by warp behind.  16384 tokens 88 us, 4.2 TB/s (a
// launch of its own for the queries: 93; rotation and storing as two operators, with the rotated keys through memory: 86, less exact), 6 prompts of 6227 tokens
// 43, 64 single tokens 7.8 (7.0 with queries dealt to whole CTAs, when 16384 tokens took 111).  Of the 88, 50 are keys and values: a group of threads goes from
// head to head in series, 16 warps an SM (registers), and waits for loads 3 of 9 cycles an instruction.
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

// A thread's pair: which it works out cosines and sines of, for any number of rows.  (Taken from the parameters once: threads that read different ones go one
// after the other, which for every row was two thirds of the time.)
struct RotaryPair {
  uint32_t f_lo, f_hi;
  int axis;
  int at;                                 // place in a row's table (below); -1: none
  __device__ __forceinline__ RotaryPair(const RotaryTable& t, int pair) {
    const int i = min(pair, t.pairs - 1);
    f_lo = t.f_lo[i];
    f_hi = t.f_hi[i];
    axis = t.axis[i];
    at = pair < t.pairs ? rotary_place(i, t.pairs, t.neighbours) : -1;
  }
  __device__ __forceinline__ void put(float* row, float2 turn) const {
    row[at] = turn.x;
    row[at + 2] = turn.y;
  }
  // The table of a row: 8 pairs an item (16 dimensions, as two chunks of 8), as four float4, cosines and sines of the two pairs that word i of the chunks
  // belongs to; those of all items side by side, so that threads of neighbouring items read side by side
  static __device__ __forceinline__ int rotary_place(int pair, int pairs, int neighbours) {
    const int k = pair & 7, word = neighbours ? k & 3 : k >> 1, which = neighbours ? k >> 2 : k & 1;
    return word * (pairs >> 1) + (pair >> 3) * 4 + which;
  }
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
// Words of two pairs: of halves, a word of the first chunk has the pairs' first values and one of the second chunk their second ones; of neighbours, a word has
// a pair.
// (lo, hi), the way there and back: bytes of a word of each chunk to (first values, second values), the same for both, by two permutations.
struct RotaryWords {
  uint32_t lo, hi;
  __device__ __forceinline__ explicit RotaryWords(int neighbours) : lo(neighbours ? 0x5410u : 0x3210u), hi(neighbours ? 0x7632u : 0x7654u) {}
};
// Word i of the item's chunks (a: first, b: second) turned: the two pairs' first values and their second ones, fp32.  cs: the item's first float4 in the row's
// table of `items` items.
template <typename T>
__device__ __forceinline__ void rotary_turn_word(const RotaryWords& w, uint32_t a, uint32_t b, const float4* cs, uint64_t& first, uint64_t& second) {
  const uint32_t u = __byte_perm(a, b, w.lo), v = __byte_perm(a, b, w.hi);
  const uint64_t u2 = pack2(Pair16<T>::lo(u), Pair16<T>::hi(u)), v2 = pack2(Pair16<T>::lo(v), Pair16<T>::hi(v));
  const float4 t = *cs;
  const uint64_t cos2 = pack2(t.x, t.y);
  first = ffma2(v2, pack2(-t.z, -t.w), fmul2(u2, cos2));
  second = ffma2(u2, pack2(t.z, t.w), fmul2(v2, cos2));
}

// One token's heads [head0, head1) of queries and keys side by side (keys behind the queries), by a warp.  cs: the warp's 64 cosines and sines.
template <int HD, int BATCH, typename T>
__device__ __forceinline__ void rotary_row(const RotaryTable& t, const RotaryRows& r, const RotaryPair (&pair)[2], int row, int head0, int head1, const int (&position)[2],
                                           float2* cs) {
  constexpr int ITEMS = HD / 16, LANES = 32 / ITEMS;                     // items a head, heads a warp takes at once (BATCH times that are in flight)
  const int lane = threadIdx.x & 31, item = lane % ITEMS, sub = lane / ITEMS;
  const bool turned = 8 * item < t.pairs;
  const RotaryWords words(t.neighbours);
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
        uint32_t a[4] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w}, b[4] = {hi[i].x, hi[i].y, hi[i].z, hi[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint64_t first, second;
          rotary_turn_word<T>(words, a[e], b[e], reinterpret_cast<const float4*>(cs) + e * (t.pairs >> 3) + item, first, second);
          float f0, f1, s0, s1;
          unpack2(first, f0, f1);
          unpack2(second, s0, s1);
          const uint32_t f = Pair16<T>::pack(f0, f1), s = Pair16<T>::pack(s0, s1);
          a[e] = __byte_perm(f, s, words.lo);
          b[e] = __byte_perm(f, s, words.hi);
        }
        lo[i] = make_uint4(a[0], a[1], a[2], a[3]);
        hi[i] = make_uint4(b[0], b[1], b[2], b[3]);
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

constexpr int kAppendThreads = 256, kAppendCtas = 2, kAppendSteps = 2, kAppendBatch = 4;      // CTAs an SM (three spill registers); rows a thread, of keys or values; heads a lane has in flight, of queries

// An item's 16 values, word by word as rotary_turn_word leaves them, to its two chunks of eight numbers, as quantise8 does it.  order: of a word's four bytes, first
// values before second ones or pair by pair
__device__ __forceinline__ void quantise16(const uint64_t (&first)[4], const uint64_t (&second)[4], float s, float inv, uint32_t order, uint2& lo, uint2& hi) {
  const uint64_t inv2 = pack2(inv, inv), magic = pack2(12582912.0f, 12582912.0f), less = pack2(-12582912.0f, -12582912.0f), minus = pack2(-1.0f, -1.0f);
  uint32_t q[16];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t r = fmul2(i & 1 ? second[i >> 1] : first[i >> 1], inv2);
    const uint64_t t = fadd2(r, magic);                            // the nearest integer in the low bits
    float a, b, d0, d1;
    unpack2(t, a, b);
    unpack2(ffma2(fadd2(t, less), minus, r), d0, d1);
    off = fmax3(off, fabsf(d0), fabsf(d1));
    q[2 * i] = __float_as_uint(a);
    q[2 * i + 1] = __float_as_uint(b);
  }
  if (__builtin_expect(off > 0.5f - 3.0517578125e-05f, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a, b;
      unpack2(i & 1 ? second[i >> 1] : first[i >> 1], a, b);
      q[2 * i] = quantise(a, s, inv);
      q[2 * i + 1] = quantise(b, s, inv);
    }
  }
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __byte_perm(__byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410), 0u, order);
  lo = make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
  hi = make_uint2(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
}

// An item is the run of one sequence's new rows that lies in one block, and some of its key/value heads: the cosines and sines of the run's rows go to
// shared memory once for all of them.  GT: threads of a head's keys or values, a warp where runs have a few rows (decoding steps, drafts).  Behind those items
// the queries: a warp takes a token's heads, or some of them.
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
  const RotaryWords words(p.t.neighbours);
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  auto cu = [&](int i) { return min(max(p.s.cu[i], 0), p.r.n_rows); };
  const int pair_items = p.pairs * p.head_parts;
  const uint32_t q_units = static_cast<uint32_t>(p.r.n_heads > 0 ? p.r.n_rows : 0) * p.q_parts;
  uint32_t it = blockIdx.x;
  for (; it < static_cast<uint32_t>(pair_items); it += gridDim.x) {
    const int pair = static_cast<int>(it) / p.head_parts, part = static_cast<int>(it) - pair * p.head_parts;
    const CacheRun r = cache_run_of(p.c, p.s, last_sequence(p.s.n_seqs, pair, [&](int i) { return (cu(i) >> p.c.bs_log2) + 2 * i; }), p.r.n_rows, pair, p.status,
                                    threadIdx.x == 0 && part == 0);
    if (r.block < 0) continue;
    const int n = r.hi - r.lo;
    // The keys or the values of one head at a time by THREADS threads, 2 rows of 16 dimensions a thread, rotated in fp32 and rounded once, to the number; then the
    // block's scale and numbers as in cache_store_kernel.  (Four rows a thread do not fit the registers of two CTAs an SM.)  A run of more rows than the
    // threads have takes several rounds, and all but the last are read again for their numbers.
    {
      const int units = 2 * min(p.part_heads, p.c.n_kv - part * p.part_heads), rounds = (n + CAP - 1) / CAP;
#pragma unroll 1
      for (int u = group; u < units || u == group; u += kAppendThreads / GT) {
        const bool values = u & 1, turned = !values && 8 * item < p.t.pairs;
        const int head = part * p.part_heads + (u >> 1);
        const long long ld = values ? p.ld_v : p.r.ld_k, at = static_cast<long long>(r.block) * p.c.n_kv + head;
        const T* src = static_cast<const T*>(values ? p.v : p.r.k) + static_cast<long long>(r.row + sub) * ld + head * HD;
        const int2 dims = values ? make_int2(16 * item, 16 * item + 8) : rotary_at(item, p.t.pairs, p.t.neighbours);
        float* scale = (values ? p.c.v_scale : p.c.k_scale) + at;
        int8_t* dst = (values ? p.c.v : p.c.k) + ((at << p.c.bs_log2) * HD);
        uint4 x[2 * STEPS];
        uint64_t first[STEPS][4], second[STEPS][4];
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
            const uint32_t a[4] = {x[2 * i].x, x[2 * i].y, x[2 * i].z, x[2 * i].w}, b[4] = {x[2 * i + 1].x, x[2 * i + 1].y, x[2 * i + 1].z, x[2 * i + 1].w};
            if (turned && row0 + sub + i * ROWS < n) {
              const float4* cs = reinterpret_cast<const float4*>(append_turns + (row0 + sub + i * ROWS) * p.t.pairs) + item;
#pragma unroll
              for (int e = 0; e < 4; ++e) rotary_turn_word<T>(words, a[e], b[e], cs + e * (p.t.pairs >> 3), first[i][e], second[i][e]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                first[i][e] = pack2(Pair16<T>::lo(a[e]), Pair16<T>::hi(a[e]));
                second[i][e] = pack2(Pair16<T>::lo(b[e]), Pair16<T>::hi(b[e]));
              }
            }
          }
        };
        load(0);
        const float old = r.lo > 0 && u < units ? *scale : 0.0f;
        if (u == group) {                                          // (beside the first loads)
          __syncthreads();                                         // (the last item's table is no longer read)
          if (k_pair.at >= 0) {
            const int apart = kAppendThreads >> pairs_log2;
            const int32_t* from = p.r.positions == nullptr ? nullptr : p.r.positions + k_pair.axis * p.r.ld_positions + r.row;
            for (int j0 = my_row; j0 < n; j0 += 8 * apart) {       // 8 positions in flight
              int position[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int j = min(j0 + e * apart, n - 1);
                position[e] = from == nullptr ? r.place + j : from[j];
              }
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (j0 + e * apart < n)
                  k_pair.put(reinterpret_cast<float*>(append_turns + (j0 + e * apart) * p.t.pairs), rotary_turn(k_pair, position[e], p.t.scale, p.t.scale));
            }
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
            for (int e = 0; e < 4; ++e) {
              float a, b;
              unpack2(first[i][e], a, b);
              largest = fmax3(largest, fabsf(a), fabsf(b));
              unpack2(second[i][e], a, b);
              largest = fmax3(largest, fabsf(a), fabsf(b));
            }
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
              uint2 lo, hi;
              quantise16(first[i], second[i], s, inv, turned && p.t.neighbours ? 0x3120u : 0x3210u, lo, hi);
              *reinterpret_cast<uint2*>(out + j * HD + dims.x) = lo;
              *reinterpret_cast<uint2*>(out + j * HD + dims.y) = hi;
            }
          }
        }
        if (grows) cache_requantise<HD, GT>(old, s, r.lo, dst, tid);      // (last: the new values' registers are free)
        if (tid == 0) *scale = s;
      }
    }
  }
  if (q_units == 0) return;
  __syncthreads();                                                 // (the table in shared memory is no longer read)
  // Queries.  Positions are read one unit ahead, as in rotary_kernel
  const int row_first = cu(0), row_end = cu(p.s.n_seqs);
  constexpr uint32_t kWarps = kAppendThreads / 32;
  auto position_of = [&](uint32_t u, int (&position)[2]) {
    position[0] = position[1] = 0;
    if (u >= q_units) return;
    const int row = static_cast<int>(u / p.q_parts);
    if (p.r.positions != nullptr) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (q_pair[i].at >= 0) position[i] = p.r.positions[q_pair[i].axis * p.r.ld_positions + row];
    } else {
      const int s = last_sequence(p.s.n_seqs, row, cu);
      position[0] = position[1] = static_cast<int>(static_cast<uint32_t>(p.s.start[s]) + static_cast<uint32_t>(row - cu(s)));
    }
  };
  uint32_t u = (it - pair_items) * kWarps + warp;
  int position[2];
  position_of(u, position);
  for (; u < q_units; u += gridDim.x * kWarps) {
    int next[2];
    position_of(u + gridDim.x * kWarps, next);
    const int row = static_cast<int>(u / p.q_parts), head0 = static_cast<int>(u - row * p.q_parts) * p.q_part_heads;
    if (row >= row_first && row < row_end)
      rotary_row<HD, kAppendBatch, T>(p.t, p.r, q_pair, row, head0, min(head0 + p.q_part_heads, p.r.n_heads), position, append_turns + warp * kRotaryMaxPairs);
    position[0] = next[0];
    position[1] = next[1];
  }
}

}  // namespace eas
