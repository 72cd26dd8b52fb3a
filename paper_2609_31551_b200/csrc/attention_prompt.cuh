// Causal softmax attention of packed prompts with grouped heads, on tcgen05 tensor cores.
//
// The query heads that share a key/value head are rows of one matrix: row r of a tile is head r % group of token r / group, so a tile
// of 128 rows holds 128 / group tokens (rounded down; the rows left over are not stored).  K and V are then read once for the whole
// group, a short prompt still fills its rows, and the rows of a tile end within 128 / group keys of one another: little of the diagonal
// is computed for nothing.  A work unit is kWg consecutive tiles of one key/value head; a softmax warpgroup (one thread per row)
// works on each.  The key loop walks 80 keys a step up to the last key that the tile's last row sees.
//
//   warp 0       TMA producer of K and V tiles (ring)
//   warps 1..    UMMA issuers, one per warpgroup: S = Q K^T (128 x 80) into TMEM, O += P V (128 x head_dim) in TMEM; they also load
//                the warpgroup's Q tile (refilled as soon as its last scores are complete)
//   warps 4..    softmax warpgroups: three at head_dim 64 (P takes S's own columns, dead once the row is in registers), two at
//                head_dim 128 (P in columns of its own: the next scores are issued as soon as the row has been read)
//
// The pipeline is that of attention_rr.cuh, whose figures gave the split: what counts is the number of tiles in flight, and tensor
// memory holds 3 x (80 + 64) or 2 x (80 + 40 + 128) columns.  At head_dim 128 a step of a tile costs the tensor pipe 640 cycles and
// the special-function unit 640, and takes some 1150 with two tiles in flight (1.17 us for both; each pipe 46 % busy): what bounds short runs is a
// tile's chain from scores to P to O, and long ones the power cap.  At head_dim 64 a step of three tiles costs the unit 1920 cycles and the tensor pipe 960.
// 16411 tokens (32 and 8 heads of 128) 1670-1710 us, 76-78 % of the rate of a library product in short runs; 8192 tokens of 16 and 4 heads of 64 205 us, 40 %.
//
// The reference maximum only moves when the row maximum grows by more than 2^8 in the exponent; then the thread rescales
// its O row in TMEM.  Scores, sums and O are fp32; P is rounded to the data type (bf16 or fp16: what the matrix product takes), and the
// output once at the end.  In fp16 P is 2^7 times what the reference gives (at most 2^15; fp16 ends at 65504), in the sum too: weights
// below 2^-21 of the reference instead of 2^-14 lose bits (20000 keys of 6.5 2^-24 each behind one that holds the rest were off by 7.7 %).
// A row's arithmetic depends on its own sequence alone, not on the unit, the packing or the SMs, unless the call is cut:
// few rows against many keys (a chunk of a prompt behind a long prefix) make fewer units than there are SMs.  SPLIT lays the key steps of all
// units end to end and cuts the line into one equal piece per SM: a piece is a few work items (the end of a unit, whole units, the beginning of
// one), each of which leaves (m, l, O) in the workspace, fp32, and prompt_join_kernel puts a unit's items together in order.  The cut, and with it a
// row's last bits, follow from the call's shapes and the device, not from sm_budget.  512 queries of 40 heads (8 key/value heads of 128) behind 11801 keys, 88 units
// of 154 steps: 167 us whole, 114 as 235 items (in 5 equal parts each, 440 items, 124 to 157: what they leave then fills L2).
//
// Masked keys: their scores are replaced by -inf (P exactly 0), whatever K held.  0 x Inf is not 0, so value rows behind the
// sequence's end are cleared in shared memory, and elements of O that are not finite although the row's sum is (a value row that later rows of the tile
// see, this one does not, holds Inf or NaN; or one that it sees does; or the sum passes the fp32 range) are looked at again, from the values that the row
// sees alone (prompt_settle).  8192 tokens with an infinity at token 100 then take 2 to 7 ms instead of 0.3, at token 7000 33 to 48.
#pragma once
#include "attention_rr.cuh"
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

constexpr int kPromptMaxSeqs = 128;      // sequences of one launch (kernel parameters)
constexpr int kPromptListed = 2048;      // units that the list of a launch holds

template <bool FP16>
constexpr float kPromptRaise = FP16 ? 7.0f : 0.0f;       // log2 of what P and its sum are times what the reference gives

constexpr uint32_t kPromptNoUnit = 0xFFFFFFFFu;   // an entry of the list without work
constexpr int kPromptPieces = 192;       // SPLIT: pieces of the line of steps, at most,
constexpr int kPromptSplitUnits = 768;   // and units

// k / d for 0 <= k < 2^24 and d <= 256 by one multiplication (by ceil(2^32 / d): off by less than k / 2^32 < 1 / d), else by division
struct Divider {
  uint32_t mul;           // 0: divide
  int d;
#ifdef __CUDACC__
  __device__ __forceinline__ int operator()(int k) const {
    return d == 1 ? k : mul != 0u ? static_cast<int>(__umulhi(static_cast<uint32_t>(k), mul)) : k / d;
  }
#endif
};

struct PromptCommon {
  CUtensorMap map_q;      // [tokens, heads, HD], box {64, group, 128 / group}, 128-byte swizzle
  CUtensorMap map_k, map_v;   // [HD / 64 halves x heads, tokens, 64], box {64, 80, HD / 64}
  const uint16_t *q, *k, *v;
  uint16_t* out;
  long long ld_q, ld_k, ld_v, ld_out;
  int out_wide;           // output rows begin on 32-byte boundaries (else on 16-byte ones)
  int group, n_kv, tile_tokens;
  float scale_log2;       // scale * log2(e)
  int n_seqs, total_units;
  Divider by_kv;
  float4* o_ws;           // SPLIT: [item][tile][HD / 4][128 rows]: O, not divided by the sum
  float2* ml_ws;          // [item][tile][128 rows]: reference and sum (-inf, 0: no key)
  uint32_t* status;
  int early_launch;
};
// The kernels' parameters, in three sizes (12 KB of them instead of 1 cost the host 1.3 us a launch).
template <int SEQS>
struct PromptSeqs : PromptCommon {
  int q0[SEQS], k0[SEQS], len_q[SEQS], len_k[SEQS];
  int tiles[SEQS], per_head[SEQS];     // of a sequence and key/value head: row tiles, units
  int unit_prefix[SEQS + 1];
};
struct PromptParamsFew : PromptSeqs<8> {                          // a few sequences, dealt one after the other
  static constexpr int kSeqs = 8;
  static constexpr bool kListed = false, kSplit = false;
};
struct PromptParams : PromptSeqs<kPromptMaxSeqs> {
  static constexpr int kSeqs = kPromptMaxSeqs;
  static constexpr bool kListed = true, kSplit = false;
  // Few rounds of units of different cost: the deal follows this list (sequence << 24 | unit of the sequence), which gives the costliest unit to
  // the CTA with the least to do, instead of the sequences one after the other (8 prompts of 1 to 1563 tokens, 608 units: 14 to 39 key steps an SM)
  int listed;
  uint32_t list[kPromptListed];
};
struct PromptParamsSplit : PromptSeqs<kPromptMaxSeqs> {           // total_units: items
  static constexpr int kSeqs = kPromptMaxSeqs;
  static constexpr bool kListed = false, kSplit = true;
  int n_pieces, n_units;
  uint16_t piece_item[kPromptPieces + 1], unit_item[kPromptSplitUnits + 1];     // first items
  uint16_t item_unit[kPromptSplitUnits + kPromptPieces];
  int item_lo[kPromptSplitUnits + kPromptPieces];                 // first key step; the last one is in front of the unit's next item's first
};

template <int HD>
struct PromptCfg {
  static constexpr bool kOwnP = HD == 128;
  static constexpr int kKeys = 80;
  static constexpr int kWg = kOwnP ? 2 : 3;
  static constexpr int kHalves = HD / 64;
  static constexpr int kStages = kOwnP ? 4 : 8;
  static constexpr int kRegsLight = kOwnP ? 112 : 80, kRegsSoftmax = kOwnP ? 192 : 144, kRegsLaunch = kOwnP ? 168 : 128;
  static constexpr int kThreads = 128 * (1 + kWg);
  static constexpr int kQHalf = 128 * 128;                 // 128 rows x 64 elements
  static constexpr int kQBytes = kQHalf * kHalves;
  static constexpr int kAtomBytes = kKeys * 128;           // 80 keys x 64 elements
  static constexpr int kTileBytes = kAtomBytes * kHalves;
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kKvOff = kWg * kQBytes;
  static constexpr int kBarOff = kKvOff + kStages * kStageBytes;
  static constexpr int kBytes = kBarOff + 512 + 1024;      // barriers + alignment slack
  // TMEM columns of warpgroup w
  static constexpr int kSCol0 = kOwnP ? kWg * HD : 0, kSStride = kOwnP ? kKeys + kKeys / 2 : kKeys + HD;
  static constexpr int kOCol0 = kOwnP ? 0 : kKeys, kOStride = kOwnP ? HD : kKeys + HD;
  static constexpr int kPOff = kOwnP ? kKeys : 0;          // from S
  static_assert(kBytes <= 232448, "exceeds the shared memory of an SM");
  static_assert(kBytes > 116224, "a second CTA must not fit beside this one");
  static_assert(kQBytes % 1024 == 0 && kAtomBytes % 1024 == 0, "tiles start on swizzle-atom boundaries");
  static_assert(kSCol0 + (kWg - 1) * kSStride + kKeys + (kOwnP ? kKeys / 2 : HD) <= 512, "tensor memory columns");
  // an issuer holds stage g while it waits for the first stage of the next unit, which is at most this many steps on: the tiles of a unit
  // end at most 128 (kWg - 1) keys apart
  static_assert((128 * (kWg - 1) + kKeys - 1) / kKeys + 1 < kStages, "the ring holds the steps between two tiles' ends");
  static_assert(128 * kRegsLight + 128 * kWg * kRegsSoftmax <= kThreads * kRegsLaunch, "setmaxnreg budget exceeds the CTA's register allocation");
  static_assert(kThreads * kRegsLaunch <= 65536, "registers");
};

struct PromptUnit {
  int q0, k0, len_q, len_k, ahead, head, tile0, n_q, n_max;   // ahead: keys in front of the first query
};
template <int HD>
__device__ __forceinline__ int prompt_steps(const PromptCommon& p, const PromptUnit& u, int w) {      // key steps of the unit's tile w
  const int seen = min((u.tile0 + w + 1) * p.tile_tokens, u.len_q) + u.ahead;
  return (max(min(seen, u.len_k), 0) + PromptCfg<HD>::kKeys - 1) / PromptCfg<HD>::kKeys;
}
// units of a sequence from its last tiles (the costliest) to its first, the heads side by side
template <int HD, typename Params>
__device__ __forceinline__ PromptUnit prompt_decode(const Params& p, int unit, int& cursor) {
  constexpr int NWG = PromptCfg<HD>::kWg;
  int lo = cursor, k;
  bool listed = false;
  if constexpr (Params::kListed) {
    if (p.listed) {
      const uint32_t e = p.list[unit];
      if (e == kPromptNoUnit) return PromptUnit{};
      lo = static_cast<int>(e >> 24);
      k = static_cast<int>(e & 0xFFFFFFu);
      listed = true;
    }
  }
  if (!listed) {
    while (lo + 1 < p.n_seqs && p.unit_prefix[lo + 1] <= unit) ++lo;
    k = unit - p.unit_prefix[lo];
    cursor = lo;
  }
  PromptUnit u;
  u.q0 = p.q0[lo];
  u.k0 = p.k0[lo];
  u.len_q = p.len_q[lo];
  u.len_k = p.len_k[lo];
  u.ahead = u.len_k - u.len_q;
  const int back = p.by_kv(k);
  u.head = k - back * p.n_kv;
  const int from = p.tiles[lo] - (back + 1) * NWG;        // a remainder of tiles is the cheapest unit, not the costliest
  u.tile0 = max(from, 0);
  u.n_q = NWG + min(from, 0);
  u.n_max = prompt_steps<HD>(p, u, u.n_q - 1);
  return u;
}

__host__ __device__ constexpr uint32_t make_idesc_16(bool fp16, int m, int n, int a_mn, int b_mn) {
  return make_idesc_bf16(m, n, a_mn, b_mn) & ~(fp16 ? (1u << 7) | (1u << 10) : 0u);      // A and B are both fp16 or both bf16
}
template <bool FP16>
__device__ __forceinline__ uint32_t pack_16x2(float lo, float hi) {
  if constexpr (FP16) return Pair16<__half>::pack(lo, hi);
  else return pack_bf16x2(lo, hi);
}

__device__ __forceinline__ void store_32bytes(void* dst, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// (volatile: issued where they stand, not where their values are used)
__device__ __forceinline__ void load_ordered(const float4* src, float& a, float& b, float& c, float& d) {
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a), "=f"(b), "=f"(c), "=f"(d) : "l"(src) : "memory");
}
__device__ __forceinline__ void load_ordered(const float2* src, float& a, float& b) {
  asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(a), "=f"(b) : "l"(src) : "memory");
}

// The second look at output elements that are not finite although their row's scores are numbers: from the keys that the row sees alone.  A NaN among an
// element's values, or infinities of both signs, make it NaN; an infinite value makes it that infinity, however small the weight (in fp32 it may be
// 0, and 0 x Inf NaN); else it is the sum.  A warp looks: lane i has HD / 32 dimensions of the row.
template <int HD, bool FP16>
struct PromptLook {
  static constexpr int N = HD / 32;
  const uint16_t *kp, *vp;         // first key's row of the head; the lane's dimensions of the first value row
  long long ld_k, ld_v;
  __device__ __forceinline__ PromptLook(const PromptCommon& p, int kv_head, int k0)
      : kp(p.k + k0 * p.ld_k + kv_head * HD), vp(p.v + k0 * p.ld_v + kv_head * HD + (threadIdx.x & 31) * N), ld_k(p.ld_k), ld_v(p.ld_v) {}
  __device__ __forceinline__ void values(int j, uint32_t (&x)[N / 2]) const {      // two a word
    if constexpr (N == 4) {
      const uint2 y = *reinterpret_cast<const uint2*>(vp + j * ld_v);
      x[0] = y.x;
      x[1] = y.y;
    } else {
      x[0] = *reinterpret_cast<const uint32_t*>(vp + j * ld_v);
    }
  }
  static __device__ __forceinline__ float element(const uint32_t (&x)[N / 2], int i) {
    return load16(static_cast<uint16_t>(i & 1 ? x[i / 2] >> 16 : x[i / 2] & 0xFFFFu), FP16);
  }
};
// What the value rows of some keys hold, bit i for dimension i of the lane.  odd: a key with an infinite value has elements that are not finite itself, so
// that its score may be -Inf and its weight 0 in earnest (the same in all lanes).
struct PromptFound {
  uint32_t up = 0, down = 0, nan = 0;      // Inf, -Inf, NaN (or infinities of both signs)
  bool odd = false;
};
template <int HD, bool FP16>
__device__ __noinline__ PromptFound prompt_scan(const PromptLook<HD, FP16> look, int from, int to, uint32_t cared, PromptFound f) {
  constexpr int N = HD / 32;
  for (int j = from; j < to && __any_sync(0xffffffffu, (cared & ~f.nan) != 0u); j += 16) {
    uint32_t x[16][N / 2], up = 0, down = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) look.values(min(j + e, to - 1), x[e]);
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float y = look.element(x[e], i);
        up |= (y == INFINITY ? 1u : 0u) << i;
        down |= (y == -INFINITY ? 1u : 0u) << i;
        f.nan |= (y != y ? 1u : 0u) << i;
      }
    f.up |= up;
    f.down |= down;
    f.nan |= f.up & f.down;
    if (!f.odd && __any_sync(0xffffffffu, ((up | down) & cared & ~f.nan) != 0u)) {
      bool odd = false;
      for (int e = j; e < min(j + 16, to); ++e)                  // (all keys of the batch: Inf is rare)
#pragma unroll
        for (int i = 0; i < N; ++i) odd = odd || !isfinite(load16(look.kp[e * look.ld_k + (threadIdx.x & 31) * N + i], FP16));
      f.odd = __any_sync(0xffffffffu, odd);
    }
  }
  return f;
}
// The sums of one row's elements `bad`: weights divided by their sum before they meet values, since values near the largest number pass the fp32 range
// otherwise (which brings their rows here).  An infinite value counts as itself where its key's score is above -Inf.
template <int HD, bool FP16>
__device__ __noinline__ void prompt_sums(const PromptCommon& p, const PromptLook<HD, FP16> look, const uint4* qp, uint16_t* dst, int limit, uint32_t bad) {
  constexpr int N = HD / 32;
  const int lane = threadIdx.x & 31;
  // 32 keys at a time, one a lane: scores, their maximum and the sum of the weights; then the weighted values
  auto score = [&](int j) {
    if (j >= limit) return -INFINITY;
    const uint4* k4 = reinterpret_cast<const uint4*>(look.kp + j * look.ld_k);
    float s = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD / 8; ++c) {
      const uint4 a = k4[c], b = qp[c];
      const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s = fmaf(load16(aw[i] & 0xFFFFu, FP16), load16(bw[i] & 0xFFFFu, FP16), s);
        s = fmaf(load16(aw[i] >> 16, FP16), load16(bw[i] >> 16, FP16), s);
      }
    }
    return s;
  };
  float m = -INFINITY, l = 0.f;
  for (int j = lane; j < limit; j += 32) {
    const float s = score(j), top = fmaxf(m, s);
    if (top > -INFINITY) l = fmaf(l, fast_ex2((m - top) * p.scale_log2), fast_ex2((s - top) * p.scale_log2));
    m = top;
  }
  __syncwarp();
  float top = m;
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  l = m == -INFINITY ? 0.f : l * fast_ex2((m - top) * p.scale_log2);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.f;
  for (int j = 0; j < limit; j += 32) {
    const float s = score(j + lane), w = fast_ex2((s - top) * p.scale_log2) / l;
    __syncwarp();
    for (int e = 0; e < 32; e += 8) {
      uint32_t x[8][N / 2];
#pragma unroll
      for (int f = 0; f < 8; ++f) look.values(min(j + e + f, limit - 1), x[f]);
#pragma unroll
      for (int f = 0; f < 8; ++f) {
        const float wf = __shfl_sync(0xffffffffu, w, e + f), sf = __shfl_sync(0xffffffffu, s, e + f);
        if (j + e + f < limit) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float y = look.element(x[f], i);
            acc[i] = isfinite(y) ? fmaf(wf, y, acc[i]) : sf > -INFINITY ? acc[i] + y : __uint_as_float(0x7FFFFFFFu);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (bad & (1u << i)) dst[i] = static_cast<uint16_t>(pack_16x2<FP16>(acc[i], 0.f));
}
// Columns col0 .. col0 + cols - 1 of up to 32 rows of one head, a lane's own (q_row, head, limit) where `marked`: the values that all of them see are
// looked through once, those that follow for each row.
template <int HD, bool FP16>
__device__ __forceinline__ void prompt_repair_rows(const PromptCommon& p, bool marked, int q_row, int head, int kv_head, int k0, int limit, int col0, int cols) {
  constexpr int N = HD / 32;
  const uint32_t rows = __ballot_sync(0xffffffffu, marked);
  if (rows == 0u) return;
  const int lane = threadIdx.x & 31, common = __reduce_min_sync(0xffffffffu, marked ? limit : 0x7fffffff);
  const PromptLook<HD, FP16> look(p, kv_head, k0);
  auto row_of = [&](int src) {
    return p.out + __shfl_sync(0xffffffffu, q_row, src) * p.ld_out + __shfl_sync(0xffffffffu, head, src) * HD + lane * N;
  };
  auto bad_of = [&](const uint16_t* dst) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane * N + i >= col0 && lane * N + i < col0 + cols && !isfinite(load16(dst[i], FP16))) bad |= 1u << i;
    return bad;
  };
  uint32_t cared = 0;
  for (uint32_t todo = rows; todo != 0u; todo &= todo - 1u) cared |= bad_of(row_of(__ffs(todo) - 1));
  const PromptFound shared = prompt_scan<HD, FP16>(look, 0, common, cared, PromptFound{});
  for (uint32_t todo = rows; todo != 0u; todo &= todo - 1u) {
    const int src = __ffs(todo) - 1, seen = __shfl_sync(0xffffffffu, limit, src);
    uint16_t* dst = row_of(src);
    uint32_t bad = bad_of(dst);
    const PromptFound f = prompt_scan<HD, FP16>(look, common, seen, bad, shared);
    constexpr uint16_t kInf = FP16 ? 0x7C00 : 0x7F80, kNan = 0x7FFF;
    const uint32_t settled = bad & (f.nan | (f.odd ? 0u : f.up | f.down));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (settled & (1u << i)) dst[i] = f.nan & (1u << i) ? kNan : f.up & (1u << i) ? kInf : static_cast<uint16_t>(kInf | 0x8000);
    bad &= ~settled;
    if (__any_sync(0xffffffffu, bad != 0u)) {
      const uint4* qp = reinterpret_cast<const uint4*>(p.q + __shfl_sync(0xffffffffu, q_row, src) * p.ld_q + __shfl_sync(0xffffffffu, head, src) * HD);
      prompt_sums<HD, FP16>(p, look, qp, dst, seen, bad);
    }
    __syncwarp();
  }
}

// key steps [lo, hi) of an item: of the unit, or (hi capped) of one of its tiles
struct PromptPart {
  int lo, hi;
};
template <int HD, typename Params>
__device__ __forceinline__ PromptUnit prompt_item(const Params& p, int item, int& cursor, PromptPart& part) {
  if constexpr (Params::kSplit) {
    const int unit = p.item_unit[item];
    const PromptUnit u = prompt_decode<HD>(p, unit, cursor);
    part.lo = p.item_lo[item];
    part.hi = item + 1 < p.unit_item[unit + 1] ? p.item_lo[item + 1] : u.n_max;
    return u;
  } else {
    const PromptUnit u = prompt_decode<HD>(p, item, cursor);
    part.lo = 0;
    part.hi = u.n_max;
    return u;
  }
}
// The items of a CTA in order
template <typename Params>
struct PromptDeal {
  const Params& p;
  int item, end, piece;
  uint32_t round;
  __device__ __forceinline__ explicit PromptDeal(const Params& params) : p(params), item(0), end(0), piece(blockIdx.x), round(0) {
    if constexpr (Params::kSplit) enter();
    else item = attn_unit_at(0);
  }
  __device__ __forceinline__ void enter() {
    if constexpr (Params::kSplit) {
      item = piece < p.n_pieces ? p.piece_item[piece] : p.total_units;
      end = piece < p.n_pieces ? p.piece_item[piece + 1] : 0;
    }
  }
  __device__ __forceinline__ bool more() const { return item < p.total_units; }
  __device__ __forceinline__ void next() {
    if constexpr (Params::kSplit) {
      if (++item == end) {
        piece += gridDim.x;
        enter();
      }
    } else {
      item = attn_unit_at(++round);
    }
  }
};

// The second look at rows whose output holds the mark, behind a warp's last unit: a row takes as long as its keys are many, and inside the
// pipeline the issuer's and the producer's waits, which end after a second, would run meanwhile.  The warp's units once more, 32 rows at a time.
constexpr uint32_t kPromptMark = 0x7FFEu;          // a NaN (in both types) that no conversion gives
template <bool FP16>
__device__ __forceinline__ uint32_t prompt_mark(uint32_t two) {
  constexpr uint32_t E = FP16 ? 0x7C00u : 0x7F80u;
  if ((two & E) == E) two = (two & 0xFFFF0000u) | kPromptMark;
  if ((two >> 16 & E) == E) two = (two & 0xFFFFu) | kPromptMark << 16;
  return two;
}
__device__ __forceinline__ bool prompt_marked(uint32_t two) { return (two & 0xFFFFu) == kPromptMark || two >> 16 == kPromptMark; }
template <int HD, bool FP16, typename Params>
__device__ __noinline__ void prompt_settle(const Params& p, int w, int row_tok, int row_head) {
  int cursor = 0;
  for (PromptDeal<Params> deal(p); deal.more(); deal.next()) {
    PromptPart part;
    const PromptUnit u = prompt_item<HD>(p, deal.item, cursor, part);
    const int tok = (u.tile0 + w) * p.tile_tokens + row_tok, q_row = u.q0 + tok, head = u.head * p.group + row_head, limit = tok + 1 + u.ahead;
    bool marked = false;
    if (w < u.n_q && row_tok < p.tile_tokens && tok < u.len_q && limit > 0) {
      const uint4* src = reinterpret_cast<const uint4*>(p.out + q_row * p.ld_out + head * HD);
      for (int c = 0; c < HD / 8; ++c) {
        const uint4 x = src[c];
        marked = marked || prompt_marked(x.x) || prompt_marked(x.y) || prompt_marked(x.z) || prompt_marked(x.w);
      }
    }
    prompt_repair_rows<HD, FP16>(p, marked, q_row, head, u.head, u.k0, limit, 0, HD);
  }
}

template <int HD, bool FP16, typename Params>
__global__ void __launch_bounds__(PromptCfg<HD>::kThreads, 1) prompt_attention_kernel(const __grid_constant__ Params p) {
  using L = PromptCfg<HD>;
  constexpr int NST = L::kStages, NWG = L::kWg, KEYS = L::kKeys;
  constexpr bool OWN_P = L::kOwnP, SPLIT = Params::kSplit;
  extern __shared__ uint8_t smem_raw_prompt[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw_prompt) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBarOff);
  uint64_t* q_full = bars;                 // [NWG]
  uint64_t* s_full = q_full + NWG;         // [NWG] scores of a step complete (and everything issued before them)
  uint64_t* p_ready = s_full + NWG;        // [NWG] P stored, O rescaled if it had to be
  uint64_t* s_free = p_ready + NWG;        // [NWG] own P: the warpgroup has read the scores out of tensor memory
  uint64_t* pv_done = s_free + NWG;        // [NWG] own P: P V of a step complete
  uint64_t* k_full = pv_done + NWG;        // [NST]
  uint64_t* v_full = k_full + NST;         // [NST]
  uint64_t* kv_empty = v_full + NST;       // [NST] every issuer hands every stage back
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(kv_empty + NST);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  static_assert((5 * NWG + 3 * NST) * 8 + 8 <= 512, "barrier area");

  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NWG; ++i) { mbar_init(&q_full[i], 1); mbar_init(&s_full[i], 1); mbar_init(&p_ready[i], 4); mbar_init(&s_free[i], 4); mbar_init(&pv_done[i], 1); }
    for (int i = 0; i < NST; ++i) { mbar_init(&k_full[i], 1); mbar_init(&v_full[i], 1); mbar_init(&kv_empty[i], NWG); }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&p.map_q);
    tma_prefetch_desc(&p.map_k);
    tma_prefetch_desc(&p.map_v);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();

  auto q_tile = [&](int w) { return smem + w * L::kQBytes; };
  auto k_tile = [&](uint32_t s) { return smem + L::kKvOff + s * L::kStageBytes; };
  auto v_tile = [&](uint32_t s) { return smem + L::kKvOff + s * L::kStageBytes + L::kTileBytes; };

  if (warp == 0) {
    // ------------------------------------------------------------------ K / V producer
    setmaxnreg_dec<L::kRegsLight>();
    if (lane == 0) {
      uint32_t g = 0;
      bool ok = true;
      int cursor = 0;
      for (PromptDeal<Params> deal(p); deal.more() && ok; deal.next()) {
        PromptPart part;
        const PromptUnit u = prompt_item<HD>(p, deal.item, cursor, part);
        for (int j = part.lo; j < part.hi; ++j, ++g) {
          const uint32_t s = g % NST;
          if (!mbar_wait(&kv_empty[s], ((g / NST) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          const int y = u.k0 + j * KEYS, z = u.head * L::kHalves;
          mbar_expect_tx(&k_full[s], L::kTileBytes);
          tma_load_3d(k_tile(s), &p.map_k, &k_full[s], 0, y, z);
          mbar_expect_tx(&v_full[s], L::kTileBytes);
          tma_load_3d(v_tile(s), &p.map_v, &v_full[s], 0, y, z);
        }
      }
      // the last hand-backs of the stages: asynchronous arrivals, in before the CTA's shared memory passes to another one
      for (uint32_t e = g; e < g + NST && ok; ++e) ok = mbar_wait(&kv_empty[e % NST], ((e / NST) & 1u) ^ 1u, abort_flag);
      if (!ok) {
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) {}     // let loads in flight land before the CTA retires
      }
    }
  } else if (warp <= NWG) {
    // ------------------------------------------------------------------ UMMA issuers, one warp per warpgroup
    // The whole warp walks the steps and one elected lane issues.  A step: P V of this step and the scores of the next one (the next
    // unit's first, behind the last).  Every issuer sees every K/V stage of the CTA land, in order, also those past its own tile's end
    // (which it hands back with a plain arrival), so that it never mistakes a barrier's phase for an earlier one.
    setmaxnreg_dec<L::kRegsLight>();
    const int w = warp - 1;
    constexpr uint32_t idesc_s = make_idesc_16(FP16, 128, KEYS, 0, 0);     // S = Q K^T, both K-major
    constexpr uint32_t idesc_o = make_idesc_16(FP16, 128, HD, 0, 1);       // O += P V, V is MN-major
    const uint32_t tm_s = tmem_base + L::kSCol0 + w * L::kSStride, tm_p = tm_s + L::kPOff, tm_o = tmem_base + L::kOCol0 + w * L::kOStride;
    uint32_t n_q = 0, n_s = 0, n_p = 0;          // Q tiles waited for, s_full phases committed, p_ready phases waited for
    bool started = false;                        // the first scores of this unit's tile are issued already
    bool owed = false;                           // the warpgroup still has to say that it has seen a bare commit
    uint32_t base = 0;                           // ring position of the unit's first K/V tile
    bool ok = true;
    int cursor = 0;
    PromptUnit un{};
    PromptPart un_part{};
    int un_steps = 0;                            // key steps of this issuer's tile in the next item (0: none)
    PromptDeal<Params> deal(p);                  // at the next item
    auto look = [&]() {
      un_steps = 0;
      if (deal.more()) {
        un = prompt_item<HD>(p, deal.item, cursor, un_part);
        if (w < un.n_q) un_steps = max(min(un_part.hi, prompt_steps<HD>(p, un, w)) - un_part.lo, 0);
      }
    };
    look();

    auto load_q = [&](const PromptUnit& u) {
      if (elect_one()) {
        const int tok = u.q0 + (u.tile0 + w) * p.tile_tokens;
        mbar_expect_tx(&q_full[w], static_cast<uint32_t>(p.tile_tokens * p.group * 128 * L::kHalves));
#pragma unroll
        for (int h = 0; h < L::kHalves; ++h) tma_load_3d(q_tile(w) + h * L::kQHalf, &p.map_q, &q_full[w], h * 64, u.head * p.group, tok);
      }
      __syncwarp();
    };
    auto q_landed = [&]() -> bool {
      if (!warp_mbar_wait(&q_full[w], n_q & 1u, abort_flag)) return false;
      ++n_q;
      return true;
    };
    auto k_landed = [&](uint32_t g) -> bool { return warp_mbar_wait(&k_full[g % NST], (g / NST) & 1u, abort_flag); };
    auto hand_back = [&](uint32_t from, uint32_t to) -> bool {   // stages past this tile's end
      for (uint32_t g = from; g < to; ++g) {
        if (!k_landed(g)) return false;
        if (elect_one()) mbar_arrive(&kv_empty[g % NST]);
        __syncwarp();
      }
      return true;
    };
    // Only the first `rows` value rows at ring position g belong to the sequence: clears the others.  Every issuer does so before
    // its own P V; later ones store the zeros that are there already.
    auto clear_behind = [&](uint32_t g, int rows) {
#pragma unroll
      for (int h = 0; h < L::kHalves; ++h) {
        uint8_t* v = v_tile(g % NST) + h * L::kAtomBytes;
#pragma unroll 4
        for (int c = rows * 8 + lane; c < KEYS * 8; c += 32)      // 16-byte chunks, 8 a row
          *reinterpret_cast<uint4*>(v + c * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      fence_proxy_async_smem();                                // generic-proxy stores -> visible to the tensor core's operand reads
      __syncwarp();
    };
    // by the elected lane: scores of the current tile (the last one waited for) against the K tile at ring position g
    auto mma_s = [&](uint32_t g) {
      const uint64_t ad = make_smem_desc(smem_u32(q_tile(w)), 16, 1024, kSwizzle128B);
      const uint64_t bd = make_smem_desc(smem_u32(k_tile(g % NST)), 16, 1024, kSwizzle128B);
#pragma unroll
      for (int h = 0; h < L::kHalves; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma_bf16_ss(tm_s, ad + h * (L::kQHalf >> 4) + 2 * k, bd + h * (L::kAtomBytes >> 4) + 2 * k, idesc_s, h != 0 || k != 0);
      umma_commit(&s_full[w]);
    };

    while (deal.more() && ok) {
      const PromptUnit u = un;
      const PromptPart part = un_part;
      const int n_steps = un_steps;
      deal.next();
      look();
      const uint32_t next_base = base + static_cast<uint32_t>(part.hi - part.lo);
      if (n_steps == 0) {
        ok = hand_back(base, next_base);
        base = next_base;
        started = false;
        continue;
      }
      const bool chain = un_steps > 0;                // the next unit's first scores follow this unit's last ones
      if (!started) {
        if (owed) {                              // the warpgroup has seen the bare commit, so s_full may be used again
          if (!warp_mbar_wait(&p_ready[w], n_p & 1u, abort_flag)) { ok = false; break; }
          ++n_p;
        }
        load_q(u);
        if (!q_landed() || !k_landed(base)) { ok = false; break; }
        if (OWN_P && n_s > 0 && !warp_mbar_wait(&s_free[w], (n_s - 1u) & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        if (elect_one()) mma_s(base);
        __syncwarp();
        ++n_s;
      }
      for (int j = 0; j < n_steps; ++j) {
        const bool last = j + 1 == n_steps;
        const bool more = !last || chain;
        const uint32_t g = base + static_cast<uint32_t>(j), gn = last ? next_base : g + 1;      // gn: the K tile of the scores to come
        if (last && chain) {                     // the Q tile is free when the last scores are complete
          if (!warp_mbar_wait(&s_full[w], (n_s - 1u) & 1u, abort_flag)) { ok = false; break; }
          load_q(un);
        }
        if (last && !hand_back(g + 1, next_base)) { ok = false; break; }
        const int rows = u.len_k - (part.lo + j) * KEYS;     // key rows of this step that belong to the sequence
        if (!OWN_P && !warp_mbar_wait(&v_full[g % NST], (g / NST) & 1u, abort_flag)) { ok = false; break; }
        if (!OWN_P && rows < KEYS) clear_behind(g, rows);
        if (more && !k_landed(gn)) { ok = false; break; }
        if (last && chain && !q_landed()) { ok = false; break; }
        if (OWN_P && more) {
          if (!warp_mbar_wait(&s_free[w], (n_s - 1u) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after_sync();
          if (elect_one()) mma_s(gn);
          __syncwarp();
          ++n_s;
        }
        if (OWN_P && !warp_mbar_wait(&v_full[g % NST], (g / NST) & 1u, abort_flag)) { ok = false; break; }
        if (OWN_P && rows < KEYS) clear_behind(g, rows);
        if (!warp_mbar_wait(&p_ready[w], n_p & 1u, abort_flag)) { ok = false; break; }
        ++n_p;
        tc_fence_after_sync();
        const uint64_t bd = make_smem_desc(smem_u32(v_tile(g % NST)), L::kAtomBytes, 1024, kSwizzle128B);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < KEYS / 16; ++ks)                 // 16 keys: 8 columns of P, 2 KB of V
            umma_bf16_ts(tm_o, tm_p + ks * 8, bd + ks * (2048 >> 4), idesc_o, (j != 0 || ks != 0) ? 1u : 0u);
          if (OWN_P) umma_commit(&pv_done[w]);
          else if (more) mma_s(gn);
          else umma_commit(&s_full[w]);                          // bare: tells the warpgroup that its O is final
          umma_commit(&kv_empty[g % NST]);
        }
        __syncwarp();
        if (!OWN_P) ++n_s;
      }
      started = chain;
      owed = !OWN_P && !chain;
      base = next_base;
    }
  } else if (warp < 4) {
    setmaxnreg_dec<L::kRegsLight>();
  } else {
    // ------------------------------------------------------------------ softmax warpgroups
    setmaxnreg_inc<L::kRegsSoftmax>();
    const int w = (warp - 4) >> 2;
    const int quarter = warp & 3;                  // TMEM lane quarter of this warp
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + L::kSCol0 + w * L::kSStride, p_addr = s_addr + L::kPOff, o_addr = lane_addr + L::kOCol0 + w * L::kOStride;
    const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
    const int row = quarter * 32 + lane, row_tok = row / p.group, row_head = row - row_tok * p.group;   // token of the tile, head of the group
    uint32_t n = 0;                                // s_full phases waited for (own P: steps done)
    bool ok = true;
    // the finished tile whose output is still in tensor memory
    bool pend = false;
    int pend_q = -1, pend_head = 0, pend_k0 = 0, pend_limit = 0;   // query row (-1: not stored), key/value head, first key row, keys seen
    float pend_l = 1.f, pend_m = 0.f;
    int pend_slot = 0;                             // SPLIT: the part's place in the workspace
    bool marks = false;                            // a row of this warp holds marks
    // 64 columns of O at a time: the trip to tensor memory is what a flush waits for (16 at a time: 1.6 us of a tile's beginning)
    auto load_64 = [&](uint32_t addr, uint32_t (&o)[64]) {
      __syncwarp();
      tmem_ld_32x32_at<0>(addr, o);
      tmem_ld_32x32_at<32>(addr, o);
      tmem_ld_wait_16<0>(o); tmem_ld_tie_16<16>(o); tmem_ld_tie_16<32>(o); tmem_ld_tie_16<48>(o);
    };
    auto flush_output = [&]() {
      if constexpr (SPLIT) {                       // (rows that are not stored leave nothing)
        float4* dst = p.o_ws + static_cast<long long>(pend_slot) * (HD / 4) * 128 + row;
#pragma unroll 1
        for (int c = 0; c < HD; c += 64) {
          uint32_t o[64];
          load_64(o_addr + c, o);
          if (pend_q >= 0) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              dst[(c / 4 + i) * 128] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
          }
        }
        if (pend_q >= 0) p.ml_ws[static_cast<long long>(pend_slot) * 128 + row] = make_float2(pend_l == 0.f ? -INFINITY : pend_m, pend_l);
        __syncwarp();
        pend = false;
        return;
      }
      const float inv = pend_limit > 0 ? 1.0f / pend_l : 0.f;
      uint4* dst = reinterpret_cast<uint4*>(p.out + static_cast<long long>(max(pend_q, 0)) * p.ld_out + (pend_head * p.group + row_head) * HD);
      bool wrong = false;
#pragma unroll 1
      for (int c = 0; c < HD; c += 64) {
        uint32_t o[64];
        load_64(o_addr + c, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t pkd[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float lo = __uint_as_float(o[16 * j + 2 * i]), hi = __uint_as_float(o[16 * j + 2 * i + 1]);
            wrong = wrong || !(lo * 0.f + hi * 0.f == 0.f);      // (Inf x 0 = NaN too: one test for both)
            pkd[i] = pend_limit > 0 ? pack_16x2<FP16>(lo * inv, hi * inv) : 0u;
          }
          // 32 bytes, a whole sector: a warp's store touches 32 rows, and it is the rows that the store unit counts
          if (pend_q >= 0 && p.out_wide) {
            store_32bytes(dst + c / 8 + 2 * j, pkd);
          } else if (pend_q >= 0) {
            dst[c / 8 + 2 * j] = make_uint4(pkd[0], pkd[1], pkd[2], pkd[3]);
            dst[c / 8 + 2 * j + 1] = make_uint4(pkd[4], pkd[5], pkd[6], pkd[7]);
          }
        }
      }
      wrong = wrong && pend_q >= 0 && pend_limit > 0 && pend_l * 0.f == 0.f;
      if (__builtin_expect(wrong, 0)) {            // (this thread's own stores: visible to it)
#pragma unroll 1
        for (int c = 0; c < HD / 8; ++c) {
          const uint4 x = dst[c];
          dst[c] = make_uint4(prompt_mark<FP16>(x.x), prompt_mark<FP16>(x.y), prompt_mark<FP16>(x.z), prompt_mark<FP16>(x.w));
        }
      }
      marks = marks || __any_sync(0xffffffffu, wrong);
      __syncwarp();
      pend = false;
    };

    int cursor = 0;
    for (PromptDeal<Params> deal(p); deal.more() && ok; deal.next()) {
      PromptPart part;
      const PromptUnit u = prompt_item<HD>(p, deal.item, cursor, part);
      const int n_steps = w < u.n_q ? max(min(part.hi, prompt_steps<HD>(p, u, w)) - part.lo, 0) : 0;
      const int tok = (u.tile0 + w) * p.tile_tokens + row_tok;
      const bool stored = w < u.n_q && row_tok < p.tile_tokens && tok < u.len_q;
      if (n_steps == 0) {                           // no tile in this unit, or one that sees no key
        if (pend) {
          if (!warp_mbar_wait(OWN_P ? &pv_done[w] : &s_full[w], (OWN_P ? n - 1u : n) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after_sync();
          flush_output();
          if (!OWN_P) {
            ++n;
            tc_fence_before_sync();
            __syncwarp();
            mbar_arrive_if(&p_ready[w], lane == 0);        // the issuer may use s_full[w] again
          }
        }
        if (SPLIT && stored) p.ml_ws[(static_cast<long long>(deal.item) * NWG + w) * 128 + row] = make_float2(-INFINITY, 0.f);
        if (!SPLIT && stored) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + (static_cast<long long>(u.q0) + tok) * p.ld_out + (u.head * p.group + row_head) * HD);
          for (int c = 0; c < HD / 8; ++c) dst[c] = make_uint4(0u, 0u, 0u, 0u);
        }
        continue;
      }
      // keys that this row sees; rows that are not stored see all (what they compute does not matter, and masking would cost every step)
      const int limit = stored ? max(tok + 1 + u.ahead, 0) : 0x7fffffff;
      float m_used = -INFINITY;                     // no reference yet
      uint64_t l2[2] = {0, 0};                      // row sum, two packed accumulators
      int left = limit - part.lo * KEYS;            // of them from this step on
#pragma unroll 1
      for (int j = 0; j < n_steps; ++j, left -= KEYS) {
        if (!warp_mbar_wait(&s_full[w], n & 1u, abort_flag)) { ok = false; break; }
        ++n;
        tc_fence_after_sync();
        if (!OWN_P && __builtin_expect(pend, 0)) flush_output();       // the previous tile's P V is complete
        uint32_t s[KEYS];
        tmem_ld_32x32_at<0>(s_addr, s);
        tmem_ld_32x32_at<32>(s_addr, s);
        tmem_ld_32x16_at<64>(s_addr, s);
        tmem_ld_wait_16<0>(s); tmem_ld_tie_16<16>(s); tmem_ld_tie_16<32>(s); tmem_ld_tie_16<48>(s); tmem_ld_tie_16<64>(s);
        if (OWN_P) {
          tc_fence_before_sync();
          __syncwarp();
          mbar_arrive_if(&s_free[w], lane == 0);
        }
        if (__builtin_expect(left < KEYS, 0)) {              // keys that the row does not see
#pragma unroll
          for (int i = 0; i < KEYS; ++i) if (i >= left) s[i] = 0xff800000u;   // -inf
        }
        float mx;
        {
          float c0 = -INFINITY, c1 = -INFINITY, c2 = -INFINITY, c3 = -INFINITY;
#pragma unroll
          for (int i = 0; i < KEYS; i += 8) {
            c0 = fmax3(c0, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
            c1 = fmax3(c1, __uint_as_float(s[i + 2]), __uint_as_float(s[i + 3]));
            c2 = fmax3(c2, __uint_as_float(s[i + 4]), __uint_as_float(s[i + 5]));
            c3 = fmax3(c3, __uint_as_float(s[i + 6]), __uint_as_float(s[i + 7]));
          }
          mx = fmax3(fmaxf(c0, c1), c2, c3);
        }
        // the reference maximum moves when the row maximum grew by more than the threshold, and to the row's first score above -inf.  Without
        // one the exponentials are those of -inf against 0.
        const float m_old = m_used;
        const bool moved = (mx - m_used) * p.scale_log2 > kRescaleThreshold;       // (-inf against -inf: NaN, no)
        m_used = moved ? mx : m_used;
        const uint32_t rescale = __ballot_sync(0xffffffffu, moved && j != 0);
        const float mb = m_used == -INFINITY ? 0.f : m_used * p.scale_log2 - kPromptRaise<FP16>;
        const uint64_t nmb2 = pack2(-mb, -mb);
        const uint64_t l_old[2] = {l2[0], l2[1]};
        l2[0] = l2[1] = 0;
        const uint32_t pv_ok = OWN_P ? mbar_try_wait(&pv_done[w], n & 1u) : 1u;      // the previous step's, tested ahead
        uint32_t pk[KEYS / 2];
#pragma unroll
        for (int i = 0; i < KEYS / 2; ++i) {
          const uint64_t t = ffma2(pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), scale2, nmb2);
          float p0, p1;
          unpack2(t, p0, p1);
          p0 = fast_ex2(p0);
          p1 = fast_ex2(p1);
          l2[i & 1] = fadd2(l2[i & 1], pack2(p0, p1));
          pk[i] = pack_16x2<FP16>(p0, p1);
        }
        if (OWN_P) {
          // P goes where the previous step's was, and O may change: that step's P V has to be complete
          if (n > 1u && !warp_mbar_wait_tested(pv_ok, &pv_done[w], n & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after_sync();
          if (__builtin_expect(pend, 0)) flush_output();
        }
        if (__builtin_expect(rescale != 0u, 0)) {
          const float corr = moved ? fast_ex2((m_old - m_used) * p.scale_log2) : 1.0f;      // (from no reference: 0)
          const uint64_t corr2 = pack2(corr, corr);
          l2[0] = fadd2(fmul2(l_old[0], corr2), l2[0]);
          l2[1] = fadd2(fmul2(l_old[1], corr2), l2[1]);
#pragma unroll 1
          for (int c = 0; c < HD / 8; ++c) {
            uint32_t o[8];
            asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]) : "r"(o_addr + c * 8) : "memory");
            asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(o[0]), "+r"(o[1]), "+r"(o[2]), "+r"(o[3]), "+r"(o[4]), "+r"(o[5]), "+r"(o[6]), "+r"(o[7])::"memory");
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
            tmem_st_32x8_from(o_addr + c * 8, o);
          }
        } else {
          l2[0] = fadd2(l_old[0], l2[0]);
          l2[1] = fadd2(l_old[1], l2[1]);
        }
        // P row: two elements per column of this thread's lane
        __syncwarp();
        tmem_st_32x32_from(p_addr, pk);
        tmem_st_32x8_from(p_addr + 32, pk + 32);
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(&p_ready[w], lane == 0);
      }
      if (!ok) break;
      pend = true;
      float a0, a1, a2, a3;
      unpack2(l2[0], a0, a1);
      unpack2(l2[1], a2, a3);
      pend_l = (a0 + a1) + (a2 + a3);
      pend_m = m_used;
      pend_q = stored ? u.q0 + tok : -1;
      pend_head = u.head;
      pend_k0 = u.k0;
      pend_limit = stored ? limit : 0;
      if (SPLIT) pend_slot = deal.item * NWG + w;
    }
    if (ok && pend) {
      if (warp_mbar_wait(OWN_P ? &pv_done[w] : &s_full[w], (OWN_P ? n - 1u : n) & 1u, abort_flag)) {
        tc_fence_after_sync();
        flush_output();
      } else {
        ok = false;
      }
    }
    if constexpr (!SPLIT) {
      if (__builtin_expect(marks && ok, 0)) prompt_settle<HD, FP16>(p, w, row_tok, row_head);
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(p.status, DEV_OK, DEV_ERR_WAIT_TIMEOUT);
}

// The second look behind the joining kernel's last piece of work: there what the calls keep in registers would cost every row.
constexpr int kPromptJoinCols = 8;
template <int HD, bool FP16>
__device__ __noinline__ void prompt_settle_joined(const PromptParamsSplit& p) {
  constexpr int NWG = PromptCfg<HD>::kWg, CHUNKS = HD / kPromptJoinCols;
  const int row = threadIdx.x & 127, row_tok = row / p.group, row_head = row - row_tok * p.group;
  int cursor = 0;
  for (int it = blockIdx.x * 4 + (threadIdx.x >> 7); it < p.n_units * NWG * CHUNKS; it += gridDim.x * 4) {
    const int unit = it / (NWG * CHUNKS), w = it / CHUNKS % NWG, col0 = it % CHUNKS * kPromptJoinCols;
    const PromptUnit u = prompt_decode<HD>(p, unit, cursor);
    const int tok = (u.tile0 + w) * p.tile_tokens + row_tok, q_row = u.q0 + tok, head = u.head * p.group + row_head, limit = tok + 1 + u.ahead;
    bool marked = false;
    if (w < u.n_q && row_tok < p.tile_tokens && tok < u.len_q && limit > 0) {
      const uint4 x = *reinterpret_cast<const uint4*>(p.out + q_row * p.ld_out + head * HD + col0);
      marked = prompt_marked(x.x) || prompt_marked(x.y) || prompt_marked(x.z) || prompt_marked(x.w);
    }
    prompt_repair_rows<HD, FP16>(p, marked, q_row, head, u.head, u.k0, limit, col0, kPromptJoinCols);
  }
}

// The items of a unit put together, in order: 128 threads, one a row, per (unit, tile, 8 columns); a thread has the loads of 8 items in flight.
// (A quarter of the columns each and one item after the other: 128 tokens of 32 heads behind 8000 in 12 parts 35 us instead of 28.)
template <int HD, bool FP16>
__global__ void __launch_bounds__(512, 1) prompt_join_kernel(const __grid_constant__ PromptParamsSplit p) {
  constexpr int NWG = PromptCfg<HD>::kWg, COLS = kPromptJoinCols, CHUNKS = HD / COLS, BATCH = 8;
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  const int row = threadIdx.x & 127, row_tok = row / p.group, row_head = row - row_tok * p.group;
  int cursor = 0;
  bool marks = false;
  for (int it = blockIdx.x * 4 + (threadIdx.x >> 7); it < p.n_units * NWG * CHUNKS; it += gridDim.x * 4) {
    const int unit = it / (NWG * CHUNKS), w = it / CHUNKS % NWG, col0 = it % CHUNKS * COLS;
    const PromptUnit u = prompt_decode<HD>(p, unit, cursor);
    if (w >= u.n_q) continue;
    const int tok = (u.tile0 + w) * p.tile_tokens + row_tok, limit = max(tok + 1 + u.ahead, 0);
    const bool stored = row_tok < p.tile_tokens && tok < u.len_q;
    float m = -INFINITY, l = 0.f, acc[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) acc[i] = 0.f;
    const int first = p.unit_item[unit], items = stored ? p.unit_item[unit + 1] - first : 0;      // (0 too where no row sees a key)
    for (int base = 0; base < items; base += BATCH) {
      float ml[BATCH][2], x[BATCH][COLS];
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        ml[e][0] = -INFINITY;
        ml[e][1] = 0.f;
        if (base + e < items) {
          const long long slot = static_cast<long long>(first + base + e) * NWG + w;
          const float4* o = p.o_ws + (slot * (HD / 4) + col0 / 4) * 128 + row;
          load_ordered(p.ml_ws + slot * 128 + row, ml[e][0], ml[e][1]);
          load_ordered(o, x[e][0], x[e][1], x[e][2], x[e][3]);         // (not written where the item has no key for any row of the tile: not used then)
          load_ordered(o + 128, x[e][4], x[e][5], x[e][6], x[e][7]);
        }
      }
      float top = m;
#pragma unroll
      for (int e = 0; e < BATCH; ++e) top = fmaxf(top, ml[e][0]);
      const float old = m == -INFINITY ? 0.f : fast_ex2((m - top) * p.scale_log2);
      l *= old;
#pragma unroll
      for (int i = 0; i < COLS; ++i) acc[i] = m == -INFINITY ? 0.f : acc[i] * old;
      m = top;
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        const bool any = ml[e][1] != 0.f;                              // (NaN: yes)
        const float f = any ? fast_ex2((ml[e][0] - m) * p.scale_log2) : 0.f;
        if (any) l = fmaf(ml[e][1], f, l);
#pragma unroll
        for (int i = 0; i < COLS; ++i) acc[i] = any ? fmaf(x[e][i], f, acc[i]) : acc[i];
      }
    }
    const float inv = limit > 0 ? 1.0f / l : 0.f;
    bool wrong = false;
    uint16_t* dst = p.out + (static_cast<long long>(u.q0) + tok) * p.ld_out + (u.head * p.group + row_head) * HD + col0;
#pragma unroll
    for (int i = 0; i < COLS; i += 8) {
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        wrong = wrong || !(acc[i + 2 * e] * 0.f + acc[i + 2 * e + 1] * 0.f == 0.f);
        y[e] = limit > 0 ? pack_16x2<FP16>(acc[i + 2 * e] * inv, acc[i + 2 * e + 1] * inv) : 0u;
      }
      if (stored) *reinterpret_cast<uint4*>(dst + i) = make_uint4(y[0], y[1], y[2], y[3]);
    }
    wrong = wrong && stored && limit > 0 && l * 0.f == 0.f;
    if (__builtin_expect(wrong, 0)) {
      uint4* x = reinterpret_cast<uint4*>(dst);
      *x = make_uint4(prompt_mark<FP16>(x->x), prompt_mark<FP16>(x->y), prompt_mark<FP16>(x->z), prompt_mark<FP16>(x->w));
    }
    marks = marks || __any_sync(0xffffffffu, wrong);
  }
  if (__builtin_expect(marks, 0)) prompt_settle_joined<HD, FP16>(p);
}

}  // namespace eas
