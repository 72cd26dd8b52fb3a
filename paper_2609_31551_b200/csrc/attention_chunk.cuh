// Attention of several new tokens a sequence over the 8-bit cache, on tcgen05 tensor cores: out = softmax(scale q K^T) V, the new tokens being the
// last of their sequence.
//
// The query heads that share a key/value head are rows of one matrix, 128 / group tokens a tile of 128 rows, as in attention_prompt.cuh; the numbers of the cache
// enter exact in fp16 as in attention_cache.cuh: queries are fp16 times a power of two per row, a block's key scale multiplies its scores in fp32, its value scale v
// is an exponent: with t = score + log2 v and w = 2^(t - m),  out = sum w number / sum w / v, m being kept 2^7 to 2^15 below the largest t.
// The weights are rounded to fp16 for their product with the numbers, the only operands that the tensor core has beside numbers exact in 16 bits, with 11 bits
// where bf16 has 8; the sum below the line takes them unrounded, and it, the references and O are fp32.  Against 64 bits the outputs are off by 0.00025 in fp16
// (0.00021 with weights of 32 bits) and by 0.0017 in bf16 either way.
//
//   warps 0, 3    bytes of K and of V, a block's tokens of a head (they are contiguous) a bulk copy, into rings of 8-bit tiles; warp 0 the scales of the steps, too, and
//                 warp 3 walks the line of units (below) and tells the others the items of the CTA, through a ring.  (One warp for both took 1100 cycles a copy and was what
//                 long caches of few rows waited for.)
//   warps 1, 2    UMMA issuers, one per softmax warpgroup
//   warps 4 ..    converters: tiles of queries, then two warps those of K and two those of V, from bytes to fp16 in the tensor core's layout: (0x6400 | (byte ^ 0x80)) - 1152,
//                 exact.  Bytes 0 and 2 of a word, then 1 and 3: four dimensions lie in the order 0, 2, 1, 3, in the queries and the output too.  (Keys as number + 128, the
//                 128 taken off the score by the row's sum, would save the subtraction, but the fp32 sums of the product round at the size of 128 sum |q|: 5e-3 of a weight
//                 for quiet keys under a loud scale.)
//   warps 8 ..    two softmax warpgroups, one thread a row
//
// A step is 80 keys: 5 parts of 16, the smallest block, and as many scores as a thread's registers hold beside their weights.  A unit of two tiles of one
// key/value head (shared) brings each K and V tile to both warpgroups; a unit of one tile gives its steps to the warpgroups in turn (alternate), which put
// their results together at its end: O lies in tensor memory, where the lanes of both can read it.  So two steps are in flight whether there are many rows
// (bound by the pipes) or few (bound by the conversion of the bytes).
//
// The units of all sequences and heads form a line, in tokens seen times tiles, cut into one equal piece an SM (a function of the shapes and the device, not of
// sm_budget).  A piece is the end of a unit, whole units, the beginning of one; cut units leave (m, l, O) in the workspace, and chunk_join_kernel puts them
// together in order.  Lengths are read on the device: each CTA sums them up itself.
//
// Measured, back to back in a graph, both launches, 32 and 8 heads of 128 unless stated: two chunks of 2048 tokens behind 14336 1.04 to 1.1 ms, 930 to 990
// TFLOP/s (the kernel for prompts, whose keys and values are 16-bit, 0.92 to 0.99), behind 30720 2.1 to 2.3 (2.17); 512 of 40 and 8 heads behind 11801 162 to
// 190 us (122 to 161); 64 tokens behind 16320 42; 12 sequences of 16384 with 16 new tokens 127, 3.2 TB/s; 12 prompts of 600 tokens, 16 heads of 64, 83 (29).
// The ranges are the clock's, under the power cap.
// Many rows: a step of both tiles takes 2520 cycles in the loop, 2700 with the units' ends, of which the tensor pipe is busy 47 %, the special functions 48 %,
// the ALUs 41 %, the issue slots 51 %: the chain of a step (scores read, weighed, P stored, waits) with two warps a scheduler.  (With biased keys, above, the
// same cycles at a clock 4 to 6 % higher.)
// Few rows: 1460 cycles a step of one warpgroup, a pair of warps converting keys in 1000 and values in 870, beside its waits.
// Short sequences: 15 cycles an instruction, 4.4 of them for instructions (7.2 when the code of all roles was 124 KB and not 97) and 5.4 for memory and tensor
// memory: a CTA begins and ends units all the time, and its first scores come 13 us after its start (lengths 1.5, the first item 2, block numbers 1, bytes 1.5,
// two tiles of queries 2 to 4 each).
// Rings of converted tiles: three of values, since the warpgroups are up to two steps apart (with two, 8 and 28 % more for the chunks of 2048 and the 12
// sequences).
#pragma once
#include <type_traits>

#include "attention_cache.cuh"
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

constexpr int kChunkMaxSeqs = 512;       // sequences of one launch (the prefix sums lie in shared memory)
constexpr int kChunkKeys = 80, kChunkParts = kChunkKeys / 16;
constexpr int kChunkUnitCost = 160;      // of a unit's beginning and end, in tokens of one tile
constexpr int kChunkLeastCost = 320;     // of a piece
constexpr int kChunkItems = 4;           // items that the roles may be apart
constexpr int kChunkMaxPieces = 1024;    // SMs of a device, at most

struct ChunkItem;
struct ChunkParams {
  CacheView c;
  const int32_t *table, *cu, *seq_lens;
  long long ld_table;
  int n_seqs, max_blocks, n_rows, max_new;
  int few_rows;                // sequences of at most so many rows a key/value head belong to another kernel (attention_cache.cuh)
  const uint16_t* q;
  uint16_t* out;
  long long ld_q, ld_out;
  int fp16, group, tile_tokens;
  uint32_t by_group;           // ceil(2^32 / group), 0 for 1
  int n_ctas;                  // SMs of the device: pieces of the line, at most
  int ws_rows;                 // rows of a tile that the workspace holds
  float scale_log2;
  float4* o_ws;                // [2 pieces][2 tiles][HD / 4][ws_rows]: O, not divided by the sum
  float2* ml_ws;               // [2 pieces][2 tiles][ws_rows]: reference and sum (-inf, 0: no key)
  ChunkItem* cut_ws;           // [pieces]: the item that a unit's first cut ends (n 0: none)
  uint32_t* status;
  int early_launch;
};

constexpr int kChunkDealBytes = 160;

template <int HD>
struct ChunkCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kRawK = HD == 128 ? 3 : 6, kRawV = HD == 128 ? 2 : 6, kKTiles = HD == 128 ? 2 : 3, kVTiles = 3;
  static constexpr int kThreads = 512;
  static constexpr int kRegsLight = 80, kRegsConvert = 96, kRegsSoftmax = 168, kRegsLaunch = 128;
  static constexpr int kQHalf = 128 * 128, kQBytes = kQHalf * kHalves;                 // 128 rows x 64 elements
  static constexpr int kAtomBytes = kChunkKeys * 128, kTileBytes = kAtomBytes * kHalves;   // 80 keys x 64 elements
  static constexpr int kRawBytes = kChunkKeys * HD;
  static constexpr int kKOff = 2 * kQBytes, kVOff = kKOff + kKTiles * kTileBytes, kRawOff = kVOff + kVTiles * kTileBytes;
  static constexpr int kPrefixOff = kRawOff + (kRawK + kRawV) * kRawBytes;              // (keys' tiles, then values')
  static constexpr int kScaleSlots = 32;
  static constexpr int kScaleOff = kPrefixOff + (kChunkMaxSeqs + 2) * 8;               // [slot][16]: key scales, log2 of value scales, their inverses
  static constexpr int kRowOff = kScaleOff + kScaleSlots * 64;                         // [2][128] factors of the rows' scores
  static constexpr int kMlOff = kRowOff + 2 * 128 * 4;                                 // [2][128] reference and sum of a warpgroup's rows
  static constexpr int kItemOff = kMlOff + 2 * 128 * 8;
  static constexpr int kDealOff = kItemOff + kChunkItems * 64;                         // where warp 3 is on the line
  static constexpr int kBarOff = kDealOff + kChunkDealBytes;
  static constexpr int kBars = 2 * (kRawK + kRawV) + 2 * kKTiles + 2 * kVTiles + kScaleSlots + 2 + 2 + 4 * 2 + 2 + 2 * kChunkItems;
  static constexpr int kBytes = kBarOff + kBars * 8 + 160 + 1024;                      // words, alignment slack
  static constexpr int kSCol0 = 2 * HD, kSStride = kChunkKeys + kChunkKeys / 2;        // tensor memory: O of both, then scores and P of each
  static_assert(kBytes <= 232448, "exceeds the shared memory of an SM");
  static_assert(kBytes > 116224, "a second CTA must not fit beside this one");
  static_assert(kQBytes % 1024 == 0 && kAtomBytes % 1024 == 0, "tiles start on swizzle-atom boundaries");
  static_assert(kSCol0 + 2 * kSStride <= 512, "tensor memory columns");
  static_assert(kRegsLight + kRegsConvert + 2 * kRegsSoftmax <= 4 * kRegsLaunch, "setmaxnreg budget exceeds the CTA's register allocation");
  // the producer is at most this many steps ahead of the softmax: a batch of scales, raw tiles, converted K tiles, one step each being read
  static_assert(6 + kRawK + 1 + kKTiles + 4 <= kScaleSlots, "a step's scales are read before their slot is filled again");
};

// row / group of a tile's row
__device__ __forceinline__ int chunk_row_token(const ChunkParams& p, int row) {
  return p.by_group == 0u ? row : static_cast<int>(__umulhi(static_cast<uint32_t>(row), p.by_group));      // (off by less than 128 / 2^32 < 1 / group)
}

// ------------------------------------------------------------------------------------ the line of units
struct ChunkSeq {              // a sequence: its visible new tokens, the tokens in front of them, and what its tiles cost a head
  int q0, n, ahead, tiles, units;
  bool mine;                   // this kernel's
  __device__ __forceinline__ ChunkSeq() : q0(0), n(0), ahead(0), tiles(0), units(0), mine(false) {}
  __device__ __forceinline__ ChunkSeq(const ChunkParams& p, int s, bool report) {
    auto cu = [&](int i) { return min(max(p.cu[i], 0), p.n_rows); };
    const int first = cu(s), given = max(cu(s + 1) - first, 0);
    const long long most = static_cast<long long>(p.max_blocks) << p.c.bs_log2;
    int len = max(p.seq_lens[s], 0);
    if (len > most || given > p.max_new) {
      if (report) raise_status(p.status, DEV_ERR_CACHE_RANGE);
      len = given > p.max_new ? 0 : static_cast<int>(most);
    }
    mine = given <= p.max_new && static_cast<long long>(given) * p.group > p.few_rows;
    if (!mine) len = 0;
    n = min(given, len);
    q0 = first + given - n;
    ahead = len - n;
    tiles = (n + p.tile_tokens - 1) / p.tile_tokens;
    units = (tiles + 1) >> 1;
  }
  // units 0 .. j - 1 cost, j < units: two tiles each, seeing ahead + 2 tile_tokens (i + 1) tokens
  __device__ __forceinline__ long long before(int j, int tile_tokens) const {
    return static_cast<long long>(j) * (kChunkUnitCost + 2LL * ahead) + 2LL * tile_tokens * j * (j + 1);
  }
  __device__ __forceinline__ bool single(int j) const { return 2 * j + 1 == tiles; }      // a unit of one tile
  __device__ __forceinline__ int seen(int j, int tile_tokens) const {                     // tokens that a unit's last row sees
    return ahead + static_cast<int>(min(static_cast<long long>(n), 2LL * tile_tokens * (j + 1)));
  }
  __device__ __forceinline__ long long cost(int j, int tile_tokens) const {
    return kChunkUnitCost + (single(j) ? 1LL : 2LL) * seen(j, tile_tokens);
  }
  __device__ __forceinline__ long long total(int tile_tokens) const {
    return units == 0 ? 0 : before(units - 1, tile_tokens) + cost(units - 1, tile_tokens);
  }
};

// Prefix sums over the sequences of what they cost, all heads, by a CTA of 512 threads: prefix[0 .. n_seqs]
__device__ __forceinline__ void chunk_prefix(const ChunkParams& p, long long* prefix, long long* sums, bool report) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long cost = 0;
  if (threadIdx.x < p.n_seqs) cost = ChunkSeq(p, threadIdx.x, report).total(p.tile_tokens) * p.c.n_kv;
  long long incl = cost;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  for (int w = 0; w < warp; ++w) incl += sums[w];
  if (threadIdx.x < p.n_seqs) prefix[threadIdx.x + 1] = incl;
  if (threadIdx.x == 0) prefix[0] = 0;
  __syncthreads();
}

struct ChunkLine {
  long long total, whole;
  int pieces, rest;
  __device__ __forceinline__ ChunkLine(long long cost, int device_pieces)
      : total(cost), pieces(static_cast<int>(min(static_cast<long long>(device_pieces), (cost + kChunkLeastCost - 1) / kChunkLeastCost))) {
    whole = pieces == 0 ? 0 : total / pieces;
    rest = static_cast<int>(total - whole * pieces);
  }
  __device__ __forceinline__ int piece_of(long long x) const {      // the one that holds position x
    int at = static_cast<int>(x / (whole + 1));                    // (the pieces are `whole` or one more long)
    while (at + 1 < pieces && begin(at + 1) <= x) ++at;
    return at;
  }
  __device__ __forceinline__ long long begin(int piece) const { return whole * piece + min(piece, rest); }      // (the first `rest` pieces are one more long)
};

// A unit and its place on the line
struct ChunkUnit {
  ChunkSeq seq;
  int s, head, j;
  long long at;                // where it begins
  int tiles, steps;            // its tiles; key steps up to its last row's end
  __device__ __forceinline__ void settle(const ChunkParams& p) {
    tiles = seq.single(j) ? 1 : 2;
    steps = (seq.seen(j, p.tile_tokens) + kChunkKeys - 1) / kChunkKeys;
  }
  // the unit that holds position x < total
  __device__ __forceinline__ void find(const ChunkParams& p, const long long* prefix, long long x) {
    int lo = 0, hi = p.n_seqs - 1;
    while (lo < hi) {                                              // the last sequence that begins at or before x (those without units are passed over)
      const int mid = (lo + hi + 1) >> 1;
      if (prefix[mid] <= x) lo = mid; else hi = mid - 1;
    }
    s = lo;
    seq = ChunkSeq(p, s, false);
    const long long a_head = seq.total(p.tile_tokens);
    x -= prefix[s];
    lo = 0;
    hi = p.c.n_kv - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (mid * a_head <= x) lo = mid; else hi = mid - 1;
    }
    head = lo;
    x -= head * a_head;
    lo = 0;
    hi = seq.units - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (seq.before(mid, p.tile_tokens) <= x) lo = mid; else hi = mid - 1;
    }
    j = lo;
    at = prefix[s] + head * a_head + seq.before(j, p.tile_tokens);
    settle(p);
  }
  __device__ __forceinline__ long long end(const ChunkParams& p) const { return at + seq.cost(j, p.tile_tokens); }
  __device__ __forceinline__ void next(const ChunkParams& p, const long long* prefix, long long line_end) {      // (past the last unit: at is the line's end)
    at = end(p);
    if (++j == seq.units) {
      j = 0;
      if (++head == p.c.n_kv) {
        head = 0;
        if (at >= line_end) return;
        do ++s; while (prefix[s + 1] == prefix[s]);
        seq = ChunkSeq(p, s, false);
      }
    }
    settle(p);
  }
  // the first key step at or behind position x of the line: step k begins at `at` + unit cost + tiles * 80 k
  __device__ __forceinline__ int step_at(long long x) const {
    const long long in = x - at - kChunkUnitCost, width = static_cast<long long>(tiles) * kChunkKeys;
    if (in <= 0) return 0;
    if (in >= steps * width) return steps;
    return static_cast<int>((static_cast<uint32_t>(in) + static_cast<uint32_t>(width) - 1u) / static_cast<uint32_t>(width));      // (below 2^32: a sequence has at most 2^30 places)
  }
  __device__ __forceinline__ int steps_of_tile(const ChunkParams& p, int w) const {
    const long long last = min(static_cast<long long>(seq.n), static_cast<long long>(2 * j + w + 1) * p.tile_tokens);
    return (seq.ahead + static_cast<int>(last) + kChunkKeys - 1) / kChunkKeys;
  }
};
// The items of a CTA in order: of each unit in its pieces, the steps [lo, hi), never none
struct ChunkDeal {
  ChunkLine line;
  ChunkUnit u;
  int piece, lo, hi;
  long long end;
  bool fresh, more;            // the next item is the first one of `piece`; there is a present one
  __device__ __forceinline__ ChunkDeal(long long cost, int n_ctas) : line(cost, n_ctas), piece(blockIdx.x), lo(0), hi(0), end(0), fresh(true), more(true) {}
  __device__ __forceinline__ void next(const ChunkParams& p, const long long* prefix) {
    do {
      if (fresh) {
        more = piece < line.pieces;
        if (!more) return;
        const long long begin = line.begin(piece);
        end = line.begin(piece + 1);
        u.find(p, prefix, begin);
        lo = u.step_at(begin);
        fresh = false;
      } else {
        u.next(p, prefix, line.total);
        lo = 0;
      }
      if (u.at >= end) {
        piece += gridDim.x;
        fresh = true;
        hi = 0;
      } else {
        hi = u.step_at(min(end, u.end(p)));
      }
    } while (lo >= hi);
  }
};
static_assert(sizeof(ChunkDeal) <= kChunkDealBytes, "its place in shared memory");
// What the other roles know of an item
struct alignas(16) ChunkItem {
  int lo, n;                   // its first key step and how many (0: there is no further item)
  int tiles, mine[2];          // its tiles; of two, how many of the steps each has keys in
  int q0, tok0, n_tok, ahead;  // the sequence's first visible row, the unit's first token of those, their number, the tokens in front
  int head, s, seen;           // key/value head, sequence, tokens that the unit's last row sees
  int slot;                    // of the workspace; -1: the item is the whole unit
  int parts;                   // of the unit's first item, if it is cut: in how many pieces the unit has steps
  int pad[2];
};
static_assert(sizeof(ChunkItem) == 64, "four loads");

// ------------------------------------------------------------------------------------ small pieces
// warp_mbar_wait in a few instructions: it stands in some twenty places, and the roles' loops share the instruction caches (see the measurements below).  The
// bound is the same; a wait that ends by it raises the CTA's abort flag, and the others end by their own.
__device__ __forceinline__ bool chunk_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  if (__builtin_expect(__all_sync(0xffffffffu, ok), 1)) return true;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .u32 t0, t1;\n\t"
      "mov.u32 t0, %%clock;\n\t"
      "LOOP%=:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE%=;\n\t"
      "mov.u32 t1, %%clock;\n\t"
      "sub.u32 t1, t1, t0;\n\t"
      "setp.lt.u32 p, t1, 2000000000;\n\t"
      "@p bra LOOP%=;\n\t"
      "setp.ne.u32 p, t1, t1;\n\t"
      "DONE%=:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  if (__all_sync(0xffffffffu, ok)) return true;
  *abort_flag = 1u;
  return false;
}
// barriers by their address in shared memory
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_arrive_if(uint32_t bar, bool pred) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(static_cast<uint32_t>(pred)) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(smem_dst)), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// f(integral constant i), one body for each i < N: a matrix instruction takes its descriptors from uniform registers, and what is not a constant to the
// compiler is moved there for every one
template <int N, typename F>
__device__ __forceinline__ void for_constant(uint32_t i, F f) {
  if (i == N - 1) f(std::integral_constant<int, N - 1>{});
  else if constexpr (N > 1) for_constant<N - 1>(i, f);
}
__host__ __device__ constexpr uint32_t make_idesc_f16(int m, int n, int a_mn, int b_mn) {
  return make_idesc_bf16(m, n, a_mn, b_mn) & ~((1u << 7) | (1u << 10));
}
// Which row of ROWS and which 16 dimensions a lane takes, so that the eight lanes that go together read 128 bytes side by side, or two rows' different
// halves, and store (below) to all banks
template <int HD>
__device__ __forceinline__ int2 lane_place(int lane) {             // (row, chunk)
  if constexpr (HD == 64) return make_int2(lane >> 2, lane & 3);
  else return make_int2(((lane >> 2) & 1) | ((lane >> 4) << 1), (lane & 3) | ((((lane >> 2) ^ (lane >> 3)) & 1) << 2));
}
// 16 fp16 dimensions 16 c .. of row r of a tile whose rows are 128 bytes an atom of 64 dimensions, 128-byte swizzle
__device__ __forceinline__ void store_row_16(uint32_t tile, uint32_t atom_bytes, int r, int c, const uint32_t (&h)[8]) {
  const uint32_t at = tile + (c >> 2) * atom_bytes + r * 128 + (((2 * (c & 3)) ^ (r & 7)) << 4);
  sts128(at, h[0], h[1], h[2], h[3]);
  sts128(at ^ 16, h[4], h[5], h[6], h[7]);
}

// ------------------------------------------------------------------------------------ the kernel
template <int HD, typename T>
__global__ void __launch_bounds__(ChunkCfg<HD>::kThreads, 1) chunk_attention_kernel(const __grid_constant__ ChunkParams p) {
  using L = ChunkCfg<HD>;
  constexpr int NRK = L::kRawK, NR = NRK + L::kRawV, NK = L::kKTiles, NV = L::kVTiles, KEYS = kChunkKeys, PARTS = kChunkParts, NS = L::kScaleSlots;
  extern __shared__ uint8_t smem_raw_chunk[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw_chunk) + 1023) & ~uintptr_t(1023));
  long long* prefix = reinterpret_cast<long long*>(smem + L::kPrefixOff);
  float* sc_ring = reinterpret_cast<float*>(smem + L::kScaleOff);
  float* row_factor = reinterpret_cast<float*>(smem + L::kRowOff);        // what a row's scores are multiplied by
  float2* ml_smem = reinterpret_cast<float2*>(smem + L::kMlOff);
  // barriers: addresses in shared memory, 8 bytes each
  const uint32_t smem_at = smem_u32(smem);
  const uint32_t raw_full = smem_at + L::kBarOff;         // [NR] bytes of a tile landed: NRK of keys, the others of values
  const uint32_t raw_empty = raw_full + 8 * NR;           // [NR] converted
  const uint32_t k_full = raw_empty + 8 * NR;             // [NK] fp16 tile written
  const uint32_t k_empty = k_full + 8 * NK;               // [NK] every issuer hands every tile back
  const uint32_t v_full = k_empty + 8 * NK;               // [NV]
  const uint32_t v_empty = v_full + 8 * NV;               // [NV]
  const uint32_t sc_full = v_empty + 8 * NV;              // [NS] scales of a step written
  const uint32_t q_full = sc_full + 8 * NS;               // [2] queries and their rows' factors
  const uint32_t q_empty = q_full + 16;                   // [2] by both issuers and all softmax warps
  const uint32_t s_full = q_empty + 16;                   // [2] scores of a step complete
  const uint32_t p_ready = s_full + 16;                   // [2] P stored, O rescaled if it had to be
  const uint32_t s_free = p_ready + 16;                   // [2] scores read out of tensor memory
  const uint32_t pv_done = s_free + 16;                   // [2] P V of a step complete
  const uint32_t met = pv_done + 16;                      // [2] alternate: both warpgroups' sums are there; both have read O
  const uint32_t item_full = met + 16;                    // [kChunkItems]
  const uint32_t item_empty = item_full + 8 * kChunkItems;      // by the 15 other warps
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kBarOff + 8 * L::kBars);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  long long* scan_sums = reinterpret_cast<long long*>(tmem_slot + 2);                    // [16]

  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NR; ++i) { mbar_init(raw_full + 8 * i, 1); mbar_init(raw_empty + 8 * i, 2); }
    for (int i = 0; i < NK; ++i) { mbar_init(k_full + 8 * i, 2); mbar_init(k_empty + 8 * i, 2); }
    for (int i = 0; i < NV; ++i) { mbar_init(v_full + 8 * i, 2); mbar_init(v_empty + 8 * i, 2); }
    for (int i = 0; i < NS; ++i) mbar_init(sc_full + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + 8 * i, 4); mbar_init(q_empty + 8 * i, 10); mbar_init(s_full + 8 * i, 1); mbar_init(p_ready + 8 * i, 4);
      mbar_init(s_free + 8 * i, 4); mbar_init(pv_done + 8 * i, 1); mbar_init(met + 8 * i, 8);
    }
    for (int i = 0; i < kChunkItems; ++i) { mbar_init(item_full + 8 * i, 1); mbar_init(item_empty + 8 * i, 15); }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 3) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  if (p.early_launch) pdl_launch_dependents();     // behind the wait: the joining kernel reads the lengths ahead of its own
  chunk_prefix(p, prefix, scan_sums, blockIdx.x == 0);

  auto q_tile = [&](uint32_t slot) { return smem_at + slot * L::kQBytes; };

  ChunkItem* const item_ring = reinterpret_cast<ChunkItem*>(smem + L::kItemOff);
  uint32_t n_items = 0;                            // taken by this warp
  auto take = [&](ChunkItem& it) {                 // the next item; false after an expired wait
    const uint32_t at = n_items % kChunkItems;
    if (!chunk_wait(item_full + 8 * at, (n_items / kChunkItems) & 1u, abort_flag)) return false;
    const uint4* src = reinterpret_cast<const uint4*>(item_ring + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(&it)[i] = src[i];
    __syncwarp();
    mbar_arrive_if(item_empty + 8 * at, lane == 0);
    ++n_items;
    return true;
  };

  if (warp < 4) {
    setmaxnreg_dec<L::kRegsLight>();
    if (warp == 0 || warp == 3) {
      // ------------------------------------------------------------------ bytes: of keys (warp 0, which has the scales too) and of values (warp 3)
      const bool values = warp == 3;
      const int8_t* const cache = values ? p.c.v : p.c.k;
      const uint32_t full = raw_full + (values ? 8 * NRK : 0), empty = raw_empty + (values ? 8 * NRK : 0), ring = values ? NR - NRK : NRK;
      const uint32_t raw = L::kRawOff + (values ? NRK * L::kRawBytes : 0);
      uint32_t g = 0;                              // steps so far
      uint32_t st = 0, free = 1;                   // the ring's next place, and the phase in which it is empty
      // A lane has a part of 16 tokens of the kBatch steps at hand.  Block numbers are asked for two batches ahead and scales one: they come from anywhere in
      // memory.
      constexpr int kBatch = 6;
      static_assert(kBatch * PARTS <= 32, "a lane has a part");
      auto stream = [&](const ChunkItem& it) {
        const int32_t* ids = p.table + it.s * p.ld_table;
        const int my_step = lane / PARTS, my_part = lane - my_step * PARTS, bs = 1 << p.c.bs_log2;
        auto wanted = [&](int j0) { return my_step < kBatch && j0 + my_step < it.n && (it.lo + j0) * KEYS + lane * 16 < it.seen; };
        auto load_id = [&](int j0) { return wanted(j0) ? ids[((it.lo + j0) * KEYS + lane * 16) >> p.c.bs_log2] : -1; };
        auto checked = [&](int id, int j0) {       // (where the number is wanted, not where it is asked for)
          if (static_cast<uint32_t>(id) < static_cast<uint32_t>(p.c.n_blocks)) return id;
          if (wanted(j0)) raise_status(p.status, DEV_ERR_CACHE_RANGE);
          return -1;
        };
        auto load_scales = [&](int id) {
          float2 sc = make_float2(0.f, 0.f);
          if (!values && id >= 0) {
            const long long at = static_cast<long long>(id) * p.c.n_kv + it.head;
            sc = make_float2(p.c.k_scale[at], p.c.v_scale[at]);
          }
          return sc;
        };
        int now = checked(load_id(0), 0), next = load_id(kBatch);
        float2 sc = load_scales(now);
        for (int j0 = 0; j0 < it.n; j0 += kBatch) {
          const int behind = load_id(j0 + 2 * kBatch), steps = min(kBatch, it.n - j0);
          // a lane copies from its part to the end of the block, of the step, or of what there is: the tokens of a head and block lie side by side
          const int place = ((it.lo + j0) * KEYS + lane * 16) & (bs - 1);
          const uint32_t have = __ballot_sync(0xffffffffu, now >= 0), lead = __ballot_sync(0xffffffffu, now >= 0 && (my_part == 0 || place == 0));
          const int bytes = min((bs - place) >> 4, __popc(have >> lane & ((1u << (PARTS - my_part)) - 1u))) * (16 * HD);
          const unsigned long long src = reinterpret_cast<unsigned long long>(cache + (((static_cast<long long>(now) * p.c.n_kv + it.head) << p.c.bs_log2) + place) * HD);
          next = checked(next, j0 + kBatch);
          const float2 sc_next = load_scales(next);
#pragma unroll 1
          for (int i = 0; i < steps; ++i) {
            if (!chunk_wait(empty + 8 * st, free, abort_flag)) return false;
            if (lane == 0) mbar_expect_tx(full + 8 * st, __popc(have >> (i * PARTS) & ((1u << PARTS) - 1u)) * (16u * HD));
            __syncwarp();
            // one elected lane issues, with operands that are the same in all lanes
            for (uint32_t todo = lead & (((1u << PARTS) - 1u) << (i * PARTS)); todo != 0u; todo &= todo - 1u) {
              const int l = __ffs(todo) - 1, n_bytes = __shfl_sync(0xffffffffu, bytes, l);
              const unsigned long long from = __shfl_sync(0xffffffffu, src, l);
              if (elect_one()) bulk_load(smem + raw + st * L::kRawBytes + (l - i * PARTS) * 16 * HD, reinterpret_cast<const void*>(from), n_bytes, full + 8 * st);
              __syncwarp();
            }
            if (++st == ring) { st = 0; free ^= 1u; }
            if (i == 0 && !values) {               // the batch's scales
              if (lane < steps * PARTS) {
                float* dst = sc_ring + (g + my_step) % NS * 16 + my_part;
                const float vs = sc.y < kCacheMinScale ? kCacheMinScale : sc.y, lg = fast_lg2(vs);      // (a NaN stays)
                dst[0] = now >= 0 ? sc.x : 0.f;
                dst[PARTS] = now >= 0 ? lg : -INFINITY;
                dst[2 * PARTS] = now >= 0 ? fast_ex2(-lg) * kWeightDown : 0.f;
              }
              __syncwarp();
              if (lane < steps) mbar_arrive(sc_full + 8 * ((g + lane) % NS));
            }
          }
          g += steps;
          now = next;
          next = behind;
          sc = sc_next;
        }
        return true;
      };
      // Warp 3 walks the line, one item ahead of its values
      if (values && lane == 0)
        for (int piece = blockIdx.x; piece < p.n_ctas; piece += gridDim.x) p.cut_ws[piece].n = 0;
      // (its place on the line lies in shared memory while the warp copies: in registers it costs the loop of the copies its own)
      ChunkDeal* const place = reinterpret_cast<ChunkDeal*>(smem + L::kDealOff);
      if (values && lane == 0) *place = ChunkDeal(prefix[p.n_seqs], p.n_ctas);
      __syncwarp();
      auto put = [&](ChunkItem& it) {
        ChunkDeal deal = *place;
        deal.next(p, prefix);
        __syncwarp();
        if (lane == 0) *place = deal;
        it = ChunkItem{};
        if (deal.more) {
          const ChunkUnit& u = deal.u;
          it.lo = deal.lo;
          it.n = deal.hi - deal.lo;
          it.tiles = u.tiles;
          it.mine[0] = min(deal.hi, u.steps_of_tile(p, 0)) - deal.lo;
          it.mine[1] = min(deal.hi, u.steps_of_tile(p, 1)) - deal.lo;
          it.q0 = u.seq.q0;
          it.tok0 = 2 * u.j * p.tile_tokens;
          it.n_tok = u.seq.n;
          it.ahead = u.seq.ahead;
          it.head = u.head;
          it.s = u.s;
          it.seen = u.seq.seen(u.j, p.tile_tokens);
          it.slot = it.n == u.steps ? -1 : 2 * deal.piece + (deal.hi == u.steps ? 0 : 1);
          if (deal.lo == 0 && deal.hi < u.steps) {
            it.parts = deal.line.piece_of(u.at + kChunkUnitCost + static_cast<long long>(u.tiles) * KEYS * (u.steps - 1)) - deal.piece + 1;
            if (lane == 0) p.cut_ws[deal.piece] = it;
          }
        }
        const uint32_t at = n_items % kChunkItems;
        if (!chunk_wait(item_empty + 8 * at, ((n_items / kChunkItems) & 1u) ^ 1u, abort_flag)) return false;
        if (lane == 0) {
          item_ring[at] = it;
          mbar_arrive(item_full + 8 * at);
        }
        __syncwarp();
        ++n_items;
        return true;
      };
      bool ok = true;
      ChunkItem it;
      it.n = -1;                                   // values: there is none yet
      while (ok && it.n != 0) {
        ChunkItem next;
        ok = values ? put(next) : take(next);
        if (!values) it = next;
        if (ok && it.n > 0) ok = stream(it);
        it = next;
      }
      // every copy has landed before the CTA's shared memory passes to another one: converted, or (after an expired wait) by time
      for (uint32_t e = g < ring ? 0 : g - ring; e < g && ok; ++e) ok = chunk_wait(empty + 8 * (e % ring), (e / ring) & 1u, abort_flag);
      if (!ok) {
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) {}
      }
    } else if (warp <= 2) {
      // ------------------------------------------------------------------ UMMA issuers
      // Every issuer sees every K and V tile of the CTA, in order, and hands back those that it does not use, so that it never mistakes a barrier's phase for
      // another.
      const int w = warp - 1;
      constexpr uint32_t idesc_s = make_idesc_f16(128, KEYS, 0, 0);        // S = Q K^T, both K-major
      constexpr uint32_t idesc_o = make_idesc_f16(128, HD, 0, 1);          // O += P V, V is MN-major
      const uint32_t tm_s = tmem_base + L::kSCol0 + w * L::kSStride, tm_p = tm_s + KEYS, tm_o = tmem_base + w * HD;
      uint32_t qn = 0, n_s = 0, n_p = 0;           // query tiles, scores issued, P waited for
      uint32_t k_st = 0, k_ph = 0, v_st = 0, v_ph = 0;                     // places in the rings, and the phases in which they are filled
      bool ok = true;
      auto next_k = [&]() { if (++k_st == NK) { k_st = 0; k_ph ^= 1u; } };
      auto next_v = [&]() { if (++v_st == NV) { v_st = 0; v_ph ^= 1u; } };
      while (ok) {
        ChunkItem it;
        ok = take(it);
        if (!ok || it.n == 0) break;
        const int n = it.n, tiles = it.tiles;
        const bool alternate = tiles == 1;
        const int first = alternate ? w : 0, stride = alternate ? 2 : 1;
        const int mine = alternate ? n : w == 0 ? it.mine[0] : it.mine[1];      // steps below this are the warpgroup's (every stride-th)
        const int last = mine <= first ? -1 : first + (mine - 1 - first) / stride * stride;
        const uint32_t slot = (qn + (alternate ? 0 : w)) & 1u;
        // queries: wait for each tile of the item, hand back what is not used
        for (int t = 0; t < tiles && ok; ++t, ++qn) {
          ok = chunk_wait(q_full + 8 * (qn & 1u), (qn >> 1) & 1u, abort_flag);
          if (ok && ((qn & 1u) != slot || last < 0)) mbar_arrive_if(q_empty + 8 * (qn & 1u), lane == 0);
        }
        int k_at = 0, v_at = 0;                    // the item's tiles that are dealt with
        // tiles up to `to`, which another warpgroup uses, as soon as they are there
        auto pass_k = [&](int to) {
          for (; k_at < to && ok; ++k_at, next_k()) {
            ok = chunk_wait(k_full + 8 * k_st, k_ph, abort_flag);
            mbar_arrive_if(k_empty + 8 * k_st, lane == 0);
          }
        };
        auto pass_v = [&](int to) {
          for (; v_at < to && ok; ++v_at, next_v()) {
            ok = chunk_wait(v_full + 8 * v_st, v_ph, abort_flag);
            mbar_arrive_if(v_empty + 8 * v_st, lane == 0);
          }
        };
        // the scores of the step behind j, into the warpgroup's columns once they are read, then P V of step j
#pragma unroll 1
        for (int j = first - stride; j <= last && ok; j += stride) {
          if (j < last) {
            pass_k(j + stride);
            if (!ok || !chunk_wait(k_full + 8 * k_st, k_ph, abort_flag) || !chunk_wait(s_free + 8 * w, (n_s & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            tc_fence_after_sync();
            if (elect_one()) {
              for_constant<2 * NK>(slot * NK + k_st, [&](auto c) {
                constexpr int Q = decltype(c)::value / NK, K = decltype(c)::value % NK;
                const uint64_t ad = make_smem_desc(smem_at + Q * L::kQBytes, 16, 1024, kSwizzle128B);
                const uint64_t bd = make_smem_desc(smem_at + L::kKOff + K * L::kTileBytes, 16, 1024, kSwizzle128B);
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h)
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    umma_bf16_ss(tm_s, ad + h * (L::kQHalf >> 4) + 2 * k, bd + h * (L::kAtomBytes >> 4) + 2 * k, idesc_s, h != 0 || k != 0);
              });
              umma_commit(s_full + 8 * w);
              umma_commit(k_empty + 8 * k_st);
              if (j + stride == last) umma_commit(q_empty + 8 * slot);
            }
            __syncwarp();
            ++k_at; next_k();
            ++n_s;
          }
          if (j < first) continue;
          pass_v(j);
          if (!ok || !chunk_wait(v_full + 8 * v_st, v_ph, abort_flag) || !chunk_wait(p_ready + 8 * w, n_p & 1u, abort_flag)) { ok = false; break; }
          ++n_p;
          tc_fence_after_sync();
          if (elect_one()) {
            for_constant<NV>(v_st, [&](auto c) {
              constexpr int V = decltype(c)::value;
              const uint64_t bd = make_smem_desc(smem_at + L::kVOff + V * L::kTileBytes, L::kAtomBytes, 1024, kSwizzle128B);
#pragma unroll
              for (int ks = 0; ks < KEYS / 16; ++ks)             // 16 keys: 8 columns of P, 2 KB of V
                umma_bf16_ts(tm_o, tm_p + ks * 8, bd + ks * (2048 >> 4), idesc_o, (j != first || ks != 0) ? 1u : 0u);
            });
            umma_commit(pv_done + 8 * w);
            umma_commit(v_empty + 8 * v_st);
          }
          __syncwarp();
          ++v_at; next_v();
        }
        pass_k(n);
        pass_v(n);
      }
      // the last hand-backs are asynchronous arrivals: in before the CTA ends
      if (w == 0) {
        for (int i = 0; i < NK && ok; ++i, next_k()) ok = chunk_wait(k_empty + 8 * k_st, k_ph ^ 1u, abort_flag);
        for (int i = 0; i < NV && ok; ++i, next_v()) ok = chunk_wait(v_empty + 8 * v_st, v_ph ^ 1u, abort_flag);
        for (int i = 0; i < 2 && ok; ++i, ++qn) ok = chunk_wait(q_empty + 8 * (qn & 1u), ((qn >> 1) & 1u) ^ 1u, abort_flag);
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------------ converters
    setmaxnreg_dec<L::kRegsConvert>();
    const int cw = warp - 4;
    constexpr int CHUNKS = HD / 16, ROWS = 32 / CHUNKS;                    // 16 dimensions a lane, rows a warp takes at once
    const int2 place = lane_place<HD>(lane);
    const int sub = place.x, chunk = place.y;
    uint32_t qn = 0;
    bool ok = true;
    // The next raw tile to fp16: keys by one pair of warps, values by the other.  (One small loop body: the code of all roles shares the instruction caches.)
    const bool keys = cw < 2;
    constexpr int STEP = 2 * ROWS, BATCH = 5, PASSES = KEYS / STEP;        // rows that a pair takes at once
    static_assert(KEYS % STEP == 0 && PASSES % BATCH == 0 && STEP % 8 == 0, "whole passes; a row's place in its swizzle pattern stays");
    const int row = (cw & 1) * ROWS + sub;
    const uint32_t raw0 = smem_at + L::kRawOff + (keys ? 0 : NRK) * L::kRawBytes + chunk * 16 + row * HD;
    const uint32_t tile0 = smem_at + (keys ? L::kKOff : L::kVOff) + (chunk >> 2) * L::kAtomBytes + row * 128 + (((2 * (chunk & 3)) ^ (row & 7)) << 4);
    const uint32_t from_full = raw_full + (keys ? 0 : 8 * NRK), from_empty = raw_empty + (keys ? 0 : 8 * NRK);
    const uint32_t full = keys ? k_full : v_full, empty = keys ? k_empty : v_empty;
    const uint32_t raws = keys ? NRK : NR - NRK, ring = keys ? NK : NV;
    uint32_t st = 0, landed = 0, to = 0, gone = 1;                         // places in the two rings, and the phases to wait for
    auto convert = [&]() {
      if (!chunk_wait(from_full + 8 * st, landed, abort_flag) || !chunk_wait(empty + 8 * to, gone, abort_flag)) return false;
      const uint32_t src = raw0 + st * L::kRawBytes, dst = tile0 + to * L::kTileBytes;
#pragma unroll 1
      for (int i0 = 0; i0 < PASSES; i0 += BATCH) {
        uint4 x[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) x[i] = lds128(src + (i0 + i) * STEP * HD);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const uint32_t at = dst + (i0 + i) * STEP * 128;
          sts128(at, bytes02_to_half2(x[i].x), bytes02_to_half2(x[i].x >> 8), bytes02_to_half2(x[i].y), bytes02_to_half2(x[i].y >> 8));
          sts128(at ^ 16, bytes02_to_half2(x[i].z), bytes02_to_half2(x[i].z >> 8), bytes02_to_half2(x[i].w), bytes02_to_half2(x[i].w >> 8));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      mbar_arrive_if(from_empty + 8 * st, lane == 0);
      mbar_arrive_if(full + 8 * to, lane == 0);
      if (++st == raws) { st = 0; landed ^= 1u; }
      if (++to == ring) { to = 0; gone ^= 1u; }
      return true;
    };
    auto queries = [&](const ChunkItem& u, int t) {
      const uint32_t slot = qn & 1u;
      constexpr int QBATCH = 2;
      const int rows = min(u.n_tok - u.tok0 - t * p.tile_tokens, p.tile_tokens) * p.group;      // (what the rows behind hold does not matter)
      const uint16_t* const from = p.q + static_cast<long long>(u.q0 + u.tok0 + t * p.tile_tokens) * p.ld_q + u.head * p.group * HD + chunk * 16;
#pragma unroll 1
      for (int row0 = cw * ROWS; row0 == cw * ROWS || row0 - cw * ROWS < rows; row0 += QBATCH * 4 * ROWS) {
        uint4 x[QBATCH][2];
#pragma unroll
        for (int i = 0; i < QBATCH; ++i) {
          const int row = row0 + i * 4 * ROWS + sub, row_tok = chunk_row_token(p, row);
          x[i][0] = x[i][1] = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows) {
            const uint4* src = reinterpret_cast<const uint4*>(from + row_tok * p.ld_q + (row - row_tok * p.group) * HD);
            x[i][0] = src[0];
            x[i][1] = src[1];
          }
        }
        if (row0 == cw * ROWS && !chunk_wait(q_empty + 8 * slot, ((qn >> 1) & 1u) ^ 1u, abort_flag)) return false;
#pragma unroll
        for (int i = 0; i < QBATCH; ++i) {
          const int row = row0 + i * 4 * ROWS + sub;
          const uint32_t xw[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
          // the row's largest magnitude: as 16-bit integers, which order Inf above every number and NaN above Inf
          uint32_t m2 = 0;
#pragma unroll
          for (int b = 0; b < 8; ++b) m2 = __vmaxu2(m2, xw[b] & 0x7FFF7FFFu);
          uint32_t m = max(m2 & 0xFFFFu, m2 >> 16);
#pragma unroll
          for (int d = 1; d < 4; d *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
          if constexpr (HD == 128) m = max(m, __shfl_xor_sync(0xffffffffu, m, 8));
          const float mx = load16(static_cast<uint16_t>(m), std::is_same_v<T, __half>);
          // the largest of the row to [2^14, 2^15) (fp16 ends at 65504), by an exponent of -126 to 126, so that both powers are normal numbers: an
          // element is off by at most 2^-25 of these, 2^-39 of the row's largest (bf16 above 2^-31 of the largest and fp16 above 2^-28 are exact)
          const int e = m != 0u ? min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127 - 14, -126), 126) : 0;
          const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23), up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
          const uint64_t down2 = pack2(down, down);
          uint32_t h[8];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float y0, y1, y2, y3;
            unpack2(fmul2(pack2(Pair16<T>::lo(xw[2 * b]), Pair16<T>::hi(xw[2 * b])), down2), y0, y1);          // (exact, and so is its rounding to fp16 but for what is lost)
            unpack2(fmul2(pack2(Pair16<T>::lo(xw[2 * b + 1]), Pair16<T>::hi(xw[2 * b + 1])), down2), y2, y3);
            h[2 * b] = Pair16<__half>::pack(y0, y2);
            h[2 * b + 1] = Pair16<__half>::pack(y1, y3);
          }
          store_row_16(q_tile(slot), L::kQHalf, row, chunk, h);
          // (an infinite element makes the row NaN: of -Inf alone its scores would count as masked)
          if (chunk == 0) row_factor[slot * 128 + row] = mx * 0.f == 0.f ? p.scale_log2 * up : __uint_as_float(0x7FFFFFFFu);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      mbar_arrive_if(q_full + 8 * slot, lane == 0);
      ++qn;
      return true;
    };
    while (ok) {
      ChunkItem it;
      ok = take(it);
      if (!ok || it.n == 0) break;
      const int n = it.n;
      for (int t = 0; t < it.tiles && ok; ++t) ok = queries(it, t);
#pragma unroll 1
      for (int j = 0; j < n && ok; ++j) ok = convert();
    }
  } else {
    // ------------------------------------------------------------------ softmax warpgroups
    setmaxnreg_inc<L::kRegsSoftmax>();
    const int w = (warp - 8) >> 2, quarter = warp & 3;                     // (the quarter of the tensor memory's lanes that the warp reads)
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + L::kSCol0 + w * L::kSStride, p_addr = s_addr + KEYS, o_addr = lane_addr + w * HD;
    const int row = quarter * 32 + lane, row_tok = chunk_row_token(p, row);
    uint32_t base = 0, qn = 0, n_s = 0, n_met = 0;                         // steps of the CTA, query tiles, the warpgroup's steps, meetings
    bool ok = true;
    while (ok) {
      ChunkItem u;
      ok = take(u);
      if (!ok || u.n == 0) break;
      const int n = u.n, tiles = u.tiles;
      const bool alternate = tiles == 1;
      const int first = alternate ? w : 0, stride = alternate ? 2 : 1;
      const int mine = alternate ? n : w == 0 ? u.mine[0] : u.mine[1];
      const uint32_t slot = (qn + (alternate ? 0 : w)) & 1u;
      float factor = 0.f;
      for (int t = 0; t < tiles && ok; ++t) {
        const uint32_t q = qn + t;
        ok = chunk_wait(q_full + 8 * (q & 1u), (q >> 1) & 1u, abort_flag);
        if (!ok) break;
        if ((q & 1u) == slot) factor = row_factor[slot * 128 + row];
        __syncwarp();
        mbar_arrive_if(q_empty + 8 * (q & 1u), lane == 0);
      }
      qn += tiles;
      if (!ok) break;
      // (what the end needs is put together here: the item's fields would cost the steps their registers)
      const int tok = u.tok0 + (alternate ? 0 : w) * p.tile_tokens + row_tok;
      const bool stored = row_tok < p.tile_tokens && tok < u.n_tok;
      const bool active = __any_sync(0xffffffffu, stored);                 // a warp without a row that is stored only keeps the barriers going
      const int part = u.slot < 0 ? -1 : u.slot * 2 + (alternate ? 0 : w);  // of the workspace; -1: the item is the whole unit
      uint16_t* const dst = p.out + static_cast<long long>(u.q0 + (stored ? tok : 0)) * p.ld_out + (u.head * p.group + row - row_tok * p.group) * HD;
      int left = stored ? u.ahead + tok + 1 - (u.lo + first) * KEYS : 0x7fffffff;      // keys from the present step on that this row sees (rows that are not stored: all, for what they compute does not matter)
      float m_ref = -INFINITY;
      uint64_t l2 = 0;                             // row sum, two halves
      bool any = false;                            // O holds a step of the item
      if (!active) {
        for (int j = first; j < mine && ok; j += stride) {
          ok = chunk_wait(s_full + 8 * w, n_s & 1u, abort_flag);
          ++n_s;
          mbar_arrive_if(s_free + 8 * w, lane == 0);
          ok = ok && chunk_wait(pv_done + 8 * w, n_s & 1u, abort_flag);    // (in front of it, p_ready may still be in the phase before)
          mbar_arrive_if(p_ready + 8 * w, lane == 0);
        }
      }
      const int fewer = stored ? stride * KEYS : 0;
#pragma unroll 1
      for (int j = first; j < mine && active; j += stride, left -= fewer) {
        const uint32_t g = base + j;
        // factors of the step's parts, beside the product
        if (!chunk_wait(sc_full + 8 * (g % NS), (g / NS) & 1u, abort_flag)) { ok = false; break; }
        float sc[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 x = reinterpret_cast<const float4*>(sc_ring + (g % NS) * 16)[i];
          sc[4 * i] = x.x; sc[4 * i + 1] = x.y; sc[4 * i + 2] = x.z; sc[4 * i + 3] = x.w;
        }
#pragma unroll
        for (int m = 0; m < PARTS; ++m) sc[m] *= factor;
        if (!chunk_wait(s_full + 8 * w, n_s & 1u, abort_flag)) { ok = false; break; }
        ++n_s;
        tc_fence_after_sync();
        uint32_t s[KEYS];
        tmem_ld_32x32_at<0>(s_addr, s);
        tmem_ld_32x32_at<32>(s_addr, s);
        tmem_ld_32x16_at<64>(s_addr, s);
        tmem_ld_wait_16<0>(s); tmem_ld_tie_16<16>(s); tmem_ld_tie_16<32>(s); tmem_ld_tie_16<48>(s); tmem_ld_tie_16<64>(s);
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(s_free + 8 * w, lane == 0);
        if (__builtin_expect(__any_sync(0xffffffffu, left < KEYS), 0)) {
          // keys that the row does not see: -inf, against factors that are not 0; a part that it does not see at all has scales of its own (NaN, maybe)
#pragma unroll
          for (int i = 0; i < KEYS; ++i) if (i >= left) s[i] = 0xff800000u;
#pragma unroll
          for (int m = 0; m < PARTS; ++m) {
            const bool hidden = 16 * m >= left;
            sc[m] = hidden || sc[m] == 0.f ? 1e-37f : sc[m];
            sc[PARTS + m] = hidden ? 0.f : sc[PARTS + m];
            sc[2 * PARTS + m] = hidden ? 0.f : sc[2 * PARTS + m];
          }
        }
        // largest t: of each 16 scores the largest, scaled
        float mx = -INFINITY;
#pragma unroll
        for (int m = 0; m < PARTS; ++m) {
          float c0 = __uint_as_float(s[16 * m]), c1 = __uint_as_float(s[16 * m + 1]);
#pragma unroll
          for (int i = 16 * m + 2; i < 16 * m + 14; i += 4) {
            c0 = fmax3(c0, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
            c1 = fmax3(c1, __uint_as_float(s[i + 2]), __uint_as_float(s[i + 3]));
          }
          c0 = fmax3(c0, __uint_as_float(s[16 * m + 14]), __uint_as_float(s[16 * m + 15]));
          mx = fmaxf(mx, fmaf(fmaxf(c0, c1), sc[m], sc[PARTS + m]));
        }
        // the reference moves to 2^7 below the row's largest t when that comes more than 2^15 above it, and to the first one above -inf
        const float m_old = m_ref;
        const bool moved = mx > m_ref + kRefMoves;
        m_ref = moved ? mx - kRefBelow : m_ref;
        const float mb = m_ref == -INFINITY ? 0.f : m_ref;
        uint64_t sum2 = 0;
        uint32_t pk[KEYS / 2];
#pragma unroll
        for (int m = 0; m < PARTS; ++m) {
          const uint64_t c2 = pack2(sc[m], sc[m]), b2 = pack2(sc[PARTS + m] - mb, sc[PARTS + m] - mb);
          uint64_t part2[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float p0, p1;
            unpack2(ffma2(pack2(__uint_as_float(s[16 * m + 2 * i]), __uint_as_float(s[16 * m + 2 * i + 1])), c2, b2), p0, p1);
            p0 = fast_ex2(p0);
            p1 = fast_ex2(p1);
            part2[i & 1] = i < 2 ? pack2(p0, p1) : fadd2(part2[i & 1], pack2(p0, p1));
            pk[8 * m + i] = Pair16<__half>::pack(p0, p1);
          }
          sum2 = ffma2(fadd2(part2[0], part2[1]), pack2(sc[2 * PARTS + m], sc[2 * PARTS + m]), sum2);
        }
        const uint32_t rescale = __ballot_sync(0xffffffffu, moved && any);
        // P goes where the previous step's was, and O may change: that step's P V has to be complete
        // (at an item's first step it is known to be: the same phase again)
        if (!chunk_wait(pv_done + 8 * w, n_s & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        if (__builtin_expect(rescale != 0u, 0)) {
          const float corr = moved ? fast_ex2(m_old - m_ref) : 1.0f;      // (from no reference: 0)
          l2 = ffma2(l2, pack2(corr, corr), sum2);
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
          l2 = fadd2(l2, sum2);
        }
        __syncwarp();
#pragma unroll
        for (int m = 0; m < PARTS; ++m) tmem_st_32x8_from(p_addr + 8 * m, pk + 8 * m);      // (eight registers at a time can be those that the scores had)
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(p_ready + 8 * w, lane == 0);
        any = true;
      }
      base += n;
      if (!ok) break;
      any = first < mine;
      // the item's end
      if (any) {
        if (!chunk_wait(pv_done + 8 * w, (n_s - 1u) & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
      }
      float l, l_hi;
      unpack2(l2, l, l_hi);
      l += l_hi;
      float m = m_ref, f_own = 1.f, f_other = 0.f;
      bool both = false;
      if (alternate) {
        ml_smem[w * 128 + row] = make_float2(m, l);
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(met, lane == 0);
        if (!chunk_wait(met, n_met & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const float2 other = ml_smem[(1 - w) * 128 + row];
        both = n > 1;                              // (of one step: the first warpgroup's alone)
        const float top = fmaxf(m, other.x);
        f_own = !any ? 0.f : m == -INFINITY && l == l ? 0.f : fast_ex2(m - top);           // (a row of NaN has no reference either)
        f_other = !(both || !any) ? 0.f : other.x == -INFINITY && other.y == other.y ? 0.f : fast_ex2(other.x - top);
        l = (any ? l * f_own : 0.f) + (both || !any ? other.y * f_other : 0.f);
        m = top;
      }
      const float inv = l == 0.f ? 0.f : kWeightDown / l;
      const int col0 = alternate ? w * (HD / 2) : 0, cols = alternate ? HD / 2 : HD;
      // 16 columns of one O (without own steps: the other's), or of both, at a time
      const bool two = alternate && both && any;
      const uint32_t o_first = any || !alternate ? o_addr : lane_addr + (1 - w) * HD, o_second = lane_addr + (1 - w) * HD;
      const float scale = part < 0 ? inv : 1.f, f_first = (any || !alternate ? f_own : f_other) * scale, f_second = f_other * scale;
#pragma unroll 1
      for (int c = col0; c < col0 + cols && active; c += 16) {
        uint32_t o[16], x[16];
        __syncwarp();
        tmem_ld_32x16(o_first + c, o);
        if (two) tmem_ld_32x16(o_second + c, x);
        tmem_ld_wait_16<0>(o);
        tmem_ld_tie_16<0>(x);
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float v = __uint_as_float(o[i]) * f_first;
          y[(i & ~3) | ((i & 1) << 1) | ((i >> 1) & 1)] = two ? fmaf(__uint_as_float(x[i]), f_second, v) : v;      // four dimensions lie in the order 0, 2, 1, 3
        }
        if (stored && part < 0) {
#pragma unroll
          for (int i = 0; i < 16; i += 8) {
            uint32_t z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = Pair16<T>::pack(y[i + 2 * e], y[i + 2 * e + 1]);
            *reinterpret_cast<uint4*>(dst + c + i) = make_uint4(z[0], z[1], z[2], z[3]);
          }
        } else if (stored) {
          float4* to = p.o_ws + (static_cast<long long>(part) * (HD / 4) + c / 4) * p.ws_rows + row;
#pragma unroll
          for (int i = 0; i < 4; ++i) to[i * p.ws_rows] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        }
      }
      if (stored && part >= 0 && (!alternate || w == 0)) p.ml_ws[static_cast<long long>(part) * p.ws_rows + row] = make_float2(l == 0.f ? -INFINITY : m, l);
      if (alternate) {
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(met + 8, lane == 0);
        if (!chunk_wait(met + 8, n_met & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        ++n_met;
      }
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == 3) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicCAS(p.status, DEV_OK, DEV_ERR_WAIT_TIMEOUT);
}

// The parts of cut units put together, in order: 128 threads, one a row, per (first cut of a unit, tile, 8 columns).  Before that, beside the end of the kernel
// that leaves them, the rows that see nothing.  Bound by the latency of three rounds of loads, eight parts at once, and by the parts' bytes where all SMs leave
// some: with 8 units in 18 pieces each, 64 tokens behind 16320, the call takes 42 us (68 when a group of threads met the same piece in every round, and all its
// columns were its own).  (Four parts at once, or two CTAs an SM: 37 -> 42 to 45 for one unit of 148 pieces, the others within 2 %.)
template <int HD>
__global__ void __launch_bounds__(512, 1) chunk_join_kernel(const __grid_constant__ ChunkParams p) {
  constexpr int COLS = 8, CHUNKS = HD / COLS, BATCH = 8;
  // On the whole device this kernel starts beside the one before it, which has let it go behind its own wait: the lengths are final
  if (!p.early_launch) pdl_wait();
  const int lane = threadIdx.x & 31, chunks = p.c.n_kv * p.group * (HD / 8);
  for (int s = blockIdx.x * 16 + (threadIdx.x >> 5); s < p.n_seqs; s += gridDim.x * 16) {
    const ChunkSeq seq(p, s, false);                               // the rows in front of a sequence's visible tokens
    if (!seq.mine) continue;
    for (int r = min(max(p.cu[s], 0), p.n_rows); r < seq.q0; ++r)
      for (int c = lane; c < chunks; c += 32) *reinterpret_cast<uint4*>(p.out + static_cast<long long>(r) * p.ld_out + c * 8) = make_uint4(0u, 0u, 0u, 0u);
  }
  pdl_wait();
  if (p.early_launch) pdl_launch_dependents();
  // the pieces that a unit's first cut ends, listed by each CTA
  __shared__ int cuts[kChunkMaxPieces], counts[16];
  const int warp = threadIdx.x >> 5;
  int n_cuts = 0;
  for (int piece0 = 0; piece0 < p.n_ctas; piece0 += 512) {
    const int piece = piece0 + static_cast<int>(threadIdx.x);
    const bool has = piece < p.n_ctas && p.cut_ws[piece].n != 0;
    const uint32_t with = __ballot_sync(0xffffffffu, has);
    if (lane == 0) counts[warp] = __popc(with);
    __syncthreads();
    int at = n_cuts;
    for (int w = 0; w < 16; ++w) {
      if (w < warp) at += counts[w];
      n_cuts += counts[w];
    }
    if (has) cuts[at + __popc(with & ((1u << lane) - 1u))] = piece;
    __syncthreads();
  }
  const int row = threadIdx.x & 127, row_tok = chunk_row_token(p, row), row_head = row - row_tok * p.group;
  for (int it = blockIdx.x + (threadIdx.x >> 7) * gridDim.x; it < n_cuts * 2 * CHUNKS; it += gridDim.x * 4) {      // (few of them: spread over the CTAs)
    const int piece = cuts[it / (2 * CHUNKS)], t = it / CHUNKS & 1, col0 = it % CHUNKS * COLS;
    const ChunkItem& u = p.cut_ws[piece];
    if (t >= u.tiles) continue;
    const int tok = u.tok0 + t * p.tile_tokens + row_tok, parts = u.parts;
    if (row_tok >= p.tile_tokens || tok >= u.n_tok) continue;
    float m = -INFINITY, l = 0.f, acc[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) acc[i] = 0.f;
    for (int b = 0; b < parts; b += BATCH) {                       // of pieces piece + b ..: the last one's is its first slot
      float ml[BATCH][2], x[BATCH][COLS];
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        ml[e][0] = -INFINITY;
        ml[e][1] = 0.f;
        if (b + e < parts) {
          const long long slot = (2LL * (piece + b + e) + (b + e + 1 == parts ? 0 : 1)) * 2 + t;
          load_floats<2>(reinterpret_cast<const float*>(p.ml_ws + slot * p.ws_rows + row), ml[e]);
          const float4* o = p.o_ws + (slot * (HD / 4) + col0 / 4) * p.ws_rows + row;
          float y[4];
          load_floats<4>(reinterpret_cast<const float*>(o), y);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[e][i] = y[i];
          load_floats<4>(reinterpret_cast<const float*>(o + p.ws_rows), y);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[e][4 + i] = y[i];
        }
      }
      float top = m;
#pragma unroll
      for (int e = 0; e < BATCH; ++e) top = fmaxf(top, ml[e][0]);
      const float old = m == -INFINITY ? 0.f : fast_ex2(m - top);
      if (l == l) l *= old;
#pragma unroll
      for (int i = 0; i < COLS; ++i) acc[i] *= old;
      m = top;
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        const bool any = ml[e][1] != 0.f;                          // (NaN: yes)
        const float f = !any ? 0.f : ml[e][1] == ml[e][1] ? fast_ex2(ml[e][0] - m) : ml[e][1];
        if (any) l = fmaf(ml[e][1], f, l);
#pragma unroll
        for (int i = 0; i < COLS; ++i) acc[i] = any ? fmaf(x[e][i], f, acc[i]) : acc[i];
      }
    }
    const float inv = l == 0.f ? 0.f : kWeightDown / l;
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = p.fp16 ? Pair16<__half>::pack(acc[2 * e] * inv, acc[2 * e + 1] * inv) : Pair16<bf16>::pack(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *reinterpret_cast<uint4*>(p.out + static_cast<long long>(u.q0 + tok) * p.ld_out + (u.head * p.group + row_head) * HD + col0) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

}  // namespace eas
