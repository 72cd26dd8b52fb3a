// Attention of single tokens over the 8-bit cache: out = softmax(scale q K^T) V for one query token a sequence; the query heads of a
// key/value head are the columns of one matrix product.
//
// What bounds it is the cache: 2 head_dim bytes a token and key/value head, read once.  So everything serves the stream of tiles:
// 12 warps an SM (8 for more than 8 query heads a key/value head), each with a ring of two (three) 8 KB stages of its own that it fills itself by
// TMA: nothing is shared between warps, so none waits for another, and some 100 to 190 KB are on their way to every SM.  The products are transposed, S^T = K Q^T and O^T += V^T P^T, so that the tokens
// of a tile fill the 16 rows of mma.sync.m16n8k16 and up to 8 query heads its columns: with single tokens there are 1 to 16 rows of
// queries, of which the 128-row tiles of tcgen05 would leave nearly all empty, and the bytes go from shared memory to registers anyway, to
// become fp16.
// The numbers -127 .. 127 are exact in fp16: 0x6400 | (byte ^ 0x80) is 1152 + number, less 1152 (two bytes by one and-xor and one
// subtraction).  Queries enter as fp16 scaled by a power of two per row (bf16 has fewer bits than fp16: nothing is lost but what is
// below 2^-24 of the row's largest).  A block's key scale multiplies its scores in fp32.  Its value scale v is an exponent: with
// t = score + log2 v and w = 2^(t - m),  out = sum w number / sum w / v,  and w fits fp16 whatever the scales are: m is kept 2^7 below the largest
// t and moves when one comes more than 2^15 above it, so the row's largest w is between 2^7 and 2^15 (fp16 ends at 65504).  w is rounded to 11 bits, and below
// 2^-14 to multiples of 2^-24, which are 2^-31 of the largest or less; the sums are fp32, that of w / v from w before its rounding.  (With m at the largest t
// itself, multiples of 2^-24 of it: 20000 tokens of 3.5 2^-24 each behind one that holds the rest were off by a seventh.)
//
// The tiles of all sequences and heads form one line, cut into as many equal pieces as the device has warps (a function of the device, not of
// sm_budget: the cut, and with it every sum, is the same on a share of the SMs).  Beginning a row of tiles (queries in, output out) costs
// about as much as kRowCost tiles, so a row counts as that many more.  Lengths are read on the device: each CTA sums them up itself.  A piece
// that holds a whole row writes its output.  What is cut leaves (m, l, O): the warps of a CTA, whose pieces are neighbours, put together what
// they hold of one row that goes on behind them, and cache_join_kernel the CTAs' parts and the row's end, all in the order of the pieces.
//
// More than 16 query heads a key/value head are rows of tiles of their own, so the cache is read once for every 16 of them, from L2 where it fits:
// 8 caches of 16384 tokens with 2 key/value heads of 128 take 20 us for 8 query heads each, 24 for 12 or 16, 36 for 32, 60 for 64.
//
// Several new tokens a sequence (CHUNK): their heads are the columns, up to 32 of them here; a column sees the places up to its own token's.  48 sequences of 4096 tokens, 32 and 8
// heads of 128: 75 us with one token, 77 with 2 (8 columns), 96 with 4 (16: two thirds more instructions a tile, 8 warps an SM instead of 12; with 10 to 12 registers spill, 101 to 109).
//
// Measured, back to back in a graph, both launches: 8 caches of 24000 to 65536 tokens (64 heads, 8 of keys and values, of 128) 109 us, 93 % of the copy rate (113
// to 121 among other calls); 48 of up to 8192 (32 and 8 heads of 128) 19.5, of them 9 for the bytes and the rest the chain from the lengths to the first
// tile; 128 of 500 to 3500 (16 heads of 64, one query head each) 90, 69 %: 900 instructions a tile of 64 tokens, three warps a scheduler.  The join is 2 us of it.
#pragma once
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

struct CacheAttnParams {
  CUtensorMap map_k, map_v;    // bytes [blocks * heads * block_size, HD], box of min(block_size, 32) rows, swizzled
  CacheView c;
  const int32_t *table, *seq_lens;
  long long ld_table;
  int n_seqs, max_blocks;
  const uint16_t* q;
  uint16_t* out;
  long long ld_q, ld_out;
  int fp16;                    // type of q and out: 0 bf16, 1 fp16
  int group, row_blocks;       // query heads per key/value head; blocks of 8 NT of them (CHUNK: of the most rows that a sequence has)
  const int32_t* cu;           // CHUNK: rows of each sequence's new tokens, their number, the most of a sequence and the most that this kernel takes
  int n_rows, max_new, most_rows;
  int n_ctas;                  // CTAs of the whole device: the line has kWarps pieces for each
  float scale_log2;            // scale * log2(e)
  float* ml_ws;                // [2 pieces][8 NT rows][2]
  float* o_ws;                 // [2 pieces][8 NT rows][HD]
  uint32_t* status;
  int early_launch;
};

constexpr int kCacheMaxSeqs = 1024;      // sequences of one launch (the prefix sums lie in shared memory)
constexpr int kRowCost = 1;
constexpr float kRefBelow = 7.0f, kRefMoves = 15.0f;      // the reference lies that far below the largest score, and moves when one is that far above it
constexpr float kWeightDown = 0.0078125f;  // 2^-kRefBelow: takes it out of w / v, so that blocks of value scale 2^-100 do not overflow their sum, and of O in the end
constexpr int kCacheJoinThreads = 512;      // (256: 1536 rows of heads are two rounds of the device, 48 ragged caches 24 instead of 19 us)

template <int HD, int NT>
struct CacheAttnCfg {
  static constexpr int kTile = 4096 / HD;           // tokens of a stage
  static constexpr int kHalfBytes = kTile * HD, kStageBytes = 2 * kHalfBytes;  // keys, then values
  static constexpr int kMt = kTile / 16;                       // matrix tiles of 16 tokens
  static constexpr int kWarps = NT == 1 ? 12 : 8, kDepth = NT == 1 ? 2 : 3;    // registers decide
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kRows = 8 * NT;
  static constexpr int kPrefixOff = kWarps * kDepth * kStageBytes;
  static constexpr int kLenOff = kPrefixOff + (kCacheMaxSeqs + 4) * 4;
  static constexpr int kNewOff = kLenOff + kCacheMaxSeqs * 4;                  // CHUNK
  static constexpr int kBarOff = kNewOff + kCacheMaxSeqs * 8;
  static constexpr int kBytes = kBarOff + kWarps * kDepth * 8 + 80 + 1024;     // barriers, words, alignment slack
  static_assert(kBytes <= 232448, "exceeds the shared memory of an SM");
  static_assert(kBytes > 116224, "a second CTA must not fit beside this one");
  static_assert(kThreads >= 256 && kWarps <= 16, "the scan of the lengths takes 256 threads");
};

// The line of tiles: pieces, and the rows of tiles along it.  A row's tiles lie at its end, behind its kRowCost.
struct CacheLine {
  int total, pieces;
  __device__ CacheLine(int cost, int rows, int device_pieces) : total(cost * rows), pieces(min(device_pieces, cost * rows)) {}
  __device__ __forceinline__ int begin(int w) const { return static_cast<int>(static_cast<long long>(w) * total / pieces); }
  __device__ __forceinline__ int piece_of(int x) const {        // the last piece that begins at or before x
    return static_cast<int>((static_cast<long long>(x + 1) * pieces - 1) / total);
  }
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
// bytes 0 and 2 of w as two fp16 numbers (low, high half); bytes 1 and 3: the same of w >> 8
__device__ __forceinline__ uint32_t bytes02_to_half2(uint32_t w) {
  const uint32_t biased = (w & 0x00FF00FFu) ^ 0x64806480u;       // 1024 + (byte ^ 0x80)
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&biased), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float fast_lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// CHUNK: several new tokens a sequence, its last ones.  Their query heads are the columns, in the order of the tokens, and a column sees the places up to its token's
// own; 8 NT columns make a row of tiles.  Sequences of more columns than most_rows belong to another kernel (attention_chunk.cuh).
struct CacheNew {
  int q0, n;                   // the first row that sees something, and how many do
  int given, first;
  __device__ __forceinline__ CacheNew(const CacheAttnParams& p, int s, int len) {
    first = min(max(p.cu[s], 0), p.n_rows);
    given = max(min(max(p.cu[s + 1], 0), p.n_rows) - first, 0);
    n = given > p.max_new || static_cast<long long>(given) * p.group > p.most_rows ? 0 : min(given, len);
    q0 = first + given - n;
  }
};

// Prefix sums over the sequences of what a row of tiles costs (CHUNK: of what all rows of tiles of the sequence do), by a whole CTA of 256 or more threads (4
// sequences a thread): prefix[0 .. n_seqs].
template <int TILE, int ROWS, bool CHUNK>
__device__ __forceinline__ void cache_prefix(const CacheAttnParams& p, int* prefix, int* lens, int2* news, int* sums, bool report) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int t[4], sum = 0;
  if (threadIdx.x < 256) {
    const long long most = static_cast<long long>(p.max_blocks) << p.c.bs_log2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = threadIdx.x * 4 + i;
      int n = s < p.n_seqs ? max(p.seq_lens[s], 0) : 0;
      if (n > most) {
        n = static_cast<int>(most);
        if (report) raise_status(p.status, DEV_ERR_CACHE_RANGE);
      }
      int rows = 1;
      if constexpr (CHUNK) {
        if (s < p.n_seqs) {
          const CacheNew c(p, s, n);
          if (report && c.given > p.max_new) raise_status(p.status, DEV_ERR_CACHE_RANGE);
          rows = (c.n * p.group + ROWS - 1) / ROWS * p.c.n_kv;
          if (rows == 0) n = 0;
          if (news != nullptr) news[s] = make_int2(c.q0, c.n);
        }
      }
      if (lens != nullptr && s < p.n_seqs) lens[s] = n;
      t[i] = sum;
      sum += n > 0 ? ((n + TILE - 1) / TILE + kRowCost) * rows : 0;
    }
  }
  int incl = sum;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  if (threadIdx.x < 256) {
    int base = incl - sum;
    for (int w = 0; w < warp; ++w) base += sums[w];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (threadIdx.x * 4 + i <= p.n_seqs) prefix[threadIdx.x * 4 + i] = base + t[i];
    if (threadIdx.x == 255 && p.n_seqs == kCacheMaxSeqs) prefix[kCacheMaxSeqs] = base + sum;
  }
  __syncthreads();
}

template <int HD, int NT, bool CHUNK = false>
__global__ void __launch_bounds__(CacheAttnCfg<HD, NT>::kThreads, 1) cache_attention_kernel(const __grid_constant__ CacheAttnParams p) {
  using L = CacheAttnCfg<HD, NT>;
  constexpr int TILE = L::kTile, MT = L::kMt, ROWS = L::kRows, WARPS = L::kWarps, DEPTH = L::kDepth;
  extern __shared__ uint8_t smem_raw_cache[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw_cache) + 1023) & ~uintptr_t(1023));
  int* sm_prefix = reinterpret_cast<int*>(smem + L::kPrefixOff);         // cost of a row of tiles, summed over the sequences before
  int* sm_len = reinterpret_cast<int*>(smem + L::kLenOff);
  int2* sm_new = reinterpret_cast<int2*>(smem + L::kNewOff);             // CHUNK: first row, rows' tokens
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBarOff);       // [warp][stage] tile landed
  int* sm_sum = reinterpret_cast<int*>(bars + WARPS * DEPTH);            // [16] sums of the scan's warps; the rows that go on behind the warps
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(sm_sum + 16);
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < WARPS * DEPTH; ++i) mbar_init(&bars[i], 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&p.map_k);
    tma_prefetch_desc(&p.map_v);
  }
  pdl_wait();
  if (p.early_launch) pdl_launch_dependents();     // behind the wait: the joining kernel reads the lengths ahead of its own
  cache_prefix<TILE, ROWS, CHUNK>(p, sm_prefix, sm_len, sm_new, sm_sum, blockIdx.x == 0);
  const int R = p.c.n_kv * p.row_blocks;                         // rows of tiles a sequence has (CHUNK: at most)
  const CacheLine line(sm_prefix[p.n_seqs], CHUNK ? 1 : R, p.n_ctas * WARPS);
  auto blocks_of = [&](int s) { return CHUNK ? (sm_new[s].y * p.group + ROWS - 1) / ROWS : p.row_blocks; };
  auto cost_of = [&](int s) { return CHUNK ? (sm_len[s] + TILE - 1) / TILE + kRowCost : sm_prefix[s + 1] - sm_prefix[s]; };      // of a row of tiles (that has some)
  const int qg = lane >> 2, qt = lane & 3;
  const int box_log2 = min(p.c.bs_log2, 5);
  uint8_t* const ring = smem + warp * DEPTH * L::kStageBytes;
  uint64_t* const full = bars + warp * DEPTH;
  uint32_t issued = 0, done = 0;                                 // tiles of this warp so far: tile i lies in stage i % DEPTH
  bool ok = true;

  for (int cta = blockIdx.x; cta < p.n_ctas && cta * WARPS < line.pieces; cta += gridDim.x) {
    const int piece = cta * WARPS + warp;
    const int begin = line.begin(min(piece, line.pieces)), end = line.begin(min(piece + 1, line.pieces));
    int open_row = -1;                                           // the row that goes on behind this piece
    // the row of tiles at the piece's beginning, and how many tiles the piece has
    int s0 = 0;
    {
      int hi = p.n_seqs - 1;
      const int x = min(begin, line.total - 1) / (CHUNK ? 1 : R);
      while (s0 < hi) {                                          // the last sequence that begins at or before x (those without tiles are passed over)
        const int mid = (s0 + hi + 1) >> 1;
        if (sm_prefix[mid] <= x) s0 = mid; else hi = mid - 1;
      }
    }
    // A walk along the line's rows from the piece's beginning.  One walker issues loads, DEPTH tiles ahead of the one that computes.
    struct Walk {
      int s, row, tile, n_tiles, left;      // sequence, row, next tile, tiles of the row; positions of the piece from the row's end on
      int kvh, len, blocks;                 // the row's key/value head, the sequence's length, its rows a key/value head
      const int32_t* ids;                   // and its line of the block table
    };
    auto at_row = [&](Walk& w) {
      w.blocks = blocks_of(w.s);
      w.kvh = w.blocks == 1 ? w.row : w.row / w.blocks;
      w.len = sm_len[w.s];
      w.ids = p.table + w.s * p.ld_table;
    };
    auto enter = [&](Walk& w) {             // at a row's first tile (or past it, at the piece's beginning)
      while (w.n_tiles <= w.tile && w.left > 0) {                // behind the row's last tile: the next row
        if (++w.row == (CHUNK ? p.c.n_kv * w.blocks : R)) {
          w.row = 0;
          do ++w.s; while (w.s < p.n_seqs && sm_prefix[w.s + 1] == sm_prefix[w.s]);
          if (w.s >= p.n_seqs) { w.left = 0; return; }
        }
        const int cost = cost_of(w.s);
        w.n_tiles = min(cost, w.left) - kRowCost;                // tiles of it that belong to this piece
        w.left -= cost;
        w.tile = 0;
        at_row(w);
      }
    };
    Walk iw;
    {
      const int cost = cost_of(s0), in_seq = begin - sm_prefix[s0] * (CHUNK ? 1 : R), row = in_seq / cost, at = in_seq - row * cost;
      iw.s = s0;
      iw.row = row;
      iw.tile = max(at - kRowCost, 0);
      iw.n_tiles = min(cost, at + end - begin) - kRowCost;
      iw.left = end - begin - (cost - at);
      at_row(iw);
      enter(iw);
    }
    Walk cw = iw;
    auto more = [](const Walk& w) { return w.tile < w.n_tiles; };

    // lane m < MT: block number of the 16 tokens m of the walker's tile (-1: none), and later its scales
    auto load_id = [&](const Walk& w) {
      int id = -1;
      const int tok = w.tile * TILE + lane * 16;
      if (lane < MT && more(w) && tok < w.len) {
        id = w.ids[tok >> p.c.bs_log2];
        if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.c.n_blocks)) {
          raise_status(p.status, DEV_ERR_CACHE_RANGE);
          id = -1;
        }
      }
      return id;
    };
    // The whole warp walks; one elected lane issues, with operands that are the same in all lanes (a TMA operation takes them from uniform
    // registers: lanes with operands of their own would go one after the other).  Returns which 16-token parts have a block.
    auto issue = [&](const Walk& w, int id) {
      const uint32_t st = issued % DEPTH, have = __ballot_sync(0xffffffffu, id >= 0);
      const int at = w.tile * TILE & ((1 << p.c.bs_log2) - 1);     // place of the tile's first token in its block (blocks of 16 begin at every part)
      if (box_log2 == 5) {
        int y[MT / 2];
#pragma unroll
        for (int b = 0; b < MT / 2; ++b)
          y[b] = ((__shfl_sync(0xffffffffu, id, 2 * b) * p.c.n_kv + w.kvh) << p.c.bs_log2) + ((at + 32 * b) & ((1 << p.c.bs_log2) - 1));
        if (elect_one()) {
          mbar_expect_tx(&full[st], __popc(have & 0x55555555u) * (2u * HD * 32u));
#pragma unroll
          for (int b = 0; b < MT / 2; ++b)
            if (have & (1u << (2 * b))) {
              tma_load_2d(ring + st * L::kStageBytes + b * 32 * HD, &p.map_k, &full[st], 0, y[b]);
              tma_load_2d(ring + st * L::kStageBytes + L::kHalfBytes + b * 32 * HD, &p.map_v, &full[st], 0, y[b]);
            }
        }
      } else {
        int y[MT];
#pragma unroll
        for (int b = 0; b < MT; ++b) y[b] = (__shfl_sync(0xffffffffu, id, b) * p.c.n_kv + w.kvh) << 4;
        if (elect_one()) {
          mbar_expect_tx(&full[st], __popc(have) * (2u * HD * 16u));
#pragma unroll
          for (int b = 0; b < MT; ++b)
            if (have & (1u << b)) {
              tma_load_2d(ring + st * L::kStageBytes + b * 16 * HD, &p.map_k, &full[st], 0, y[b]);
              tma_load_2d(ring + st * L::kStageBytes + L::kHalfBytes + b * 16 * HD, &p.map_v, &full[st], 0, y[b]);
            }
        }
      }
      __syncwarp();
      ++issued;
      return have;
    };
    auto load_scales = [&](const Walk& w, int id) {
      float2 sc = make_float2(0.f, 0.f);
      if (id >= 0) {
        const long long at = static_cast<long long>(id) * p.c.n_kv + w.kvh;
        sc = make_float2(p.c.k_scale[at], p.c.v_scale[at]);
      }
      return sc;
    };
    auto advance = [&](Walk& w) {
      ++w.tile;
      enter(w);
    };

    // scales of the tiles under way, the next tile's block numbers
    float2 scales[DEPTH];
    uint32_t some[DEPTH];                                          // which of the 16-token parts have a block
    int next_id = load_id(iw);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      scales[d] = make_float2(0.f, 0.f);
      some[d] = 0;
      if (more(iw)) {
        some[d] = issue(iw, next_id);
        scales[d] = load_scales(iw, next_id);
        advance(iw);
        next_id = load_id(iw);
      }
    }

    while (more(cw) && ok) {
      const int s = cw.s, kvh = cw.kvh, head0 = (cw.row - kvh * cw.blocks) * ROWS;      // head0: within the group
      const int q0 = CHUNK ? sm_new[s].x : s, n_new = CHUNK ? sm_new[s].y : 1;
      const int n_rows = min(ROWS, n_new * p.group - head0);
      const int first = cw.tile, last = cw.n_tiles, row_tiles = cost_of(s) - kRowCost, len = cw.len;
      auto token_of = [&](int r) { return CHUNK ? (head0 + r) / p.group : 0; };                // of row r, and the place of its query or output
      auto at_row_of = [&](int r, long long ld) {
        const int tok = token_of(r);
        return (q0 + tok) * ld + static_cast<long long>(kvh * p.group + head0 + r - tok * p.group) * HD;
      };
      int limit[NT][2];                                          // CHUNK: places that this lane's columns see
      if constexpr (CHUNK) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int b = 0; b < 2; ++b) limit[j][b] = len - n_new + 1 + min(token_of(j * 8 + 2 * qt + b), n_new - 1);
      }
      float m_ref[NT][2], l[NT][2], o[HD / 16][NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        m_ref[j][0] = m_ref[j][1] = -INFINITY;
        l[j][0] = l[j][1] = 0.f;
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.f;
      }
      // queries: column qg of 8, the dims that pair with this lane's bytes of a key row (see the products below)
      uint32_t qf[HD / 16][NT][2];
      float c_row[NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int h = j * 8 + qg;
        float x[HD / 4];
        const uint16_t* src = p.q + at_row_of(CHUNK ? min(h, n_rows - 1) : h, p.ld_q) + qt * (HD / 4);
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
          const uint4 v = h < n_rows ? *reinterpret_cast<const uint4*>(src + i * 8) : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            x[i * 8 + 2 * b] = load16(static_cast<uint16_t>(vw[b] & 0xFFFFu), p.fp16);
            x[i * 8 + 2 * b + 1] = load16(static_cast<uint16_t>(vw[b] >> 16), p.fp16);
          }
        }
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < HD / 4; ++i) mx = fmaxf(mx, fabsf(x[i]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // the largest of the row to [1, 2): exponent e with 2^e <= mx (-126 to 126, so that 2^e and 2^-e are normal numbers: a subnormal row stays below 1,
        // one from 2^127 on below 4)
        const int e = mx > 0.f ? min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127, -126), 126) : 0;
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {
          qf[i][j][0] = Pair16<__half>::pack(x[4 * i] * down, x[4 * i + 2] * down);
          qf[i][j][1] = Pair16<__half>::pack(x[4 * i + 1] * down, x[4 * i + 3] * down);
        }
        // an infinite element makes every score Inf, -Inf or NaN, and the softmax of them NaN (of -Inf alone too: without this they would count as masked)
        const float c = mx == INFINITY ? __uint_as_float(0x7FFFFFFFu) : p.scale_log2 * up;      // of column qg; this lane's scores are columns 2 qt and 2 qt + 1
        c_row[j][0] = __shfl_sync(0xffffffffu, c, 8 * qt);
        c_row[j][1] = __shfl_sync(0xffffffffu, c, 8 * qt + 4);
      }

#pragma unroll 1
      for (int tile = first; tile < last; ++tile) {
        const uint32_t st = done % DEPTH;
        if (!warp_mbar_wait(&full[st], (done / DEPTH) & 1u, abort_flag)) { ok = false; break; }
        ++done;
        const uint32_t kb = smem_u32(ring) + st * L::kStageBytes, vb = kb + L::kHalfBytes;
        // scores: token rows qg and qg + 8 of each 16, columns 2 qt and 2 qt + 1
        float sc[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int j = 0; j < NT; ++j) sc[m][j][0] = sc[m][j][1] = sc[m][j][2] = sc[m][j][3] = 0.f;
          const int ra = m * 16 + qg, rb = ra + 8;
#pragma unroll
          for (int c = 0; c < HD / 64; ++c) {
            // 16 bytes of a row: chunk qt * (HD / 64) + c, at the swizzled place.  Its word i is k-step 4 c + i of the product: bytes
            // 0 and 2 are the lane's columns 2 qt and 2 qt + 1, bytes 1 and 3 its columns 2 qt + 8 and 2 qt + 9
            const int chunk = qt * (HD / 64) + c;
            const uint4 a = lds128(kb + ra * HD + ((HD == 128 ? chunk ^ (ra & 7) : chunk ^ ((ra >> 1) & 3)) << 4));
            const uint4 b = lds128(kb + rb * HD + ((HD == 128 ? chunk ^ (rb & 7) : chunk ^ ((rb >> 1) & 3)) << 4));
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a0 = bytes02_to_half2(aw[i]), a1 = bytes02_to_half2(bw[i]);
              const uint32_t a2 = bytes02_to_half2(aw[i] >> 8), a3 = bytes02_to_half2(bw[i] >> 8);
#pragma unroll
              for (int j = 0; j < NT; ++j) mma_f16(sc[m][j], a0, a1, a2, a3, qf[4 * c + i][j][0], qf[4 * c + i][j][1]);
            }
          }
        }
        // the tile's scales (lane m has those of its tokens 16 m ..): v as log2 v and 2^-kRefBelow / v
        const float vs = scales[0].y < kCacheMinScale ? kCacheMinScale : scales[0].y;      // (a NaN stays)
        const float lane_lg = fast_lg2(vs), lane_inv = fast_ex2(-lane_lg) * kWeightDown;
        float v_inv[MT];
        bool higher = false;
        float mx[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) mx[j][0] = mx[j][1] = -INFINITY;
        const bool cut = tile * TILE + TILE > (CHUNK ? len - n_new + 1 : len) || some[0] != (1u << MT) - 1u;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float ks = __shfl_sync(0xffffffffu, scales[0].x, m), lg = __shfl_sync(0xffffffffu, lane_lg, m);
          v_inv[m] = __shfl_sync(0xffffffffu, lane_inv, m);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const float c0 = c_row[j][0] * ks, c1 = c_row[j][1] * ks;
            sc[m][j][0] = fmaf(sc[m][j][0], c0, lg);
            sc[m][j][1] = fmaf(sc[m][j][1], c1, lg);
            sc[m][j][2] = fmaf(sc[m][j][2], c0, lg);
            sc[m][j][3] = fmaf(sc[m][j][3], c1, lg);
          }
          if (cut) {                                             // tokens behind the sequence's end, or without a block
            const int left = some[0] & (1u << m) ? len - tile * TILE - m * 16 : 0;
            if (left <= 0) v_inv[m] = 0.f;
            if constexpr (CHUNK) {
#pragma unroll
              for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const int seen = min(left, limit[j][b] - tile * TILE - m * 16);
                  if (qg >= seen) sc[m][j][b] = -INFINITY;
                  if (qg + 8 >= seen) sc[m][j][b + 2] = -INFINITY;
                }
            } else {
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                if (qg >= left) sc[m][j][0] = sc[m][j][1] = -INFINITY;
                if (qg + 8 >= left) sc[m][j][2] = sc[m][j][3] = -INFINITY;
              }
            }
          }
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            mx[j][0] = fmax3(mx[j][0], sc[m][j][0], sc[m][j][2]);
            mx[j][1] = fmax3(mx[j][1], sc[m][j][1], sc[m][j][3]);
          }
        }
        // (the first tile: always)
#pragma unroll
        for (int j = 0; j < NT; ++j) higher = higher || mx[j][0] > m_ref[j][0] + kRefMoves || mx[j][1] > m_ref[j][1] + kRefMoves;
        if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              float x = fmaxf(mx[j][b] - kRefBelow, m_ref[j][b]);
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
              const float corr = x == -INFINITY ? 1.0f : fast_ex2(m_ref[j][b] - x);
              m_ref[j][b] = x;
              l[j][b] *= corr;
#pragma unroll
              for (int i = 0; i < HD / 16; ++i) {
                o[i][j][b] *= corr;
                o[i][j][b + 2] *= corr;
              }
            }
        }
        float ref[NT][2];                                        // (no token counted yet: 2^-inf = 0, against any reference)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int b = 0; b < 2; ++b) ref[j][b] = fmaxf(m_ref[j][b], -3.0e38f);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          uint32_t pf[NT][2];
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const float r0 = ref[j][0], r1 = ref[j][1];
            const float w0 = fast_ex2(sc[m][j][0] - r0), w1 = fast_ex2(sc[m][j][1] - r1);
            const float w2 = fast_ex2(sc[m][j][2] - r0), w3 = fast_ex2(sc[m][j][3] - r1);
            if (CHUNK && cut) {                                  // (the scale of a part that the column does not see may be NaN)
              if (limit[j][0] > tile * TILE + m * 16) l[j][0] = fmaf(w0 + w2, v_inv[m], l[j][0]);
              if (limit[j][1] > tile * TILE + m * 16) l[j][1] = fmaf(w1 + w3, v_inv[m], l[j][1]);
            } else {
              l[j][0] = fmaf(w0 + w2, v_inv[m], l[j][0]);
              l[j][1] = fmaf(w1 + w3, v_inv[m], l[j][1]);
            }
            pf[j][0] = transpose_8x8(Pair16<__half>::pack(w0, w1));         // tokens to columns 2 qt, 2 qt + 1, queries to rows
            pf[j][1] = transpose_8x8(Pair16<__half>::pack(w2, w3));
          }
          // values: tokens 2 qt, 2 qt + 1, 2 qt + 8, 2 qt + 9 of the 16, dims qg * (HD / 8) .. of each
          const int r0 = m * 16 + 2 * qt;
          uint32_t v[4][HD / 32];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int r = r0 + (b & 1) + (b >> 1) * 8;
            if constexpr (HD == 128) {
              const uint4 x = lds128(vb + r * HD + ((qg ^ (r & 7)) << 4));
              v[b][0] = x.x; v[b][1] = x.y; v[b][2] = x.z; v[b][3] = x.w;
            } else {
              const uint2 x = lds64(vb + r * HD + (((qg >> 1) ^ ((r >> 1) & 3)) << 4) + (qg & 1) * 8);
              v[b][0] = x.x; v[b][1] = x.y;
            }
          }
#pragma unroll
          for (int i = 0; i < HD / 32; ++i) {
            // word i: dims 4 i .. 4 i + 3 of the lane's; two matrix tiles of 16 dims (rows qg: even dims, qg + 8: odd ones)
            const uint32_t e0 = __byte_perm(v[0][i], v[1][i], 0x5410), e1 = __byte_perm(v[2][i], v[3][i], 0x5410);
            const uint32_t f0 = __byte_perm(v[0][i], v[1][i], 0x7632), f1 = __byte_perm(v[2][i], v[3][i], 0x7632);
            const uint32_t a0 = bytes02_to_half2(e0), a1 = bytes02_to_half2(e0 >> 8), a2 = bytes02_to_half2(e1), a3 = bytes02_to_half2(e1 >> 8);
            const uint32_t b0 = bytes02_to_half2(f0), b1 = bytes02_to_half2(f0 >> 8), b2 = bytes02_to_half2(f1), b3 = bytes02_to_half2(f1 >> 8);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              mma_f16(o[2 * i][j], a0, a1, a2, a3, pf[j][0], pf[j][1]);
              mma_f16(o[2 * i + 1][j], b0, b1, b2, b3, pf[j][0], pf[j][1]);
            }
          }
        }
        // the stage is read: the tile DEPTH ahead goes into it, and the block numbers of the one behind that are asked for
        __syncwarp();
#pragma unroll
        for (int d = 0; d + 1 < DEPTH; ++d) {
          scales[d] = scales[d + 1];
          some[d] = some[d + 1];
        }
        if (more(iw)) {
          some[DEPTH - 1] = issue(iw, next_id);
          scales[DEPTH - 1] = load_scales(iw, next_id);
          advance(iw);
          next_id = load_id(iw);
        }
      }
      if (!ok) break;      // (the CTA's barriers below are still met)

      // the row's part of this piece: lane (qg, qt) has dims qg * (HD / 8) .. of queries 2 qt and 2 qt + 1.  The whole row goes out; a row's end
      // into the workspace; a row that goes on is the last thing this piece has: into the warp's ring, for the CTA.
      const bool ends = last == row_tiles, whole = ends && first == 0;
      float* part = ends ? p.o_ws + 2LL * piece * ROWS * HD : reinterpret_cast<float*>(ring);
      float* part_ml = ends ? p.ml_ws + 4LL * piece * ROWS : reinterpret_cast<float*>(ring) + ROWS * HD;
      if (!ends) open_row = s * R + cw.row;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float x = l[j][b];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          const int r = j * 8 + 2 * qt + b;
          if (r >= n_rows) continue;
          if (whole) {
            const float inv = x == 0.f ? 0.f : kWeightDown / x;
            uint16_t* dst = p.out + at_row_of(r, p.ld_out) + qg * (HD / 8);
#pragma unroll
            for (int i = 0; i < HD / 16; i += 4) {
              uint32_t y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                y[e] = p.fp16 ? Pair16<__half>::pack(o[i + e][j][b] * inv, o[i + e][j][b + 2] * inv) : Pair16<bf16>::pack(o[i + e][j][b] * inv, o[i + e][j][b + 2] * inv);
              *reinterpret_cast<uint4*>(dst + 2 * i) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          } else {
            float* dst = part + r * HD + qg * (HD / 8);
#pragma unroll
            for (int i = 0; i < HD / 16; i += 2)
              *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(o[i][j][b], o[i][j][b + 2], o[i + 1][j][b], o[i + 1][j][b + 2]);
            if (qg == 0) *reinterpret_cast<float2*>(part_ml + r * 2) = make_float2(m_ref[j][b], x);
          }
        }
      cw.tile = last;
      enter(cw);
    }

    // rows that go on behind their pieces: neighbouring warps of one row put theirs together, into the second slot of the first of them
    if (lane == 0) sm_sum[warp] = open_row;
    __syncthreads();
    for (int w0 = 0, w1; w0 < WARPS; w0 = w1) {
      const int row = sm_sum[w0];
      for (w1 = w0 + 1; w1 < WARPS && sm_sum[w1] == row && row >= 0; ++w1) {}
      if (row < 0) continue;
      for (int e = threadIdx.x; e < ROWS * HD / 4; e += L::kThreads) {
        const int r = e / (HD / 4);
        auto ml_of = [&](int w) { return *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(smem + w * DEPTH * L::kStageBytes) + ROWS * HD + r * 2); };
        float m = -INFINITY, l = 0.f;
        for (int w = w0; w < w1; ++w) m = fmaxf(m, ml_of(w).x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = w0; w < w1; ++w) {
          const float2 ml = ml_of(w);
          const float f = ml.x == -INFINITY && ml.y == ml.y ? 0.f : fast_ex2(ml.x - m);
          const float4 x = reinterpret_cast<const float4*>(smem + w * DEPTH * L::kStageBytes)[e];
          l = fmaf(ml.y, f, l);
          acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y);
          acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
        }
        const long long slot = 2LL * (cta * WARPS + w0) + 1;
        reinterpret_cast<float4*>(p.o_ws + slot * ROWS * HD)[e] = acc;
        if (e % (HD / 4) == 0) *reinterpret_cast<float2*>(p.ml_ws + (slot * ROWS + r) * 2) = make_float2(m, l);
      }
    }
    __syncthreads();
    fence_proxy_async_smem();                                    // the rings held plain stores: before the next loads into them
  }
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000) {}     // let loads in flight land before the CTA retires
    if (lane == 0) raise_status(p.status, DEV_ERR_WAIT_TIMEOUT);
  }
}

template <int N>
__device__ __forceinline__ void load_floats(const float* src, float (&x)[N]) {      // (volatile: issued where it stands, not where x is used)
  if constexpr (N == 4) asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "l"(src) : "memory");
  else asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "l"(src) : "memory");
}

// What the CTAs' and pieces' ends cut, put together: one warp per (sequence, query head), the parts in order.  Rows that one piece held are
// there already; sequences without tokens get zeros.
template <int HD, int NT, bool CHUNK = false>
__global__ void __launch_bounds__(kCacheJoinThreads, 1) cache_join_kernel(const __grid_constant__ CacheAttnParams p) {
  constexpr int ROWS = 8 * NT, N = HD / 32, WARPS = CacheAttnCfg<HD, NT>::kWarps;
  __shared__ int prefix[kCacheMaxSeqs + 1], sums[kCacheJoinThreads / 32];
  // On the whole device this kernel starts beside the one before it, which has let it go behind its own wait: the lengths are final
  if (!p.early_launch) pdl_wait();
  constexpr int TILE = CacheAttnCfg<HD, NT>::kTile;
  cache_prefix<TILE, ROWS, CHUNK>(p, prefix, nullptr, nullptr, sums, false);
  const int lane = threadIdx.x & 31, heads = p.c.n_kv * p.group, R = p.c.n_kv * p.row_blocks;
  const CacheLine line(prefix[p.n_seqs], CHUNK ? 1 : R, p.n_ctas * WARPS);
  bool waited = false;
  constexpr int kJoinWarps = kCacheJoinThreads / 32;
  for (int u = blockIdx.x * kJoinWarps + (threadIdx.x >> 5); u < (CHUNK ? p.n_rows : p.n_seqs) * heads; u += gridDim.x * kJoinWarps) {
    const int q_row = u / heads, h = u - q_row * heads, kvh = h / p.group;
    int s = q_row, column = h - kvh * p.group, blocks = p.row_blocks, cost;
    if constexpr (CHUNK) {
      s = last_sequence(p.n_seqs, q_row, [&](int i) { return min(max(p.cu[i], 0), p.n_rows); });
      const int len = min(static_cast<long long>(max(p.seq_lens[s], 0)), static_cast<long long>(p.max_blocks) << p.c.bs_log2);
      const CacheNew c(p, s, len);
      if (q_row < c.first || q_row >= c.first + c.given || c.given > p.max_new || static_cast<long long>(c.given) * p.group > p.most_rows) continue;
      cost = q_row < c.q0 ? 0 : (len + TILE - 1) / TILE + kRowCost;      // 0: it sees nothing
      column += (q_row - c.q0) * p.group;
      blocks = (c.n * p.group + ROWS - 1) / ROWS;
    } else {
      cost = prefix[s + 1] - prefix[s];
    }
    const int row = kvh * blocks + column / ROWS, r = column % ROWS;
    int w0 = 0, w1 = 0;                                            // the row's first and last piece
    if (cost > 0) {
      const int a = prefix[s] * (CHUNK ? 1 : R) + row * cost;
      w0 = line.piece_of(a + kRowCost);
      w1 = line.piece_of(a + cost - 1);
      if (w0 == w1) continue;
    }
    if (!waited) {
      pdl_wait();
      waited = true;
    }
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
    if (cost > 0) {
      // parts: one for each CTA that the row goes on behind, then the row's end in piece w1
      const int c0 = w0 / WARPS, parts = (w1 - 1) / WARPS - c0 + 2;
      auto slot = [&](int i) { return (i + 1 == parts ? 2LL * w1 : 2LL * max(w0, (c0 + i) * WARPS) + 1) * ROWS + r; };
      // 32 at a time: their references and sums, one a lane; their O, 8 in flight, the first asked for along with the references
      float m = -INFINITY, l = 0.f, o[8][N];
      auto fetch = [&](int part) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (part + e < parts) load_floats<N>(p.o_ws + slot(part + e) * HD + lane * N, o[e]);
      };
      for (int base = 0; base < parts; base += 32) {
        const int n = min(32, parts - base);
        float ml[2] = {-INFINITY, 0.f};
        if (lane < n) load_floats<2>(p.ml_ws + slot(base + lane) * 2, ml);
        fetch(base);
        float top = fmaxf(m, ml[0]);
#pragma unroll
        for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float f = ml[0] == -INFINITY && ml[1] == ml[1] ? 0.f : fast_ex2(ml[0] - top);
        const float old = m == -INFINITY ? 0.f : fast_ex2(m - top);
        float sum = ml[1] * f;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l = fmaf(l, old, sum);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= old;
        m = top;
        for (int k = 0; k < n; k += 8) {
          if (k > 0) fetch(base + k);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float fe = __shfl_sync(0xffffffffu, f, (k + e) & 31);
            if (k + e < n) {
#pragma unroll
              for (int i = 0; i < N; ++i) acc[i] = fmaf(o[e][i], fe, acc[i]);
            }
          }
        }
      }
      const float inv = l == 0.f ? 0.f : kWeightDown / l;
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] *= inv;
    }
    uint16_t* dst = p.out + q_row * p.ld_out + static_cast<long long>(h) * HD + lane * N;
#pragma unroll
    for (int i = 0; i < N; i += 2)
      *reinterpret_cast<uint32_t*>(dst + i) = p.fp16 ? Pair16<__half>::pack(acc[i], acc[i + 1]) : Pair16<bf16>::pack(acc[i], acc[i + 1]);
  }
  if (!waited) pdl_wait();                                         // (whoever follows relies on every CTA having waited)
  if (p.early_launch) pdl_launch_dependents();
}

}  // namespace eas
