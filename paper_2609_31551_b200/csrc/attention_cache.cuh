// Attention of single tokens over the 8-bit cache: out = softmax(scale q K^T) V for one query token a sequence; the query heads of a
// key/value head are the columns of one matrix product.
//
// What bounds it is the cache: 2 head_dim bytes a token and key/value head, read once.  So everything serves the stream of tiles:
//   4 producer warps, 4 lanes each: a lane finds the sequence, head and block of its tile and brings keys and values by TMA
//               into a ring of 8 KB stages; a tile's chain (block number, then its bytes and scales) is two trips to memory,
//               and with four warps 16 of them are under way
//   8 or 12 consumer warps take the tiles in turn.  The products are transposed, S^T = K Q^T and O^T += V^T P^T, so that the tokens of a
//               tile fill the 16 rows of mma.sync.m16n8k16 and up to 8 query heads its columns: with single tokens there are 1 to
//               16 rows of queries, of which the 128-row tiles of tcgen05 would leave nearly all empty, and the bytes go
//               from shared memory to registers anyway, to become fp16.
// The numbers -127 .. 127 are exact in fp16: 0x6400 | (byte ^ 0x80) is 1152 + number, less 1152 (two bytes by one and-xor and one
// subtraction).  Queries enter as fp16 scaled by a power of two per row (bf16 has fewer bits than fp16: nothing is lost but what is
// below 2^-24 of the row's largest).  A block's key scale multiplies its scores in fp32.  Its value scale v is an exponent: with
// t = score + log2 v and w = 2^(t - m),  out = sum w number / sum w / v,  so w <= 2^8 fits fp16 whatever the scales are (w is
// rounded to its 11 bits), and the sums are fp32.
//
// The tiles of all sequences and heads form one line, cut into as many equal pieces as the device has SMs (not sm_budget: the cut, and
// with it every sum, is the same on a share of the SMs).  Lengths are read on the device: each CTA sums them up itself.  A piece
// that holds a whole (sequence, head) writes its output; what is cut leaves (m, l, O) in the workspace, and cache_join_kernel puts
// it together, in order.
#pragma once
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

struct CacheAttnParams {
  CUtensorMap map_k, map_v;    // bytes [blocks * heads * block_size, HD], box of min(block_size, tile) rows, swizzled
  CacheView c;
  const int32_t *table, *seq_lens;
  long long ld_table;
  int n_seqs, max_blocks;
  const uint16_t* q;
  uint16_t* out;
  long long ld_q, ld_out;
  int fp16;                    // type of q and out: 0 bf16, 1 fp16
  int group, row_blocks;       // query heads per key/value head; blocks of 8 NT of them
  int n_pieces, min_tiles;
  float scale_log2;            // scale * log2(e)
  int* head_ws;                // [n_seqs + 1] tiles of the sequences before, then the tiles of a piece
  float* ml_ws;                // [2 pieces][8 NT rows][2]
  float* o_ws;                 // [2 pieces][8 NT rows][HD]
  uint32_t* status;
  int early_launch;
};

constexpr int kCacheMaxSeqs = 1024;      // sequences of one launch (the prefix sums lie in shared memory)
constexpr int kCacheProducers = 4;       // producer warps
constexpr int kCacheStep = 4;            // tiles that a producer brings at once

template <int HD, int NT>
struct CacheAttnCfg {
  static constexpr int kTile = 4096 / HD;                      // tokens of a stage
  static constexpr int kMt = kTile / 16;                       // matrix tiles of 16 tokens
  static constexpr int kWarps = NT == 1 ? 12 : 8;              // consumers: their registers decide
  static constexpr int kThreads = 32 * (kWarps + kCacheProducers);
  static constexpr int kRegsProducer = 40, kRegsConsumer = NT == 1 ? 152 : 224, kRegsLaunch = NT == 1 ? 128 : 168;
  static constexpr int kStages = NT == 1 ? 20 : 16;
  static constexpr int kRows = 8 * NT;
  static constexpr int kOPitch = HD + 4;                       // floats: the fragments' float2 stores then cover all banks
  static constexpr int kRingBytes = kStages * 8192;
  static constexpr int kOOff = kRingBytes;
  static constexpr int kMlOff = kOOff + kWarps * kRows * kOPitch * 4;
  static constexpr int kMetaOff = kMlOff + kWarps * kRows * 8;            // [stage][kMt] {key scale, log2 and reciprocal of the value scale, tokens}
  static constexpr int kPrefixOff = kMetaOff + kStages * kMt * 16;
  static constexpr int kLenOff = kPrefixOff + (kCacheMaxSeqs + 4) * 4;
  static constexpr int kBarOff = kLenOff + kCacheMaxSeqs * 4;
  static constexpr int kBytes = kBarOff + 2 * kStages * 8 + (16 + kStages + 4) * 4 + 1024;         // barriers, words, alignment slack
  static_assert(kBytes <= 232448, "exceeds the shared memory of an SM");
  static_assert(kBytes > 116224, "a second CTA must not fit beside this one");
  static_assert(kStages >= kCacheProducers * kCacheStep, "no step waits for a tile of its own or of one under way beside it");
  static_assert(32 * (kWarps * kRegsConsumer + kCacheProducers * kRegsProducer) <= kThreads * kRegsLaunch && kThreads * kRegsLaunch <= 65536,
                "setmaxnreg budget exceeds the CTA's register allocation");
  static_assert(kWarps % 4 == 0 && kCacheProducers % 4 == 0, "setmaxnreg acts on warpgroups");
  static_assert(32 * kWarps >= 256 && kWarps <= 12, "the scan of the lengths takes 256 threads");
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

// Waits (bounded) until *word, in shared memory, is `value`.
__device__ __forceinline__ bool word_wait(const volatile int* word, int value, volatile uint32_t* abort_flag) {
  if (*word == value) return true;
  const long long t0 = clock64();
  uint32_t it = 0;
  while (*word != value) {
    if ((++it & 63u) == 0u) {
      if (*abort_flag) return false;
      if (clock64() - t0 > kWaitCycleLimit) {
        *abort_flag = 1u;
        return false;
      }
    }
  }
  return true;
}

template <int HD, int NT>
__global__ void __launch_bounds__(CacheAttnCfg<HD, NT>::kThreads, 1) cache_attention_kernel(const __grid_constant__ CacheAttnParams p) {
  using L = CacheAttnCfg<HD, NT>;
  constexpr int TILE = L::kTile, MT = L::kMt, NST = L::kStages, ROWS = L::kRows, PITCH = L::kOPitch, WARPS = L::kWarps;
  extern __shared__ uint8_t smem_raw_cache[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw_cache) + 1023) & ~uintptr_t(1023));
  float* sm_o = reinterpret_cast<float*>(smem + L::kOOff);
  float2* sm_ml = reinterpret_cast<float2*>(smem + L::kMlOff);
  float4* sm_meta = reinterpret_cast<float4*>(smem + L::kMetaOff);
  int* sm_prefix = reinterpret_cast<int*>(smem + L::kPrefixOff);         // tiles (of one head) of the sequences before
  int* sm_len = reinterpret_cast<int*>(smem + L::kLenOff);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBarOff);
  uint64_t* empty = full + NST;
  int* sm_sum = reinterpret_cast<int*>(empty + NST);                     // [16] sums of the scan's warps
  // The tile that a stage was last given to.  Neighbouring uses of a stage belong to different warps, on both sides, and a barrier's parity
  // tells only neighbouring phases apart; so whoever waits for a stage's barrier first waits until the tile before (producers) or the tile
  // itself (consumers) has been issued: the barrier is then in the phase that is waited for, or just past it.
  volatile int* sm_tile = sm_sum + 16;                                   // [NST]
  volatile uint32_t* abort_flag = reinterpret_cast<uint32_t*>(sm_sum + 16 + NST);
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); sm_tile[i] = i - NST; }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&p.map_k);
    tma_prefetch_desc(&p.map_v);
  }
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();

  // lengths, and the prefix sums of their tiles: 4 sequences a thread of warps 0..7
  {
    int t[4], sum = 0;
    if (threadIdx.x < 256) {
      const long long most = static_cast<long long>(p.max_blocks) << p.c.bs_log2;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = threadIdx.x * 4 + i;
        int n = s < p.n_seqs ? max(__ldg(p.seq_lens + s), 0) : 0;
        if (n > most) {
          n = static_cast<int>(most);
          if (blockIdx.x == 0) raise_status(p.status, DEV_ERR_CACHE_RANGE);
        }
        if (s < p.n_seqs) sm_len[s] = n;
        t[i] = sum;
        sum += (n + TILE - 1) / TILE;
      }
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 31) sm_sum[warp] = incl;
    __syncthreads();
    if (threadIdx.x < 256) {
      int base = incl - sum;
      for (int w = 0; w < warp; ++w) base += sm_sum[w];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = threadIdx.x * 4 + i;
        if (s <= p.n_seqs) sm_prefix[s] = base + t[i];
        if (s <= p.n_seqs && blockIdx.x == 0) p.head_ws[s] = base + t[i];
      }
      if (threadIdx.x == 255 && p.n_seqs == kCacheMaxSeqs) {
        sm_prefix[kCacheMaxSeqs] = base + sum;
        if (blockIdx.x == 0) p.head_ws[kCacheMaxSeqs] = base + sum;
      }
    }
    __syncthreads();
  }
  const int R = p.c.n_kv * p.row_blocks;                         // rows of tiles a sequence has
  const int total = sm_prefix[p.n_seqs] * R;
  const int quota = max(p.min_tiles, (total + p.n_pieces - 1) / p.n_pieces);
  if (blockIdx.x == 0 && threadIdx.x == 0) p.head_ws[p.n_seqs + 1] = quota;
  // the sequence of tile `pos` of the line: the last one whose first tile is not behind it (sequences without tiles are passed over)
  auto find = [&](int pos) {
    int lo = 0, hi = p.n_seqs - 1;
    const int x = pos / R;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sm_prefix[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
  };

  if (warp >= WARPS) {
    // ------------------------------------------------------------------ producers: each takes every fourth step
    setmaxnreg_dec<L::kRegsProducer>();
    const int me = warp - WARPS;
    const int box_log2 = min(p.c.bs_log2, TILE == 32 ? 5 : 6), boxes = TILE >> box_log2;
    uint32_t g = 0;
    bool ok = true;
    for (long long piece = blockIdx.x; ok && piece * quota < total; piece += gridDim.x) {
      const int first = static_cast<int>(piece) * quota, end = min(first + quota, total);
      for (int pos = first + me * kCacheStep; pos < end; pos += kCacheProducers * kCacheStep) {
        const uint32_t it = g + static_cast<uint32_t>(pos - first + lane);
        if (lane < kCacheStep && pos + lane < end) {
          const int at = pos + lane, s = find(at);
          const int n_tiles = sm_prefix[s + 1] - sm_prefix[s], in_seq = at - sm_prefix[s] * R;
          const int row = in_seq / n_tiles, tok = (in_seq - row * n_tiles) * TILE;
          const int kvh = row / p.row_blocks, left = min(sm_len[s] - tok, TILE);
          const int32_t* ids = p.table + s * p.ld_table;
          int id[MT];
          bool good = true;
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            id[b] = -1;
            if (b < boxes && (b << box_log2) < left) {
              id[b] = __ldg(ids + ((tok + (b << box_log2)) >> p.c.bs_log2));
              good = good && id[b] >= 0 && id[b] < p.c.n_blocks;
            }
          }
          if (!good) raise_status(p.status, DEV_ERR_CACHE_RANGE);
          const int st = it % NST;
          if (!word_wait(&sm_tile[st], static_cast<int>(it) - NST, abort_flag) || !mbar_wait(&empty[st], ((it / NST) & 1u) ^ 1u, abort_flag)) {
            ok = false;
          } else {
            uint8_t* kd = smem + st * 8192;
            uint32_t bytes = 0;
#pragma unroll
            for (int b = 0; b < MT; ++b) {
              if (b < boxes && id[b] >= 0 && id[b] < p.c.n_blocks) {
                const int y = ((id[b] * p.c.n_kv + kvh) << p.c.bs_log2) + ((tok + (b << box_log2)) & ((1 << p.c.bs_log2) - 1));
                tma_load_2d(kd + (b << box_log2) * HD, &p.map_k, &full[st], 0, y);
                tma_load_2d(kd + 4096 + (b << box_log2) * HD, &p.map_v, &full[st], 0, y);
                bytes += 2u * (HD << box_log2);
              }
            }
            // scales of the 16-token tiles, while the bytes are on their way (the phase cannot complete before the arrival below)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const int b = (m * 16) >> box_log2;
              int blk = -1;
#pragma unroll
              for (int i = 0; i < MT; ++i) blk = i == b ? id[i] : blk;
              float4 meta = make_float4(0.f, 0.f, 0.f, 0.f);
              if (blk >= 0 && blk < p.c.n_blocks) {
                const long long sc = static_cast<long long>(blk) * p.c.n_kv + kvh;
                meta.x = __ldg(p.c.k_scale + sc);
                float v = __ldg(p.c.v_scale + sc);
                v = v < kCacheMinScale ? kCacheMinScale : v;      // (a NaN stays)
                meta.y = fast_lg2(v);
                meta.z = fast_ex2(-meta.y);
                meta.w = static_cast<float>(min(max(left - m * 16, 0), 16));
              }
              sm_meta[st * MT + m] = meta;
            }
            sm_tile[st] = static_cast<int>(it);
            mbar_expect_tx(&full[st], bytes);
          }
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
      }
      g += static_cast<uint32_t>(end - first);
    }
    if (!ok) {
      const long long t0 = clock64();
      while (clock64() - t0 < 4000000) {}     // let loads in flight land before the CTA retires
    }
  } else {
    // ------------------------------------------------------------------ consumers
    setmaxnreg_inc<L::kRegsConsumer>();
    const int qg = lane >> 2, qt = lane & 3;
    uint32_t g = 0;                                    // tiles of this CTA so far: tile g lies in stage g % NST
    for (long long piece = blockIdx.x; piece * quota < total; piece += gridDim.x) {
      const int first = static_cast<int>(piece) * quota, end = min(first + quota, total);
      for (int pos = first; pos < end;) {
        const int s = find(pos);
        const int n_tiles = sm_prefix[s + 1] - sm_prefix[s], in_seq = pos - sm_prefix[s] * R;
        const int row = in_seq / n_tiles, tile0 = in_seq - row * n_tiles, n = min(n_tiles - tile0, end - pos);
        const int kvh = row / p.row_blocks, head0 = (row - kvh * p.row_blocks) * ROWS;      // first query head, within the group
        const int n_rows = min(ROWS, p.group - head0);
        // this warp's first tile: they go round from the piece's first, so that a sum's order does not depend on what the CTA did before
        const uint32_t k0 = static_cast<uint32_t>(warp + WARPS - (pos - first) % WARPS) % WARPS;
        float m_ref[NT][2], l[NT][2], o[HD / 16][NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          m_ref[j][0] = m_ref[j][1] = -INFINITY;
          l[j][0] = l[j][1] = 0.f;
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.f;
        }
        if (k0 < static_cast<uint32_t>(n)) {
          // queries: column qg of 8, the dims that pair with this lane's bytes of a key row (see the products below)
          uint32_t qf[HD / 16][NT][2];
          float c_row[NT][2];
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const int h = j * 8 + qg;
            float x[HD / 4];
            const uint16_t* src = p.q + s * p.ld_q + static_cast<long long>(kvh * p.group + head0 + h) * HD + qt * (HD / 4);
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
            // the largest of the row to [1, 4): exponent e with 2^e <= mx (126 at most, so that 2^-e is a normal number)
            const int e = mx > 0.f ? min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127, -126), 126) : 0;
            const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
            const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) {
              qf[i][j][0] = Pair16<__half>::pack(x[4 * i] * down, x[4 * i + 2] * down);
              qf[i][j][1] = Pair16<__half>::pack(x[4 * i + 1] * down, x[4 * i + 3] * down);
            }
            const float c = p.scale_log2 * up;                   // of column qg; this lane's scores are columns 2 qt and 2 qt + 1
            c_row[j][0] = __shfl_sync(0xffffffffu, c, 8 * qt);
            c_row[j][1] = __shfl_sync(0xffffffffu, c, 8 * qt + 4);
          }
          for (uint32_t k = k0; k < static_cast<uint32_t>(n); k += WARPS) {
            const uint32_t it = g + k;
            const int st = it % NST;
            if (!__all_sync(0xffffffffu, word_wait(&sm_tile[st], static_cast<int>(it), abort_flag)) ||
                !warp_mbar_wait(&full[st], (it / NST) & 1u, abort_flag)) break;
            const uint32_t kb = smem_u32(smem) + st * 8192, vb = kb + 4096;
            // scores: token rows qg and qg + 8 of each 16, columns 2 qt and 2 qt + 1
            float sc[MT][NT][4];
            float4 meta[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              meta[m] = sm_meta[st * MT + m];
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
            bool higher = false;
            float mx[NT][2];
#pragma unroll
            for (int j = 0; j < NT; ++j) mx[j][0] = mx[j][1] = -INFINITY;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const bool in0 = static_cast<float>(qg) < meta[m].w, in1 = static_cast<float>(qg + 8) < meta[m].w;
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                const float c0 = c_row[j][0] * meta[m].x, c1 = c_row[j][1] * meta[m].x;
                sc[m][j][0] = in0 ? fmaf(sc[m][j][0], c0, meta[m].y) : -INFINITY;
                sc[m][j][1] = in0 ? fmaf(sc[m][j][1], c1, meta[m].y) : -INFINITY;
                sc[m][j][2] = in1 ? fmaf(sc[m][j][2], c0, meta[m].y) : -INFINITY;
                sc[m][j][3] = in1 ? fmaf(sc[m][j][3], c1, meta[m].y) : -INFINITY;
                mx[j][0] = fmax3(mx[j][0], sc[m][j][0], sc[m][j][2]);
                mx[j][1] = fmax3(mx[j][1], sc[m][j][1], sc[m][j][3]);
              }
            }
            // the reference moves only when a score is more than 2^8 above it (the first tile: always)
#pragma unroll
            for (int j = 0; j < NT; ++j) higher = higher || mx[j][0] > m_ref[j][0] + 8.0f || mx[j][1] > m_ref[j][1] + 8.0f;
            if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
              for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  float x = fmaxf(mx[j][b], m_ref[j][b]);
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
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              uint32_t pf[NT][2];
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                const float r0 = m_ref[j][0] == -INFINITY ? 0.f : m_ref[j][0], r1 = m_ref[j][1] == -INFINITY ? 0.f : m_ref[j][1];
                const float w0 = fast_ex2(sc[m][j][0] - r0), w1 = fast_ex2(sc[m][j][1] - r1);
                const float w2 = fast_ex2(sc[m][j][2] - r0), w3 = fast_ex2(sc[m][j][3] - r1);
                l[j][0] = fmaf(w0 + w2, meta[m].z, l[j][0]);
                l[j][1] = fmaf(w1 + w3, meta[m].z, l[j][1]);
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
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);
          }
        }
        // ---------------- the warps' parts of this (sequence, head): put together by all of them, in the order of the warps
        asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");           // the parts of the one before have been read
        float* part = sm_o + warp * ROWS * PITCH;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            float x = l[j][b];
            x += __shfl_xor_sync(0xffffffffu, x, 4);
            x += __shfl_xor_sync(0xffffffffu, x, 8);
            x += __shfl_xor_sync(0xffffffffu, x, 16);
            if (qg == 0) sm_ml[warp * ROWS + j * 8 + 2 * qt + b] = make_float2(m_ref[j][b], x);
          }
          if (k0 < static_cast<uint32_t>(n)) {
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) {                    // dims qg * (HD / 8) + 2 i and + 1, at float i * 16 + qg * 2
              *reinterpret_cast<float2*>(part + (j * 8 + 2 * qt) * PITCH + i * 16 + qg * 2) = make_float2(o[i][j][0], o[i][j][2]);
              *reinterpret_cast<float2*>(part + (j * 8 + 2 * qt + 1) * PITCH + i * 16 + qg * 2) = make_float2(o[i][j][1], o[i][j][3]);
            }
          }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
        constexpr int kQuads = HD / 4, kPass = 32 * WARPS / kQuads;     // 4 dims a thread
        const int d0 = (threadIdx.x % kQuads) * 4, og = d0 / (HD / 8), oi = (d0 % (HD / 8)) / 2;
        const bool whole = n == n_tiles;
        const long long slot = 2 * piece + (pos == first ? 0 : 1);
        for (int r = threadIdx.x / kQuads; r < n_rows; r += kPass) {
          float mr = -INFINITY;
#pragma unroll
          for (int w = 0; w < WARPS; ++w) mr = fmaxf(mr, sm_ml[w * ROWS + r].x);
          float lr = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < WARPS; ++w) {
            const float2 ml = sm_ml[w * ROWS + r];
            if (ml.x == -INFINITY && ml.y == ml.y) continue;       // no token of this warp counts (its O may never have been written)
            const float f = fast_ex2(ml.x - mr);
            const float2 x = *reinterpret_cast<const float2*>(sm_o + (w * ROWS + r) * PITCH + oi * 16 + og * 2);
            const float2 y = *reinterpret_cast<const float2*>(sm_o + (w * ROWS + r) * PITCH + (oi + 1) * 16 + og * 2);
            lr = fmaf(ml.y, f, lr);
            acc[0] = fmaf(x.x, f, acc[0]); acc[1] = fmaf(x.y, f, acc[1]);
            acc[2] = fmaf(y.x, f, acc[2]); acc[3] = fmaf(y.y, f, acc[3]);
          }
          if (whole) {
            const float inv = lr == 0.f ? 0.f : 1.0f / lr;
            uint2 y;
            if (p.fp16) {
              y.x = Pair16<__half>::pack(acc[0] * inv, acc[1] * inv);
              y.y = Pair16<__half>::pack(acc[2] * inv, acc[3] * inv);
            } else {
              y.x = Pair16<bf16>::pack(acc[0] * inv, acc[1] * inv);
              y.y = Pair16<bf16>::pack(acc[2] * inv, acc[3] * inv);
            }
            *reinterpret_cast<uint2*>(p.out + s * p.ld_out + static_cast<long long>(kvh * p.group + head0 + r) * HD + d0) = y;
          } else {
            *reinterpret_cast<float4*>(p.o_ws + (slot * ROWS + r) * HD + d0) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            if (d0 == 0) *reinterpret_cast<float2*>(p.ml_ws + (slot * ROWS + r) * 2) = make_float2(mr, lr);
          }
        }
        g += static_cast<uint32_t>(n);
        pos += n;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) raise_status(p.status, DEV_ERR_WAIT_TIMEOUT);
}

// What the pieces' ends cut, put together: one warp per (sequence, query head), the pieces in order.  Rows that one piece held are
// there already; sequences without tokens get zeros.
template <int HD, int NT>
__global__ void __launch_bounds__(256) cache_join_kernel(const __grid_constant__ CacheAttnParams p) {
  constexpr int ROWS = 8 * NT, N = HD / 32;
  if (p.early_launch) pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, heads = p.c.n_kv * p.group, R = p.c.n_kv * p.row_blocks;
  const int quota = p.head_ws[p.n_seqs + 1];
  for (int u = blockIdx.x * 8 + (threadIdx.x >> 5); u < p.n_seqs * heads; u += gridDim.x * 8) {
    const int s = u / heads, h = u - s * heads, kvh = h / p.group, in_group = h - kvh * p.group;
    const int row = kvh * p.row_blocks + in_group / ROWS, r = in_group % ROWS;
    const int before = p.head_ws[s], n_tiles = p.head_ws[s + 1] - before;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
    if (n_tiles > 0) {
      const int a = before * R + row * n_tiles, w0 = a / quota, w1 = (a + n_tiles - 1) / quota;
      if (w0 == w1) continue;
      auto slot = [&](int w) { return (2LL * w + (w == w0 && a > w * quota ? 1 : 0)) * ROWS + r; };
      float m = -INFINITY, l = 0.f;
      for (int w = w0 + lane; w <= w1; w += 32) m = fmaxf(m, p.ml_ws[slot(w) * 2]);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
#pragma unroll 4
      for (int w = w0; w <= w1; ++w) {
        const float2 ml = *reinterpret_cast<const float2*>(p.ml_ws + slot(w) * 2);
        const float f = ml.x == -INFINITY && ml.y == ml.y ? 0.f : fast_ex2(ml.x - m);
        l = fmaf(ml.y, f, l);
        const float* o = p.o_ws + slot(w) * HD + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = fmaf(o[i], f, acc[i]);
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] *= inv;
    }
    uint16_t* dst = p.out + s * p.ld_out + static_cast<long long>(h) * HD + lane * N;
#pragma unroll
    for (int i = 0; i < N; i += 2)
      *reinterpret_cast<uint32_t*>(dst + i) = p.fp16 ? Pair16<__half>::pack(acc[i], acc[i + 1]) : Pair16<bf16>::pack(acc[i], acc[i + 1]);
  }
}

}  // namespace eas
