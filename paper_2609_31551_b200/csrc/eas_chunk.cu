// C ABI of the attention of several new tokens a sequence over the cache (include/eas_language.h): checks and launches.
#include <algorithm>
#include <cmath>

#include "attention_cache.cuh"
#include "attention_chunk.cuh"
#include "cache_handle.cuh"

using namespace eas;

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// scratch of a launch: two parts a piece of the line, two tiles each
static size_t chunk_workspace(const eas_cache* c, int32_t max_new, int32_t n_heads, int* ws_rows, size_t* ml_off, size_t* cut_off) {
  const int group = n_heads / c->d.n_kv_heads;
  *ws_rows = std::min(128 / group, std::max(max_new, 1)) * group;
  const size_t rows = static_cast<size_t>(4) * c->sm_count * *ws_rows;
  *ml_off = up256(rows * c->d.head_dim * 4);
  *cut_off = *ml_off + up256(rows * 8);
  return *cut_off + up256(c->sm_count * sizeof(ChunkItem));
}

template <int HD, typename T>
static eas_status launch_chunk(const ChunkParams& p, int budget, bool all, cudaStream_t stream) {
  using L = ChunkCfg<HD>;
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(chunk_attention_kernel<HD, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes));
    CUDA_TRY(cudaFuncSetAttribute(chunk_join_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  EAS_TRY(launch_kernel(chunk_attention_kernel<HD, T>, std::min(budget, p.n_ctas), L::kThreads, L::kBytes, stream, p));
  return launch_kernel(chunk_join_kernel<HD>, std::min(budget, p.n_ctas), 512, all ? 0 : kOnePerSmSmem, stream, p);
}

// ------------------------------------------------------------------------------------ few rows
// Up to so many query rows a key/value head (new tokens times heads of the group) a sequence goes to the kernels of single tokens, which read the cache once for
// every 16 of them, rather than to the tiles of 128 rows.  In us, these kernels and the tiles, back to back, 8 key/value heads of 128: 48 sequences of 4096 tokens
// with 8 rows 77 and 135, with 16 rows 96 and 136; of 32 rows, 64 sequences of 500 57 and 65, 4 of 4096 25 and 27, one of 700 12.3 and 14.8; 48 of 2048 (16 heads
// of 64) 125 and 144.
constexpr int kFewRows = 32;
// But with more than 16 rows and heads of 128 the second reading is dear where the cache does not fit L2 (126 MB): 32 rows of 48 sequences of 4096 tokens take
// 180 and 136, of 2 of 65536 112 and 86, of 16 of 4096 68 and 59.  How long the sequences are is known on the device alone; the width of the table stands for
// it, so a table far wider than its sequences may cost the 8 us of the 64 sequences above, and sequences' last bits may depend on it.
// And most of them must have more than 16 rows.  48 sequences of 4096 with up to 8 tokens of 4 heads, by their rows on average: 7.5 102 and 112, 11 112 and
// 122, 17 115 and 136, 18 (half with 32 rows, half with 4) 134 and 136, 22 to 24 (half with 32, half with 12 or 16) 137 and 138, 25 157 and 137, 28 157 and
// 137; 20, if all have 20, 173 and 135.
constexpr int64_t kFewBytes = 128 << 20;
constexpr int kFewAverage = 20;

static int few_columns(int rows) { return rows <= 8 ? 8 : 16; }
static int64_t few_blocks(int rows) { return (rows + few_columns(rows) - 1) / few_columns(rows); }
static size_t few_workspace(const eas_cache* c, int rows, size_t* o_off) {
  const int r = few_columns(rows), warps = r == 8 ? CacheAttnCfg<128, 1>::kWarps : CacheAttnCfg<128, 2>::kWarps;
  const size_t n = static_cast<size_t>(2) * c->sm_count * warps * r;
  *o_off = up256(n * 8);
  return *o_off + up256(n * c->d.head_dim * 4);
}
template <int HD, int NT>
static eas_status launch_few(const CacheAttnParams& p, int budget, bool all, cudaStream_t stream) {
  using L = CacheAttnCfg<HD, NT>;
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(cache_attention_kernel<HD, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes));
    CUDA_TRY(cudaFuncSetAttribute(cache_join_kernel<HD, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  EAS_TRY(launch_kernel(cache_attention_kernel<HD, NT, true>, std::min(budget, p.n_ctas), L::kThreads, L::kBytes, stream, p));
  const int64_t heads = static_cast<int64_t>(p.n_rows) * p.c.n_kv * p.group;
  constexpr int kJoinWarps = kCacheJoinThreads / 32;
  return launch_kernel(cache_join_kernel<HD, NT, true>, static_cast<int>(std::min<int64_t>(budget, (heads + kJoinWarps - 1) / kJoinWarps)), kCacheJoinThreads,
                       all ? 0 : kOnePerSmSmem, stream, p);
}

// Which kernels a call needs: those for few rows alone, where no sequence has more; both, where most sequences have less than half of the most (a
// prompt's chunk beside single tokens); else the tiles of 128 rows for all.
// A chunk beside which there is at most a token a sequence, as far as max_new and n_rows tell, has the others' rows in 8 columns: 512 tokens and 63 single ones
// behind 4096, 32 and 8 heads of 128, 176 us instead of 188.  (With a few drafts among them it has not: 1187 tokens, 19 single ones and drafts of 2, 3 and 4
// would take 174 instead of 170, the last two by tiles.) A max_new of n_rows or more, the default of the binding, tells nothing of how the rows are spread;
// their average does.  With it, 64 single tokens behind 4096 take 103 us (124 in 16 columns), 48 drafts of 4 104 (143 by tiles), of 8 147 (189 in 16 columns).
// The kernels for few rows add up what all sequences may cost in 32 bits; behind a table so wide that the sum could pass them (8 sequences of 8 key/value heads
// and 2^30 places each), the tiles, whose line has 64, take all.
struct ChunkPlan {
  int few_rows = 0;            // most rows a key/value head of the sequences that the kernels for few rows take
  bool tiles = false;
};
static ChunkPlan chunk_plan(const eas_cache* c, int32_t n_seqs, int32_t n_rows, int32_t max_new, int group, int64_t places) {
  ChunkPlan plan;
  const int64_t most = static_cast<int64_t>(max_new) * group, token_bytes = 2LL * c->d.n_kv_heads * c->d.head_dim;
  const bool twice_dear = c->d.head_dim == 128 && static_cast<int64_t>(n_rows) * group >= static_cast<int64_t>(n_seqs) * kFewAverage &&
                          n_seqs * places >= kFewBytes / token_bytes;
  plan.tiles = most > kFewRows || (most > 16 && twice_dear);
  if (!plan.tiles) {
    plan.few_rows = static_cast<int>(std::max<int64_t>(most, 1));
  } else if (group <= kFewRows && static_cast<int64_t>(n_rows) * 2 < static_cast<int64_t>(n_seqs) * max_new) {
    const bool known = max_new < n_rows;
    const bool single = known ? n_rows - max_new <= n_seqs - 1 : n_rows <= n_seqs;
    plan.few_rows = group <= 8 && single ? 8 : !known && twice_dear ? 16 : kFewRows;
  }
  if (plan.few_rows > 0) {
    const int64_t tiles = (places + 31) / 32 + kRowCost;           // (no variant's tile is smaller)
    const int64_t row_tiles = few_blocks(plan.few_rows) * c->d.n_kv_heads;
    if (tiles * row_tiles > 0x7fffffffLL / std::clamp(n_seqs, 1, kCacheMaxSeqs)) return ChunkPlan{0, true};
  }
  return plan;
}

// The kernels of a call run one behind the other: they share the scratch.
static size_t plan_workspace(const eas_cache* c, const ChunkPlan& plan, int32_t n_rows, int32_t max_new, int32_t n_heads) {
  int ws_rows = 0;
  size_t a = 0, b = 0, bytes = 256;
  if (plan.few_rows > 0) bytes = std::max(bytes, few_workspace(c, plan.few_rows, &a));
  if (plan.tiles) bytes = std::max(bytes, chunk_workspace(c, std::min(max_new, n_rows), n_heads, &ws_rows, &a, &b));
  return bytes;
}

static eas_status chunk_attention(const eas_cache* c, const eas_cache_seqs* s, const void* q, int64_t ld_q, void* out, int64_t ld_out, int32_t n_rows,
                                  int32_t max_new, int32_t n_heads, int32_t dtype, float scale, void* workspace, size_t workspace_bytes, int32_t sm_budget,
                                  void* stream, uint32_t* status_dev) {
  int budget = 0;
  EAS_TRY(check_cache_call(c, s, false, dtype, status_dev, sm_budget, &budget));
  const int G = c->d.n_kv_heads, hd = c->d.head_dim;
  if (s->n_seqs > 0 && s->cu_seqlens == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (n_heads <= 0 || n_heads % G != 0) return fail(EAS_ERR_INVALID_ARG, "%d query heads for %d key/value heads", n_heads, G);
  if (n_rows < 0 || max_new < 0) return fail(EAS_ERR_INVALID_ARG, "n_rows %d, max_new %d", n_rows, max_new);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(EAS_ERR_INVALID_ARG, "scale must be positive and finite");
  const int group = n_heads / G;
  if (group > 128) return fail(EAS_ERR_UNSUPPORTED, "%d query heads per key/value head (at most 128)", group);
  if (s->n_seqs == 0 || n_rows == 0) return EAS_OK;
  if (q == nullptr || out == nullptr || workspace == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (!aligned16(q) || !aligned16(out)) return fail(EAS_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  const int64_t w = static_cast<int64_t>(n_heads) * hd;
  if (ld_q < w || ld_out < w || ld_q % 8 != 0 || ld_out % 8 != 0)
    return fail(EAS_ERR_INVALID_ARG, "token distances must be multiples of 8 that hold a token's heads");
  const int64_t places = static_cast<int64_t>(s->max_blocks) * c->d.block_size;
  if (places > (1LL << 30)) return fail(EAS_ERR_UNSUPPORTED, "max_blocks %d: more than 2^30 places a sequence", s->max_blocks);
  const ChunkPlan plan = chunk_plan(c, s->n_seqs, n_rows, max_new, group, places);
  const size_t need = plan_workspace(c, plan, n_rows, max_new, n_heads);
  if (workspace_bytes < need) return fail(EAS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return fail(EAS_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  if (static_cast<int64_t>(n_rows) * n_heads > 0x7fffffffLL) return fail(EAS_ERR_UNSUPPORTED, "too many rows for one call");
  const bool all = budget == c->sm_count;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  if (plan.few_rows > 0) {
    const int columns = few_columns(plan.few_rows);
    CacheAttnParams p{};
    p.map_k = c->map_k; p.map_v = c->map_v;
    p.c = view_of(c);
    p.group = group;
    p.row_blocks = static_cast<int>(few_blocks(plan.few_rows));
    p.n_rows = n_rows; p.max_new = max_new; p.most_rows = plan.few_rows;
    p.ld_table = s->ld_table; p.max_blocks = s->max_blocks;
    p.q = static_cast<const uint16_t*>(q); p.out = static_cast<uint16_t*>(out);
    p.ld_q = ld_q; p.ld_out = ld_out; p.fp16 = dtype == EAS_DTYPE_FP16;
    p.n_ctas = c->sm_count;
    p.scale_log2 = static_cast<float>(scale * kLog2e);
    size_t o_off = 0;
    few_workspace(c, plan.few_rows, &o_off);
    p.ml_ws = reinterpret_cast<float*>(ws); p.o_ws = reinterpret_cast<float*>(ws + o_off);
    p.status = status_dev;
    for (int first = 0; first < s->n_seqs; first += kCacheMaxSeqs) {
      p.n_seqs = std::min(kCacheMaxSeqs, s->n_seqs - first);
      p.table = s->block_table + first * s->ld_table;
      p.cu = s->cu_seqlens + first;
      p.seq_lens = s->seq_lens + first;
      EAS_TRY(hd == 64 ? (columns == 8 ? launch_few<64, 1>(p, budget, all, st) : launch_few<64, 2>(p, budget, all, st))
                       : (columns == 8 ? launch_few<128, 1>(p, budget, all, st) : launch_few<128, 2>(p, budget, all, st)));
    }
  }
  if (!plan.tiles) return EAS_OK;
  if (c->sm_count > kChunkMaxPieces) return fail(EAS_ERR_ARCH, "%d SMs (at most %d)", c->sm_count, kChunkMaxPieces);
  ChunkParams p{};
  size_t ml_off = 0, cut_off = 0;
  chunk_workspace(c, std::min(max_new, n_rows), n_heads, &p.ws_rows, &ml_off, &cut_off);
  p.c = view_of(c);
  p.ld_table = s->ld_table; p.max_blocks = s->max_blocks; p.n_rows = n_rows; p.max_new = max_new; p.few_rows = plan.few_rows;
  p.q = static_cast<const uint16_t*>(q); p.out = static_cast<uint16_t*>(out);
  p.ld_q = ld_q; p.ld_out = ld_out; p.fp16 = dtype == EAS_DTYPE_FP16; p.group = group; p.tile_tokens = 128 / group;
  p.by_group = group == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + group - 1) / group);
  p.n_ctas = c->sm_count;
  p.scale_log2 = static_cast<float>(scale * kLog2e);
  p.o_ws = reinterpret_cast<float4*>(ws);
  p.ml_ws = reinterpret_cast<float2*>(ws + ml_off);
  p.cut_ws = reinterpret_cast<ChunkItem*>(ws + cut_off);
  p.status = status_dev;
  for (int first = 0; first < s->n_seqs; first += kChunkMaxSeqs) {
    p.n_seqs = std::min(kChunkMaxSeqs, s->n_seqs - first);
    p.table = s->block_table + first * s->ld_table;
    p.cu = s->cu_seqlens + first;
    p.seq_lens = s->seq_lens + first;
    EAS_TRY(hd == 64 ? (p.fp16 ? launch_chunk<64, __half>(p, budget, all, st) : launch_chunk<64, bf16>(p, budget, all, st))
                     : (p.fp16 ? launch_chunk<128, __half>(p, budget, all, st) : launch_chunk<128, bf16>(p, budget, all, st)));
  }
  return EAS_OK;
}

extern "C" size_t eas_cache_chunk_workspace_bytes(const eas_cache* cache, int32_t n_seqs, int32_t n_rows, int32_t max_new, int32_t n_heads) {
  if (cache == nullptr || n_seqs < 0 || n_rows < 0 || max_new < 0 || n_heads <= 0 || n_heads % cache->d.n_kv_heads != 0) {
    fail(EAS_ERR_INVALID_ARG, "bad arguments");
    return 0;
  }
  if (n_heads / cache->d.n_kv_heads > 128) {
    fail(EAS_ERR_UNSUPPORTED, "%d query heads per key/value head (at most 128)", n_heads / cache->d.n_kv_heads);
    return 0;
  }
  // for a table of any width: a wider one brings the tiles in, or has them take all
  size_t bytes = 0;
  for (const int64_t places : {int64_t{0}, int64_t{1} << 30})
    bytes = std::max(bytes, plan_workspace(cache, chunk_plan(cache, n_seqs, n_rows, max_new, n_heads / cache->d.n_kv_heads, places), n_rows, max_new, n_heads));
  return bytes;
}

extern "C" eas_status eas_cache_chunk_attention(const eas_cache* cache, const eas_cache_seqs* seqs, const void* q, int64_t ld_q, void* out, int64_t ld_out,
                                                int32_t n_rows, int32_t max_new, int32_t n_heads, int32_t dtype, float scale, void* workspace,
                                                size_t workspace_bytes, int32_t sm_budget, void* stream, uint32_t* status_dev) {
  return chunk_attention(cache, seqs, q, ld_q, out, ld_out, n_rows, max_new, n_heads, dtype, scale, workspace, workspace_bytes, sm_budget, stream, status_dev);
}
