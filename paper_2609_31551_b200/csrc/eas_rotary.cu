// C ABI of rotary positions and of appending to the cache (include/eas_language.h): checks and launches.
#include <algorithm>
#include <cmath>
#include <new>

#include "cache_handle.cuh"
#include "rotary.cuh"

using namespace eas;

struct eas_rotary {
  RotaryTable t{};
  int head_dim = 0, n_axes = 0;
};

static eas_status rotary_create(const eas_rotary_desc* d, eas_rotary** out) {
  if (out == nullptr) return fail(EAS_ERR_INVALID_ARG, "out is null");
  *out = nullptr;
  if (d == nullptr || d->inv_freq == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(EAS_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
  if (d->rotary_dim <= 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 16 != 0)
    return fail(EAS_ERR_UNSUPPORTED, "rotary_dim %d (supported: multiples of 16 up to head_dim)", d->rotary_dim);
  if (d->pairing != EAS_ROTARY_HALVES && d->pairing != EAS_ROTARY_NEIGHBOURS) return fail(EAS_ERR_INVALID_ARG, "pairing %d", d->pairing);
  if (d->n_axes < 1 || d->n_axes > kRotaryMaxAxes) return fail(EAS_ERR_UNSUPPORTED, "%d axes (supported: 1 to %d)", d->n_axes, kRotaryMaxAxes);
  if (!(d->scale > 0.0f) || !std::isfinite(d->scale)) return fail(EAS_ERR_INVALID_ARG, "scale must be positive and finite");
  eas_rotary r;
  r.head_dim = d->head_dim;
  r.n_axes = d->n_axes;
  r.t.pairs = d->rotary_dim / 2;
  r.t.neighbours = d->pairing == EAS_ROTARY_NEIGHBOURS;
  r.t.scale = d->scale;
  for (int i = 0; i < r.t.pairs; ++i) {
    if (!std::isfinite(d->inv_freq[i])) return fail(EAS_ERR_INVALID_ARG, "inv_freq[%d] is not finite", i);
    const int axis = d->axis == nullptr ? 0 : d->axis[i];
    if (axis < 0 || axis >= d->n_axes) return fail(EAS_ERR_INVALID_ARG, "axis[%d] = %d outside 0..%d", i, axis, d->n_axes - 1);
    constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;
    long double turns = static_cast<long double>(d->inv_freq[i]) / kTwoPi;
    turns = std::nearbyint((turns - std::floor(turns)) * 18446744073709551616.0L);               // 0 .. 2^64
    const uint64_t f = turns >= 18446744073709551616.0L ? 0 : static_cast<uint64_t>(turns);
    r.t.f_lo[i] = static_cast<uint32_t>(f);
    r.t.f_hi[i] = static_cast<uint32_t>(f >> 32);
    r.t.axis[i] = static_cast<uint8_t>(axis);
  }
  *out = new (std::nothrow) eas_rotary(r);
  return *out != nullptr ? EAS_OK : fail(EAS_ERR_INVALID_ARG, "out of host memory");
}

// one side (queries or keys) of a call with rows
static eas_status check_rows(const char* name, const void* in, const void* out, int64_t ld_in, int64_t ld_out, int64_t width) {
  if (in == nullptr || out == nullptr) return fail(EAS_ERR_INVALID_ARG, "%s: a required pointer is null", name);
  if (!aligned16(in) || !aligned16(out)) return fail(EAS_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  if (ld_in < width || ld_out < width || ld_in % 8 != 0 || ld_out % 8 != 0)
    return fail(EAS_ERR_INVALID_ARG, "%s: token distances must be multiples of 8 that hold a token's heads", name);
  return EAS_OK;
}
// The axes lie n_rows apart or more, or are one and the same (kernels only read them)
static eas_status check_positions(const eas_rotary* r, const eas_rotary_inputs* in) {
  if (in->positions == nullptr || (in->ld_positions != 0 && in->ld_positions < in->n_rows))
    return fail(EAS_ERR_INVALID_ARG, "positions: [%d][%d] wanted", r->n_axes, in->n_rows);
  return EAS_OK;
}
static eas_status check_inputs(const eas_rotary* r, const eas_rotary_inputs* in) {
  if (r == nullptr || in == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (in->dtype != EAS_DTYPE_BF16 && in->dtype != EAS_DTYPE_FP16) return fail(EAS_ERR_UNSUPPORTED, "dtype %d", in->dtype);
  if (in->n_rows < 0 || in->n_heads < 0 || in->n_kv_heads < 0 || in->n_heads > 65536 || in->n_kv_heads > 65536)
    return fail(EAS_ERR_INVALID_ARG, "%d rows of %d and %d heads", in->n_rows, in->n_heads, in->n_kv_heads);
  if (in->inverse != 0 && in->inverse != 1) return fail(EAS_ERR_INVALID_ARG, "inverse %d", in->inverse);
  return EAS_OK;
}
static RotaryRows rows_of(const eas_rotary_inputs* in) {
  RotaryRows r{};
  r.q = in->q; r.k = in->k; r.out_q = in->out_q; r.out_k = in->out_k;
  r.ld_q = in->ld_q; r.ld_k = in->ld_k; r.ld_out_q = in->ld_out_q; r.ld_out_k = in->ld_out_k;
  r.positions = in->positions; r.ld_positions = in->ld_positions;
  r.n_rows = in->n_rows; r.n_heads = in->n_heads; r.n_kv = in->n_kv_heads; r.inverse = in->inverse;
  return r;
}

// A token's heads go to one warp, whose 64 cosines serve them all, unless that leaves warps of the device without work: then to as many as there are batches of
// loads (a warp takes `batch` heads at once).
static void split_heads(int rows, int heads, int batch, int64_t warps, uint32_t* parts, int* part_heads) {
  int n = 1;
  const int most = (heads + batch - 1) / batch;
  while (n < most && static_cast<int64_t>(rows) * n < warps) ++n;
  if (static_cast<int64_t>(rows) * n > 0x7fffffff) n = 1;
  *part_heads = (heads + n - 1) / n;
  *parts = static_cast<uint32_t>((heads + *part_heads - 1) / *part_heads);
}

template <int HD, typename T>
static eas_status launch_rotary(RotaryParams& p, int budget, bool all, cudaStream_t stream) {
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(rotary_kernel<HD, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  constexpr int kWarps = kRotaryThreads / 32;
  const int64_t units = static_cast<int64_t>(p.r.n_rows) * p.parts;
  int warps = kWarps;                                              // few units: fewer warps a CTA, so that every SM has some
  while (warps > 1 && static_cast<int64_t>(warps / 2) * budget >= units) warps /= 2;
  return launch_kernel(rotary_kernel<HD, T>, static_cast<int>(std::min<int64_t>(budget, (units + warps - 1) / warps)), warps * 32, all ? 0 : kOnePerSmSmem, stream, p);
}

static eas_status rotary_apply(const eas_rotary* rotary, const eas_rotary_inputs* in, int32_t sm_budget, void* stream) {
  EAS_TRY(check_inputs(rotary, in));
  const int hd = rotary->head_dim;
  if (in->n_rows > 0) {
    if (in->n_heads > 0) EAS_TRY(check_rows("q", in->q, in->out_q, in->ld_q, in->ld_out_q, static_cast<int64_t>(in->n_heads) * hd));
    if (in->n_kv_heads > 0) EAS_TRY(check_rows("k", in->k, in->out_k, in->ld_k, in->ld_out_k, static_cast<int64_t>(in->n_kv_heads) * hd));
    EAS_TRY(check_positions(rotary, in));
  }
  int budget = 0;
  EAS_TRY(resolve_budget(sm_budget, &budget));
  const int heads = in->n_heads + in->n_kv_heads;
  if (in->n_rows == 0 || heads == 0) return EAS_OK;
  RotaryParams p{};
  p.t = rotary->t;
  p.r = rows_of(in);
  p.r.in_place = (in->n_heads == 0 || (in->q == in->out_q && in->ld_q == in->ld_out_q)) && (in->n_kv_heads == 0 || (in->k == in->out_k && in->ld_k == in->ld_out_k));
  const bool all = budget == g_device_sms, h = in->dtype == EAS_DTYPE_FP16;
  split_heads(in->n_rows, heads, kRotaryBatch * 32 / (hd / 16), static_cast<int64_t>(g_device_sms) * (kRotaryThreads / 32), &p.parts, &p.part_heads);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (hd == 64) return h ? launch_rotary<64, __half>(p, budget, all, st) : launch_rotary<64, bf16>(p, budget, all, st);
  return h ? launch_rotary<128, __half>(p, budget, all, st) : launch_rotary<128, bf16>(p, budget, all, st);
}

template <int HD, int GT, typename T>
static eas_status launch_append(AppendParams& p, int budget, bool all, cudaStream_t stream) {
  const int table = std::max((p.t.pairs * 8) << p.c.bs_log2, kAppendThreads / 32 * kRotaryMaxPairs * 8);
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(cache_append_kernel<HD, GT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  // Key/value heads of an item: all of a block's, whose cosines then are worked out once, unless that leaves CTAs without work; at the least one pass of a CTA.
  constexpr int kLeast = kAppendThreads / GT > 1 ? kAppendThreads / GT / 2 : 1;
  const int64_t ctas = static_cast<int64_t>(kAppendCtas) * g_device_sms;
  const int64_t blocks = std::max<int64_t>(p.pairs - p.s.n_seqs, 1);      // (about half of the sequences' spare numbers have a block)
  p.part_heads = p.c.n_kv;
  while (p.part_heads > kLeast && blocks * ((p.c.n_kv + p.part_heads - 1) / p.part_heads) < ctas) p.part_heads = (p.part_heads + 1) / 2;
  p.head_parts = (p.c.n_kv + p.part_heads - 1) / p.part_heads;
  if (static_cast<int64_t>(p.pairs) * p.head_parts > 0x3fffffff) return fail(EAS_ERR_UNSUPPORTED, "too many rows for one call");
  split_heads(p.r.n_rows, std::max(p.r.n_heads, 1), kAppendBatch * 32 / (HD / 16), ctas * (kAppendThreads / 32), &p.q_parts, &p.q_part_heads);
  const int64_t items = static_cast<int64_t>(p.pairs) * p.head_parts + (static_cast<int64_t>(p.r.n_heads > 0 ? p.r.n_rows : 0) * p.q_parts + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
  return launch_kernel(cache_append_kernel<HD, GT, T>, static_cast<int>(std::min<int64_t>(all ? ctas : budget, items)), kAppendThreads, all ? table : kOnePerSmSmem,
                       stream, p);
}
// threads of a head's keys or values: 32 values each of what a sequence has on average in a block
template <int HD, typename T>
static eas_status launch_append(AppendParams& p, int budget, bool all, cudaStream_t stream) {
  const int64_t rows = std::min<int64_t>((p.r.n_rows + p.s.n_seqs - 1) / p.s.n_seqs, 1 << p.c.bs_log2), values = rows * HD;
  if (values > 4096) return launch_append<HD, 256, T>(p, budget, all, stream);
  if (values > 2048) return launch_append<HD, 128, T>(p, budget, all, stream);
  if (values > 1024) return launch_append<HD, 64, T>(p, budget, all, stream);
  return launch_append<HD, 32, T>(p, budget, all, stream);
}

static eas_status cache_append(const eas_cache* c, const eas_cache_seqs* s, const eas_rotary* rotary, const eas_rotary_inputs* in, const void* v, int64_t ld_v,
                               int32_t sm_budget, void* stream, uint32_t* status_dev) {
  EAS_TRY(check_inputs(rotary, in));
  int budget = 0;
  EAS_TRY(check_cache_call(c, s, true, in->dtype, status_dev, sm_budget, &budget));
  const int hd = c->d.head_dim, G = c->d.n_kv_heads;
  if (rotary->head_dim != hd) return fail(EAS_ERR_INVALID_ARG, "heads of %d in the cache, of %d in the rotary positions", hd, rotary->head_dim);
  if (in->n_kv_heads != G) return fail(EAS_ERR_INVALID_ARG, "%d key/value heads for a cache of %d", in->n_kv_heads, G);
  if (in->out_k != nullptr || in->inverse != 0) return fail(EAS_ERR_INVALID_ARG, "the rotated keys go to the cache: out_k is null, inverse 0");
  if (in->n_rows == 0 || s->n_seqs == 0) return EAS_OK;
  if (in->n_heads > 0) EAS_TRY(check_rows("q", in->q, in->out_q, in->ld_q, in->ld_out_q, static_cast<int64_t>(in->n_heads) * hd));
  EAS_TRY(check_rows("k", in->k, in->k, in->ld_k, in->ld_k, static_cast<int64_t>(G) * hd));
  EAS_TRY(check_rows("v", v, v, ld_v, ld_v, static_cast<int64_t>(G) * hd));
  if (in->positions != nullptr) EAS_TRY(check_positions(rotary, in));
  AppendParams p{};
  p.c = view_of(c);
  p.s = CacheSeqs{s->block_table, s->cu_seqlens, s->start, s->ld_table, s->n_seqs, s->max_blocks};
  p.t = rotary->t;
  p.r = rows_of(in);
  p.r.n_kv = 0;
  p.r.in_place = in->q == in->out_q && in->ld_q == in->ld_out_q;
  p.v = v; p.ld_v = ld_v;
  const int64_t pairs = (in->n_rows >> c->bs_log2) + 2LL * s->n_seqs;
  if (pairs > 0x3fffffff) return fail(EAS_ERR_UNSUPPORTED, "too many rows for one call");
  p.pairs = static_cast<int>(pairs);
  while ((1 << p.pairs_log2) < p.t.pairs) ++p.pairs_log2;
  p.status = status_dev;
  const bool all = budget == c->sm_count, h = in->dtype == EAS_DTYPE_FP16;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (hd == 64) return h ? launch_append<64, __half>(p, budget, all, st) : launch_append<64, bf16>(p, budget, all, st);
  return h ? launch_append<128, __half>(p, budget, all, st) : launch_append<128, bf16>(p, budget, all, st);
}

// ------------------------------------------------------------------------------------ entry points (nothing in them throws)
extern "C" eas_status eas_rotary_create(const eas_rotary_desc* desc, eas_rotary** out) { return rotary_create(desc, out); }

extern "C" void eas_rotary_destroy(eas_rotary* rotary) { delete rotary; }

extern "C" eas_status eas_rotary_apply(const eas_rotary* rotary, const eas_rotary_inputs* in, int32_t sm_budget, void* stream) {
  return rotary_apply(rotary, in, sm_budget, stream);
}

extern "C" eas_status eas_cache_append(const eas_cache* cache, const eas_cache_seqs* seqs, const eas_rotary* rotary, const eas_rotary_inputs* in, const void* v,
                                       int64_t ld_v, int32_t sm_budget, void* stream, uint32_t* status_dev) {
  return cache_append(cache, seqs, rotary, in, v, ld_v, sm_budget, stream, status_dev);
}
