// C ABI of the language-model operators (include/eas_language.h): checks, tensor maps, launches.
#include "../../include/eas_language.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "attention_cache.cuh"
#include "attention_prompt.cuh"
#include "cache_handle.cuh"
#include "host.cuh"
#include "kv_cache.cuh"

using namespace eas;


// ------------------------------------------------------------------------------------ prompts
// [tokens, heads * HD] with token distance ld, seen as {HD, heads, tokens}: one box holds a tile's rows, the heads of a token side by side
static eas_status prompt_q_map(CUtensorMap* m, const void* q, int heads, int hd, int64_t tokens, int64_t ld, int group, int tile_tokens) {
  const uint64_t dims[3] = {static_cast<uint64_t>(hd), static_cast<uint64_t>(heads), static_cast<uint64_t>(tokens)};
  const uint64_t strides[2] = {static_cast<uint64_t>(hd) * 2, static_cast<uint64_t>(ld) * 2};
  const uint32_t box[3] = {64, static_cast<uint32_t>(group), static_cast<uint32_t>(tile_tokens)};
  return make_tmap(m, q, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// the same seen as {64, tokens, heads * HD / 64}: one box holds 80 keys of a head, its 64-column halves one behind the other
static eas_status prompt_kv_map(CUtensorMap* m, const void* k, int heads, int hd, int64_t tokens, int64_t ld, int keys) {
  const uint64_t dims[3] = {64, static_cast<uint64_t>(tokens), static_cast<uint64_t>(heads) * hd / 64};
  const uint64_t strides[2] = {static_cast<uint64_t>(ld) * 2, 128};
  const uint32_t box[3] = {64, static_cast<uint32_t>(keys), static_cast<uint32_t>(hd / 64)};
  return make_tmap(m, k, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int HD, bool FP16, typename Params>
static eas_status launch_prompt(const Params& pp, int budget, bool all, cudaStream_t stream) {
  using L = PromptCfg<HD>;
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(prompt_attention_kernel<HD, FP16, Params>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes));
    if constexpr (Params::kSplit) CUDA_TRY(cudaFuncSetAttribute(prompt_join_kernel<HD, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  int grid = pp.total_units;
  if constexpr (Params::kSplit) grid = pp.n_pieces;
  EAS_TRY(launch_kernel(prompt_attention_kernel<HD, FP16, Params>, std::min(budget, grid), L::kThreads, L::kBytes, stream, pp));
  if constexpr (Params::kSplit) {
    const int64_t items = static_cast<int64_t>(pp.n_units) * L::kWg * (HD / 8);      // 4 a CTA
    return launch_kernel(prompt_join_kernel<HD, FP16>, static_cast<int>(std::min<int64_t>(budget, (items + 3) / 4)), 512, all ? 0 : kOnePerSmSmem, stream, pp);
  }
  return EAS_OK;
}
template <typename Params>
static eas_status launch_prompt(const Params& pp, int hd, bool fp16, int budget, bool all, cudaStream_t st) {
  if (hd == 64) return fp16 ? launch_prompt<64, true>(pp, budget, all, st) : launch_prompt<64, false>(pp, budget, all, st);
  return fp16 ? launch_prompt<128, true>(pp, budget, all, st) : launch_prompt<128, false>(pp, budget, all, st);
}

static PromptParamsFew few_of(const PromptParams& pp) {
  PromptParamsFew f;
  static_cast<PromptCommon&>(f) = pp;
  const int n = pp.n_seqs;
  std::copy_n(pp.q0, n, f.q0); std::copy_n(pp.k0, n, f.k0); std::copy_n(pp.len_q, n, f.len_q); std::copy_n(pp.len_k, n, f.len_k);
  std::copy_n(pp.tiles, n, f.tiles); std::copy_n(pp.per_head, n, f.per_head); std::copy_n(pp.unit_prefix, n + 1, f.unit_prefix);
  return f;
}

// How the work of a call is laid out: the sequences in the order in which their units are dealt.
struct PromptPlan {
  std::vector<int> order;        // sequences with queries, longest first (stable): the tail of the static deal is short work
  int wg = 0, tile_tokens = 0;
};
static PromptPlan prompt_plan(const eas_prompt_inputs* in) {
  PromptPlan plan;
  plan.wg = in->head_dim == 64 ? PromptCfg<64>::kWg : PromptCfg<128>::kWg;
  plan.tile_tokens = 128 / (in->n_heads / in->n_kv_heads);
  for (int i = 0; i < in->n_seqs; ++i)
    if (in->cu_q[i + 1] > in->cu_q[i]) plan.order.push_back(i);
  std::stable_sort(plan.order.begin(), plan.order.end(),
                   [&](int a, int b) { return in->cu_k[a + 1] - in->cu_k[a] > in->cu_k[b + 1] - in->cu_k[b]; });
  return plan;
}
// key steps of a unit whose last tile is the sequence's tile number `tiles` (counted from 1)
static int64_t prompt_unit_steps(int64_t len_q, int64_t len_k, int64_t tiles, int tile_tokens) {
  constexpr int keys = PromptCfg<64>::kKeys;
  const int64_t seen = std::min(tiles * tile_tokens, len_q) + len_k - len_q;
  return (std::max<int64_t>(seen, 0) + keys - 1) / keys;
}
// Into how many pieces the line of key steps of sequences order[first .. first + n) is cut (0: it is not, units are dealt whole), and the number of
// items.  Costs in key steps of a unit (1.2 us), fitted to calls of head_dim 128 on both sides: the busiest SM's steps, kUnitSteps a whole unit and
// kItemSteps an item for its beginning and end and its way through L2, kJoinSteps for the joining launch.  Only for calls of at most kSplitUnits units
// an SM with long key ranges, where the deal leaves SMs without work.
constexpr int kSplitUnits = 4, kSplitLeastSteps = 24, kPieceLeastSteps = 8;
constexpr double kUnitSteps = 2.0, kItemSteps = 5.0, kJoinSteps = 6.0;
struct PromptCut {
  int pieces = 0, items = 0, units = 0;
  int64_t steps = 0;
};
static PromptCut prompt_cut(const eas_prompt_inputs* in, const PromptPlan& plan, int first, int n, int sms) {
  PromptCut cut;
  int64_t units = 0, empty = 0, total = 0, most = 0;       // of all units: their number, those without steps, key steps; the costliest
  const int64_t most_units = std::min<int64_t>(static_cast<int64_t>(kSplitUnits) * sms, kPromptSplitUnits);
  for (int j = 0; j < n; ++j) {
    const int i = plan.order[first + j], len_q = in->cu_q[i + 1] - in->cu_q[i], len_k = in->cu_k[i + 1] - in->cu_k[i];
    const int64_t tiles = (static_cast<int64_t>(len_q) + plan.tile_tokens - 1) / plan.tile_tokens, per_head = (tiles + plan.wg - 1) / plan.wg;
    units += per_head * in->n_kv_heads;
    if (units > most_units) return cut;
    for (int64_t t = tiles; t > 0; t -= plan.wg) {
      const int64_t steps = prompt_unit_steps(len_q, len_k, t, plan.tile_tokens);
      most = std::max(most, steps);
      total += steps * in->n_kv_heads;
      empty += steps == 0 ? in->n_kv_heads : 0;
    }
  }
  if (most < kSplitLeastSteps) return cut;
  const int64_t rounds = (units + sms - 1) / sms;          // whole units: the busiest SM has that many of middling cost, or the costliest one
  const double whole = std::max(static_cast<double>(rounds) * total / units, static_cast<double>(most)) + rounds * kUnitSteps;
  const int64_t pieces = std::min<int64_t>({sms, kPromptPieces, total / kPieceLeastSteps}), items = units - empty + pieces - 1;
  const double in_pieces = 1.05 * (static_cast<double>(total) / pieces + ((units + pieces - 1) / pieces + 1) * kItemSteps) + kJoinSteps;
  if (in_pieces >= whole) return cut;
  cut.pieces = static_cast<int>(pieces);
  cut.items = static_cast<int>(items);                     // (at most: a piece may end where a unit does)
  cut.units = static_cast<int>(units);
  cut.steps = total;
  return cut;
}
// The items of a cut launch
static void prompt_items(PromptParamsSplit& pp, const PromptCut& cut, int wg) {
  int unit = 0, item = 0, piece = 0;
  int64_t at = 0;                                          // on the line
  for (int s = 0; s < pp.n_seqs; ++s)
    for (int b = 0; b < pp.per_head[s]; ++b) {
      const int64_t steps = prompt_unit_steps(pp.len_q[s], pp.len_k[s], pp.tiles[s] - static_cast<int64_t>(b) * wg, pp.tile_tokens);
      for (int h = 0; h < pp.n_kv; ++h, ++unit) {
        pp.unit_item[unit] = static_cast<uint16_t>(item);
        for (int64_t lo = 0; lo < steps;) {
          if (at + lo == cut.steps * piece / cut.pieces) pp.piece_item[piece++] = static_cast<uint16_t>(item);
          pp.item_unit[item] = static_cast<uint16_t>(unit);
          pp.item_lo[item++] = static_cast<int>(lo);
          lo = std::min(steps, cut.steps * piece / cut.pieces - at);
        }
        at += steps;
      }
    }
  pp.unit_item[unit] = pp.piece_item[piece] = static_cast<uint16_t>(item);
  pp.n_units = unit;
  pp.n_pieces = piece;
  pp.total_units = item;
}
// The units of a launch by cost, costliest first (a counting sort over their key steps), each to the CTA of `grid` with the least to do so far.  The
// CTAs' loads are small whole numbers, so those with the same load form a list, and the least load only grows.  (Dealt in rounds of alternating
// direction instead, costliest first: 8 prompts of 1 to 1563 tokens of head_dim 128 53 instead of 49 us, 10 of 3 to 1000 29 instead of 25.5.  Of head_dim 64,
// 13 mixes: 1.5 to 25 % more in nine of them, the 8 prompts 42.7 instead of 36.4, one of 1500 beside thirty of 20 33.7 instead of 31.2; 1 % less in four, the 10
// prompts 23.1 instead of 23.4.  The host takes 9 ns a unit for the list, 4 in rounds: 280 units 2.5 us instead of 1.0, which calls that wait for the host pay.)
static void prompt_list(PromptParams& pp, int wg, int grid) {
  std::vector<int> count;
  auto steps = [&](int s, int back) {
    return static_cast<size_t>(prompt_unit_steps(pp.len_q[s], pp.len_k[s], pp.tiles[s] - static_cast<int64_t>(back) * wg, pp.tile_tokens));
  };
  for (int s = 0; s < pp.n_seqs; ++s)
    for (int b = 0; b < pp.per_head[s]; ++b) {
      const size_t c = steps(s, b);
      if (count.size() <= c) count.resize(c + 1, 0);
      count[c] += pp.n_kv;
    }
  const size_t most = count.size() - 1 + static_cast<size_t>(kUnitSteps);
  int64_t load = 0;
  int at = 0;
  for (size_t c = count.size(); c-- > 0;) {
    const int n = count[c];
    load += static_cast<int64_t>(n) * (c + static_cast<size_t>(kUnitSteps));
    count[c] = at;
    at += n;
  }
  std::vector<std::pair<uint32_t, int>> sorted(pp.total_units);   // (unit, cost)
  for (int s = 0; s < pp.n_seqs; ++s)
    for (int b = 0; b < pp.per_head[s]; ++b) {
      const size_t c = steps(s, b);
      for (int h = 0; h < pp.n_kv; ++h)
        sorted[count[c]++] = {static_cast<uint32_t>(s) << 24 | static_cast<uint32_t>(b * pp.n_kv + h), static_cast<int>(c) + static_cast<int>(kUnitSteps)};
    }
  std::vector<int> with(load / grid + most + 1, -1), next(grid), held(grid, 0);      // the first CTA with a load, the next with the same, a CTA's units
  for (int j = grid; j-- > 0;) { next[j] = with[0]; with[0] = j; }
  int rounds = 0;
  size_t least = 0;
  auto place = [&](int r, int j) { return r * grid + (r & 1 ? grid - 1 - j : j); };  // (attn_unit_at)
  for (const auto& [unit, cost] : sorted) {
    while (with[least] < 0) ++least;
    const int j = with[least], r = held[j]++;
    with[least] = next[j];
    next[j] = with[least + cost];
    with[least + cost] = j;
    if ((r + 1) * grid > kPromptListed) return;                  // (dealt without a list)
    rounds = std::max(rounds, r + 1);
    pp.list[place(r, j)] = unit;
  }
  for (int j = 0; j < grid; ++j)
    for (int r = held[j]; r < rounds; ++r) pp.list[place(r, j)] = kPromptNoUnit;
  pp.total_units = rounds * grid;
  pp.listed = 1;
}
static Divider divider(int d) {
  return Divider{d >= 2 && d <= 256 ? static_cast<uint32_t>(((1ull << 32) + d - 1) / d) : 0u, d};
}
static int64_t prompt_units(const eas_prompt_inputs* in, const PromptPlan& plan, int i) {
  const int64_t tiles = (static_cast<int64_t>(in->cu_q[i + 1]) - in->cu_q[i] + plan.tile_tokens - 1) / plan.tile_tokens;
  return (tiles + plan.wg - 1) / plan.wg * in->n_kv_heads;
}
static size_t prompt_part_bytes(int wg, int hd) { return static_cast<size_t>(wg) * 128 * (static_cast<size_t>(hd) * 4 + 8); }

static eas_status check_prompt(const eas_prompt_inputs* in) {
  if (in == nullptr) return fail(EAS_ERR_INVALID_ARG, "inputs are null");
  const int H = in->n_heads, G = in->n_kv_heads, hd = in->head_dim, n = in->n_seqs;
  if (n < 0) return fail(EAS_ERR_INVALID_ARG, "n_seqs %d", n);
  if (in->cu_q == nullptr || in->cu_k == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (in->dtype != EAS_DTYPE_BF16 && in->dtype != EAS_DTYPE_FP16) return fail(EAS_ERR_UNSUPPORTED, "dtype %d", in->dtype);
  if (hd != 64 && hd != 128) return fail(EAS_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", hd);
  if (H <= 0 || G <= 0 || H % G != 0) return fail(EAS_ERR_INVALID_ARG, "%d query heads for %d key/value heads", H, G);
  if (H / G > 128) return fail(EAS_ERR_UNSUPPORTED, "%d query heads per key/value head (at most 128)", H / G);
  if (in->cu_q[0] < 0 || in->cu_k[0] < 0) return fail(EAS_ERR_INVALID_ARG, "cu_q and cu_k start at 0 or above");
  for (int i = 0; i < n; ++i)
    if (in->cu_q[i + 1] < in->cu_q[i] || in->cu_k[i + 1] < in->cu_k[i])
      return fail(EAS_ERR_INVALID_ARG, "cu_q or cu_k decreases at sequence %d", i);
  return EAS_OK;
}

// the cuts of a call's launches on this device, and its scratch: that of its costliest launch
static size_t prompt_cuts(const eas_prompt_inputs* in, const PromptPlan& plan, int sms, std::vector<PromptCut>* cuts) {
  size_t bytes = 0;
  const int rows = static_cast<int>(plan.order.size());
  for (int first = 0; first < rows; first += kPromptMaxSeqs) {
    cuts->push_back(prompt_cut(in, plan, first, std::min(kPromptMaxSeqs, rows - first), sms));
    bytes = std::max(bytes, static_cast<size_t>(cuts->back().items) * prompt_part_bytes(plan.wg, in->head_dim));
  }
  return bytes;
}
// every launch of a call, before the first one
static eas_status check_prompt_units(const eas_prompt_inputs* in, const PromptPlan& plan) {
  int64_t units = 0;
  for (size_t j = 0; j < plan.order.size(); ++j) {
    units = (j % kPromptMaxSeqs == 0 ? 0 : units) + prompt_units(in, plan, plan.order[j]);
    if (units > (1 << 24)) return fail(EAS_ERR_UNSUPPORTED, "too many query rows for one call");
  }
  return EAS_OK;
}

static eas_status prompt_attention(const eas_prompt_inputs* in, void* workspace, size_t workspace_bytes, int32_t sm_budget, void* stream,
                                   uint32_t* status_dev) {
  EAS_TRY(check_prompt(in));
  if (status_dev == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (!(in->scale > 0.0f) || !std::isfinite(in->scale)) return fail(EAS_ERR_INVALID_ARG, "scale must be positive and finite");
  const int H = in->n_heads, G = in->n_kv_heads, hd = in->head_dim, n = in->n_seqs;
  const int64_t Tq = in->cu_q[n], Tk = in->cu_k[n], wq = static_cast<int64_t>(H) * hd, wk = static_cast<int64_t>(G) * hd;
  if (Tq > in->cu_q[0]) {
    if (in->q == nullptr || in->out == nullptr || (Tk > 0 && (in->k == nullptr || in->v == nullptr)))
      return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
    if (!aligned16(in->q) || !aligned16(in->out) || (Tk > 0 && (!aligned16(in->k) || !aligned16(in->v))))
      return fail(EAS_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
    if (in->ld_q < wq || in->ld_out < wq || in->ld_q % 8 != 0 || in->ld_out % 8 != 0 ||
        (Tk > 0 && (in->ld_k < wk || in->ld_v < wk || in->ld_k % 8 != 0 || in->ld_v % 8 != 0)))
      return fail(EAS_ERR_INVALID_ARG, "token distances must be multiples of 8 that hold a token's heads");
  }
  const PromptPlan plan = prompt_plan(in);
  EAS_TRY(check_prompt_units(in, plan));
  int budget = 0;
  EAS_TRY(resolve_budget(sm_budget, &budget));
  if (Tq == in->cu_q[0]) return EAS_OK;                          // no query

  PromptParams pp;                                               // (the list behind it is not cleared)
  pp.listed = 0; pp.o_ws = nullptr; pp.ml_ws = nullptr;
  pp.group = H / G; pp.n_kv = G; pp.tile_tokens = 128 / pp.group;
  EAS_TRY(prompt_q_map(&pp.map_q, in->q, H, hd, Tq, in->ld_q, pp.group, pp.tile_tokens));
  if (Tk > 0) {
    EAS_TRY(prompt_kv_map(&pp.map_k, in->k, G, hd, Tk, in->ld_k, PromptCfg<64>::kKeys));
    EAS_TRY(prompt_kv_map(&pp.map_v, in->v, G, hd, Tk, in->ld_v, PromptCfg<64>::kKeys));
  } else {                                                       // (no key at all: no tile is ever loaded)
    pp.map_k = pp.map_v = pp.map_q;
  }
  static_assert(PromptCfg<64>::kKeys == PromptCfg<128>::kKeys, "one box for both");
  pp.q = static_cast<const uint16_t*>(in->q); pp.k = static_cast<const uint16_t*>(in->k); pp.v = static_cast<const uint16_t*>(in->v);
  pp.out = static_cast<uint16_t*>(in->out);
  pp.ld_q = in->ld_q; pp.ld_k = in->ld_k; pp.ld_v = in->ld_v; pp.ld_out = in->ld_out;
  pp.out_wide = (reinterpret_cast<uintptr_t>(in->out) & 31) == 0 && in->ld_out % 16 == 0;
  pp.scale_log2 = static_cast<float>(in->scale * kLog2e);
  pp.status = status_dev;
  const int sms = g_device_sms;
  std::vector<PromptCut> cuts;
  const size_t need = prompt_cuts(in, plan, sms, &cuts);
  if (workspace_bytes < need || (need > 0 && workspace == nullptr))
    return fail(EAS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace == nullptr ? 0 : workspace_bytes, need);
  if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return fail(EAS_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  const bool all = budget == sms, h = in->dtype == EAS_DTYPE_FP16;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int rows = static_cast<int>(plan.order.size());
  for (int first = 0; first < rows; first += kPromptMaxSeqs) {
    pp.n_seqs = std::min(kPromptMaxSeqs, rows - first);
    int64_t units = 0;
    for (int j = 0; j < pp.n_seqs; ++j) {
      const int i = plan.order[first + j];
      pp.q0[j] = in->cu_q[i]; pp.len_q[j] = in->cu_q[i + 1] - in->cu_q[i];
      pp.k0[j] = in->cu_k[i]; pp.len_k[j] = in->cu_k[i + 1] - in->cu_k[i];
      pp.unit_prefix[j] = static_cast<int>(units);
      pp.tiles[j] = (pp.len_q[j] - 1) / pp.tile_tokens + 1;
      pp.per_head[j] = (pp.tiles[j] - 1) / plan.wg + 1;
      units += prompt_units(in, plan, i);
    }
    pp.unit_prefix[pp.n_seqs] = static_cast<int>(units);
    pp.total_units = static_cast<int>(units);
    pp.by_kv = divider(G);
    const PromptCut& cut = cuts[first / kPromptMaxSeqs];
    if (cut.pieces > 0) {
      PromptParamsSplit split;
      static_cast<PromptSeqs<kPromptMaxSeqs>&>(split) = pp;
      prompt_items(split, cut, plan.wg);
      split.o_ws = static_cast<float4*>(workspace);
      split.ml_ws = reinterpret_cast<float2*>(split.o_ws + static_cast<size_t>(split.total_units) * plan.wg * 128 * (hd / 4));
      EAS_TRY(launch_prompt(split, hd, h, budget, all, st));
      continue;
    }
    pp.listed = 0;
    if (units <= kPromptListed && units > budget && pp.n_seqs > 1) prompt_list(pp, plan.wg, budget);
    EAS_TRY(pp.listed || pp.n_seqs > PromptParamsFew::kSeqs ? launch_prompt(pp, hd, h, budget, all, st) : launch_prompt(few_of(pp), hd, h, budget, all, st));
  }
  return EAS_OK;
}

// ------------------------------------------------------------------------------------ cache
// the cache as rows of head_dim bytes: a box is part of one head of one block
static eas_status cache_map(CUtensorMap* m, const int8_t* base, const eas_cache_desc& d) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = get_encode_fn();
  if (fn == nullptr) return fail(EAS_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t gdim[2] = {static_cast<cuuint64_t>(d.head_dim), static_cast<cuuint64_t>(d.n_blocks) * d.n_kv_heads * d.block_size};
  const cuuint64_t gstr[1] = {static_cast<cuuint64_t>(d.head_dim)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(d.head_dim), static_cast<cuuint32_t>(std::min(d.block_size, 32))};
  const cuuint32_t es[2] = {1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(base), gdim, gstr, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  d.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(EAS_ERR_CUDA, "cuTensorMapEncodeTiled (cache) failed with code %d", static_cast<int>(r));
  return EAS_OK;
}

static eas_status cache_create(const eas_cache_desc* d, eas_cache** out) {
  if (out == nullptr) return fail(EAS_ERR_INVALID_ARG, "out is null");
  *out = nullptr;
  if (d == nullptr || d->k == nullptr || d->v == nullptr || d->k_scale == nullptr || d->v_scale == nullptr)
    return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(EAS_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
  if (d->block_size != 16 && d->block_size != 32 && d->block_size != 64 && d->block_size != 128)
    return fail(EAS_ERR_UNSUPPORTED, "block_size %d (supported: 16, 32, 64, 128)", d->block_size);
  if (d->n_blocks <= 0 || d->n_kv_heads <= 0) return fail(EAS_ERR_INVALID_ARG, "non-positive cache size");
  if (static_cast<int64_t>(d->n_blocks) * d->n_kv_heads > 0x7fffffffLL / d->block_size)
    return fail(EAS_ERR_UNSUPPORTED, "more than 2^31 - 1 rows of tokens and heads");
  if (!aligned16(d->k) || !aligned16(d->v)) return fail(EAS_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  eas_cache c{};
  c.d = *d;
  EAS_TRY(device_check(&c.sm_count, &c.device));
  for (c.bs_log2 = 4; (1 << c.bs_log2) < d->block_size; ++c.bs_log2) {}
  EAS_TRY(cache_map(&c.map_k, d->k, *d));
  EAS_TRY(cache_map(&c.map_v, d->v, *d));
  *out = new (std::nothrow) eas_cache(c);
  return *out != nullptr ? EAS_OK : fail(EAS_ERR_INVALID_ARG, "out of host memory");
}

// One CTA an SM: on a share of the SMs the shared-memory request keeps a second one out; on all of them it is not needed, and L1 is larger.
template <int HD, int GT, typename T>
static eas_status launch_store(const CacheRowsParams& p, int budget, bool all, cudaStream_t stream) {
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(cache_store_kernel<HD, GT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  int groups = 512 / GT;                                         // few units: fewer groups of threads a CTA, so that every SM has some
  while (groups > 1 && static_cast<long long>(groups / 2) * budget >= p.units) groups /= 2;
  const int grid = static_cast<int>(std::min<long long>(budget, (p.units + groups - 1) / groups));
  return launch_kernel(cache_store_kernel<HD, GT, T>, grid, groups * GT, all ? 0 : kOnePerSmSmem, stream, p);
}
template <int HD, typename T>
static eas_status launch_rows(bool store, const CacheRowsParams& p, int budget, bool all, cudaStream_t stream) {
  if (store) {
    switch (HD << p.c.bs_log2) {                                 // values of a block and head: 64 a thread
      case 16384: return launch_store<HD, 256, T>(p, budget, all, stream);
      case 8192: return launch_store<HD, 128, T>(p, budget, all, stream);
      case 4096: return launch_store<HD, 64, T>(p, budget, all, stream);
      default: return launch_store<HD, 32, T>(p, budget, all, stream);
    }
  }
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(cache_load_kernel<HD, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  int warps = 16;
  while (warps > 4 && warps / 2 * budget >= p.n_rows) warps /= 2;
  return launch_kernel(cache_load_kernel<HD, T>, std::min(budget, (p.n_rows + warps - 1) / warps), warps * 32, all ? 0 : kOnePerSmSmem, stream, p);
}

static eas_status cache_rows(bool store, const eas_cache* c, const eas_cache_seqs* s, void* k, int64_t ld_k, void* v, int64_t ld_v, int32_t n_rows,
                             int32_t dtype, int32_t sm_budget, void* stream, uint32_t* status_dev) {
  int budget = 0;
  EAS_TRY(check_cache_call(c, s, true, dtype, status_dev, sm_budget, &budget));
  if (n_rows < 0) return fail(EAS_ERR_INVALID_ARG, "n_rows %d", n_rows);
  if (n_rows == 0 || s->n_seqs == 0) return EAS_OK;
  if (k == nullptr || v == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  const int64_t w = static_cast<int64_t>(c->d.n_kv_heads) * c->d.head_dim;
  if (!aligned16(k) || !aligned16(v)) return fail(EAS_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (ld_k < w || ld_v < w || ld_k % 8 != 0 || ld_v % 8 != 0)
    return fail(EAS_ERR_INVALID_ARG, "token distances must be multiples of 8 that hold a token's heads");
  CacheRowsParams p{};
  p.c = view_of(c);
  p.s = CacheSeqs{s->block_table, s->cu_seqlens, s->start, s->ld_table, s->n_seqs, s->max_blocks};
  p.k = k; p.v = v; p.ld_k = ld_k; p.ld_v = ld_v; p.n_rows = n_rows;
  const int64_t pairs = (n_rows >> c->bs_log2) + 2LL * s->n_seqs;
  if (pairs * c->d.n_kv_heads > 0x7fffffffLL) return fail(EAS_ERR_UNSUPPORTED, "too many rows for one call");
  p.units = pairs * c->d.n_kv_heads * 2;
  p.status = status_dev;
  const bool all = budget == c->sm_count, h = dtype == EAS_DTYPE_FP16;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (c->d.head_dim == 64) return h ? launch_rows<64, __half>(store, p, budget, all, st) : launch_rows<64, bf16>(store, p, budget, all, st);
  return h ? launch_rows<128, __half>(store, p, budget, all, st) : launch_rows<128, bf16>(store, p, budget, all, st);
}

// pieces of the line of tiles: a function of the device, not of sm_budget (the sums' order depends on them)
static int attention_rows(int group) { return group <= 8 ? 8 : 16; }
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
static size_t attention_workspace(const eas_cache* c, int32_t n_heads, size_t* o_off) {
  const int r = attention_rows(n_heads / c->d.n_kv_heads);
  const int warps = r == 8 ? CacheAttnCfg<128, 1>::kWarps : CacheAttnCfg<128, 2>::kWarps;
  const size_t rows = static_cast<size_t>(2) * c->sm_count * warps * r;
  *o_off = up256(rows * 8);
  return *o_off + rows * c->d.head_dim * 4;
}

template <int HD, int NT>
static eas_status launch_attention(CacheAttnParams& p, int budget, bool all, cudaStream_t stream) {
  using L = CacheAttnCfg<HD, NT>;
  static OncePerDevice once;
  if (once.first()) {
    CUDA_TRY(cudaFuncSetAttribute(cache_attention_kernel<HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes));
    CUDA_TRY(cudaFuncSetAttribute(cache_join_kernel<HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOnePerSmSmem));
    once.settled();
  }
  EAS_TRY(launch_kernel(cache_attention_kernel<HD, NT>, std::min(budget, p.n_ctas), L::kThreads, L::kBytes, stream, p));
  constexpr int kJoinWarps = kCacheJoinThreads / 32;
  const int64_t heads = static_cast<int64_t>(p.n_seqs) * p.c.n_kv * p.group;
  return launch_kernel(cache_join_kernel<HD, NT>, static_cast<int>(std::min<int64_t>(budget, (heads + kJoinWarps - 1) / kJoinWarps)), kCacheJoinThreads, all ? 0 : kOnePerSmSmem, stream, p);
}

static eas_status cache_attention(const eas_cache* c, const eas_cache_seqs* s, const void* q, int64_t ld_q, void* out, int64_t ld_out, int32_t n_heads,
                                  int32_t dtype, float scale, void* workspace, size_t workspace_bytes, int32_t sm_budget, void* stream,
                                  uint32_t* status_dev) {
  int budget = 0;
  EAS_TRY(check_cache_call(c, s, false, dtype, status_dev, sm_budget, &budget));
  const int G = c->d.n_kv_heads, hd = c->d.head_dim;
  if (n_heads <= 0 || n_heads % G != 0) return fail(EAS_ERR_INVALID_ARG, "%d query heads for %d key/value heads", n_heads, G);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(EAS_ERR_INVALID_ARG, "scale must be positive and finite");
  if (s->n_seqs == 0) return EAS_OK;
  if (q == nullptr || out == nullptr || workspace == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (!aligned16(q) || !aligned16(out)) return fail(EAS_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  const int64_t w = static_cast<int64_t>(n_heads) * hd;
  if (ld_q < w || ld_out < w || ld_q % 8 != 0 || ld_out % 8 != 0)
    return fail(EAS_ERR_INVALID_ARG, "token distances must be multiples of 8 that hold a token's heads");
  size_t o_off = 0;
  const size_t need = attention_workspace(c, n_heads, &o_off);
  if (workspace_bytes < need) return fail(EAS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return fail(EAS_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  CacheAttnParams p{};
  p.map_k = c->map_k; p.map_v = c->map_v;
  p.c = view_of(c);
  p.group = n_heads / G;
  const int rows = attention_rows(p.group), tile = 32;      // (no variant's tile is smaller)
  p.row_blocks = (p.group + rows - 1) / rows;
  const int64_t places = static_cast<int64_t>(s->max_blocks) * c->d.block_size, tiles = (places + tile - 1) / tile + kRowCost;
  if (places > 0x7fffffffLL || tiles * G * p.row_blocks > 0x7fffffffLL / std::min(s->n_seqs, kCacheMaxSeqs))
    return fail(EAS_ERR_UNSUPPORTED, "max_blocks %d is too large for %d sequences", s->max_blocks, s->n_seqs);
  p.ld_table = s->ld_table; p.max_blocks = s->max_blocks;
  p.ld_q = ld_q; p.ld_out = ld_out; p.fp16 = dtype == EAS_DTYPE_FP16;
  p.n_ctas = c->sm_count;
  p.scale_log2 = static_cast<float>(scale * kLog2e);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.ml_ws = reinterpret_cast<float*>(ws); p.o_ws = reinterpret_cast<float*>(ws + o_off);
  p.status = status_dev;
  const bool all = budget == c->sm_count;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < s->n_seqs; first += kCacheMaxSeqs) {
    p.n_seqs = std::min(kCacheMaxSeqs, s->n_seqs - first);
    p.table = s->block_table + first * s->ld_table;
    p.seq_lens = s->seq_lens + first;
    p.q = static_cast<const uint16_t*>(q) + first * ld_q;
    p.out = static_cast<uint16_t*>(out) + first * ld_out;
    EAS_TRY(hd == 64 ? (rows == 8 ? launch_attention<64, 1>(p, budget, all, st) : launch_attention<64, 2>(p, budget, all, st))
                     : (rows == 8 ? launch_attention<128, 1>(p, budget, all, st) : launch_attention<128, 2>(p, budget, all, st)));
  }
  return EAS_OK;
}

// ------------------------------------------------------------------------------------ entry points (no exception passes them)
extern "C" size_t eas_prompt_attention_workspace_bytes(const eas_prompt_inputs* in) {
  int sms = 0;
  if (check_prompt(in) != EAS_OK || device_check(&sms) != EAS_OK) return 0;
  try {
    std::vector<PromptCut> cuts;
    return prompt_cuts(in, prompt_plan(in), sms, &cuts);
  } catch (const std::bad_alloc&) {
    fail(EAS_ERR_INVALID_ARG, "out of host memory");
    return 0;
  }
}

extern "C" eas_status eas_prompt_attention(const eas_prompt_inputs* in, void* workspace, size_t workspace_bytes, int32_t sm_budget, void* stream,
                                           uint32_t* status_dev) {
  try {
    return prompt_attention(in, workspace, workspace_bytes, sm_budget, stream, status_dev);
  } catch (const std::bad_alloc&) {
    return fail(EAS_ERR_INVALID_ARG, "out of host memory");
  }
}

extern "C" eas_status eas_cache_create(const eas_cache_desc* desc, eas_cache** out) { return cache_create(desc, out); }

extern "C" void eas_cache_destroy(eas_cache* cache) { delete cache; }

extern "C" eas_status eas_cache_store(const eas_cache* cache, const eas_cache_seqs* seqs, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                      int32_t n_rows, int32_t dtype, int32_t sm_budget, void* stream, uint32_t* status_dev) {
  return cache_rows(true, cache, seqs, const_cast<void*>(k), ld_k, const_cast<void*>(v), ld_v, n_rows, dtype, sm_budget, stream, status_dev);
}

extern "C" eas_status eas_cache_load(const eas_cache* cache, const eas_cache_seqs* seqs, void* k, int64_t ld_k, void* v, int64_t ld_v, int32_t n_rows,
                                     int32_t dtype, int32_t sm_budget, void* stream, uint32_t* status_dev) {
  return cache_rows(false, cache, seqs, k, ld_k, v, ld_v, n_rows, dtype, sm_budget, stream, status_dev);
}

extern "C" size_t eas_cache_attention_workspace_bytes(const eas_cache* cache, int32_t n_seqs, int32_t n_heads) {
  if (cache == nullptr || n_seqs < 0 || n_heads <= 0 || n_heads % cache->d.n_kv_heads != 0) {
    fail(EAS_ERR_INVALID_ARG, "bad arguments");
    return 0;
  }
  size_t o_off = 0;
  return attention_workspace(cache, n_heads, &o_off);
}

extern "C" eas_status eas_cache_attention(const eas_cache* cache, const eas_cache_seqs* seqs, const void* q, int64_t ld_q, void* out, int64_t ld_out,
                                          int32_t n_heads, int32_t dtype, float scale, void* workspace, size_t workspace_bytes, int32_t sm_budget,
                                          void* stream, uint32_t* status_dev) {
  return cache_attention(cache, seqs, q, ld_q, out, ld_out, n_heads, dtype, scale, workspace, workspace_bytes, sm_budget, stream, status_dev);
}
