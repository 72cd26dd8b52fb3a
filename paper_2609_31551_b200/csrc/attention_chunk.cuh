// Attention of several new tokens a sequence over the 8-bit cache: out = softmax(scale q K^T) V, the new tokens being the last of their sequence.
#pragma once
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace eas {

struct ChunkParams {
  CacheView c;
  const int32_t *table, *cu, *seq_lens;
  long long ld_table;
  int n_seqs, max_blocks, n_rows, max_new;
  const uint16_t* q;
  uint16_t* out;
  long long ld_q, ld_out;
  int fp16, group;
  float scale_log2;
  uint32_t* status;
  int early_launch;
};

// The simplest form: 128 threads per (row, query head), 128 tokens at a time: a thread has a token's score, then a dimension's sum.
template <int HD>
__global__ void __launch_bounds__(128) chunk_simple_kernel(const __grid_constant__ ChunkParams p) {
  __shared__ float q[HD], w[128], vs[128];
  __shared__ int ids[128];
  pdl_wait();
  if (p.early_launch) pdl_launch_dependents();
  const int heads = p.c.n_kv * p.group, t = threadIdx.x;
  auto cu = [&](int i) { return min(max(p.cu[i], 0), p.n_rows); };
  for (long long u = blockIdx.x; u < static_cast<long long>(p.n_rows) * heads; u += gridDim.x) {
    const int row = static_cast<int>(u / heads), h = static_cast<int>(u - static_cast<long long>(row) * heads), kvh = h / p.group;
    int s = 0, hi = p.n_seqs - 1;
    while (s < hi) {
      const int mid = (s + hi + 1) >> 1;
      if (cu(mid) <= row) s = mid; else hi = mid - 1;
    }
    const int first = cu(s), n = cu(s + 1) - first;
    if (row < first || row >= first + n) continue;
    const long long most = static_cast<long long>(p.max_blocks) << p.c.bs_log2;
    const int len = static_cast<int>(min(static_cast<long long>(max(p.seq_lens[s], 0)), most));
    if (t == 0 && (n > p.max_new || p.seq_lens[s] > most)) raise_status(p.status, DEV_ERR_CACHE_RANGE);
    if (n > p.max_new) continue;
    const int limit = len - n + row - first + 1;
    __syncthreads();
    for (int i = t; i < HD; i += 128) q[i] = load16(p.q[row * p.ld_q + h * HD + i], p.fp16);
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int base = 0; base < limit; base += 128) {
      float x = -INFINITY;
      int id = -1;
      float v_scale = 0.f;
      if (base + t < limit) {
        id = p.table[s * p.ld_table + ((base + t) >> p.c.bs_log2)];
        if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.c.n_blocks)) {
          raise_status(p.status, DEV_ERR_CACHE_RANGE);
          id = -1;
        }
      }
      __syncthreads();
      if (id >= 0) {
        const long long at = static_cast<long long>(id) * p.c.n_kv + kvh;
        const int8_t* k = p.c.k + ((at << p.c.bs_log2) + ((base + t) & ((1 << p.c.bs_log2) - 1))) * HD;
        float d = 0.f;
        for (int i = 0; i < HD; ++i) d = fmaf(q[i], static_cast<float>(k[i]), d);
        x = d * p.c.k_scale[at] * p.scale_log2;
        v_scale = p.c.v_scale[at];
      }
      w[t] = x;
      vs[t] = v_scale;
      ids[t] = id;
      __syncthreads();
      float top = m;
      for (int i = 0; i < 128; ++i) top = fmaxf(top, w[i]);
      const float corr = m == -INFINITY ? 0.f : fast_ex2(m - top);
      m = top;
      l *= corr;
      o *= corr;
      for (int i = 0; i < 128 && base + i < limit; ++i) {
        if (ids[i] < 0) continue;
        const float e = fast_ex2(w[i] - m);
        l += e;
        if (t < HD) {
          const long long at = static_cast<long long>(ids[i]) * p.c.n_kv + kvh;
          o = fmaf(e * vs[i], static_cast<float>(p.c.v[((at << p.c.bs_log2) + ((base + i) & ((1 << p.c.bs_log2) - 1))) * HD + t]), o);
        }
      }
      __syncthreads();
    }
    if (t < HD) {
      const float y = l == 0.f ? 0.f : o / l;
      p.out[row * p.ld_out + h * HD + t] = static_cast<uint16_t>((p.fp16 ? Pair16<__half>::pack(y, 0.f) : Pair16<bf16>::pack(y, 0.f)) & 0xFFFFu);
    }
  }
}

}  // namespace eas
