// sb_tree_attention_quant: argument checks, choice of kernel and of KV chunks, and the merge of chunks that do not share
// a cluster.
#include "quant_attention.cuh"

namespace sb {

// Log-sum-exp merge of the chunks' partials, 16 bytes of a row per lane.  P16: fp16 partials with exponents (tcgen05 kernel), else fp32.
// A NaN partial makes the row NaN.
template <int D, bool P16>
__global__ void __launch_bounds__(256) quant_merge_kernel(const QuantAttnParams p) {
  constexpr int EPL = P16 ? 8 : 4, LPR = D / EPL, RPW = 32 / LPR;
  pdl_wait();
  pdl_release();
  const int b = blockIdx.y;
  const QuantSeq si = load_quant_seq(p, b);
  if (!si.can_write) return;
  const int Hq = p.tree.n_q_heads, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rr = (blockIdx.x * 8 + warp) * RPW + lane / LPR, col = lane % LPR;
  if (rr >= si.nq * Hq) return;
  const long long rows_all = (long long)p.total_q * Hq;
  const long long grow = (long long)si.q_off * Hq + rr;
  if (!SB_CHECKED_ACCESS(grow, rows_all, &p.status[b])) return;
  float M = -INFINITY;
  for (int s = 0; s < p.outer; ++s) M = fmaxf(M, p.part_lse[s * rows_all + grow]);
  float acc[EPL], sum = 0.f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
#pragma unroll 4
  for (int s = 0; s < p.outer; ++s) {
    const float lse2 = p.part_lse[s * rows_all + grow];
    const char* row = reinterpret_cast<const char*>(p.part_o) + (s * rows_all + grow) * (P16 ? kPartRow<D> : D * 4);
    const uint4 raw = *reinterpret_cast<const uint4*>(row + col * 16);
    float w = lse2 == -INFINITY ? 0.f : fast_exp2(lse2 - M);
    sum += w;
    if (P16) w *= __uint_as_float((uint32_t)(*reinterpret_cast<const uint8_t*>(row + D * 2 + col) - 14) << 23);
    const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (P16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[e]));
        acc[(2 * e) % EPL] = fmaf(w, f.x, acc[(2 * e) % EPL]);
        acc[(2 * e + 1) % EPL] = fmaf(w, f.y, acc[(2 * e + 1) % EPL]);
      } else {
        acc[e] = fmaf(w, __uint_as_float(u[e]), acc[e]);
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + grow * D + col * EPL);
#pragma unroll
  for (int e = 0; e < EPL; e += 2) dst[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
  if (p.lse && col == 0) p.lse[grow] = sum == 0.f ? 0.f : (M + log2f(sum)) * kLn2;
}

struct QuantPlan {
  bool tc;                         // the tcgen05 kernel; else the 16-row kernel
  int cluster, outer, grid_tiles;  // grid_tiles: row tiles (16 or 128 rows) per KV head
};

static QuantPlan plan_quant(const sb_quant_cache* kv, const sb_quant_tree* tree, int total_q, int window, int sinks, int num_splits) {
  QuantPlan pl;
  const int G = tree->n_q_heads / kv->n_kv_heads;
  const int nq = tree->max_nodes < total_q ? tree->max_nodes : total_q;
  const int rows = (nq > 0 ? nq : 1) * G;
  long long keys = tree->max_prefix;  // visible ones, at most
  if (window > 0 && (long long)window + sinks + 64 < keys) keys = (long long)window + sinks + 64;
  const int sms = device_sms();
  // The 16-row kernel starts and ends in less time (9 us against 12), but walks the keys once per 16 rows, with the slower matrix
  // instructions.  us by it and by the tcgen05 kernel, 8 KV heads, groups of 4: 1 to 4 nodes (one tile), 2k keys 11.7 / 18.6, 64 ragged 8k
  // prefixes 143 / 199; 16 nodes over 128, 512, 2k keys 10 / 12, 11 / 15, 14 / 18; 32 nodes 11 / 12, 13 / 15, 19 / 18.5; 60 nodes
  // 13 / 13, 17 / 16, 29 / 20; 8 nodes, 4 ragged 8k prefixes 37 / 34, 16 of them 84 / 70, 64 of them 232 / 199.  (These and the counts of chunks
  // below were measured with D = 128 and that head layout; others go by the same numbers.)
  const long long tiles = (long long)kv->batch * kv->n_kv_heads * ceil_div(rows, 16);
  pl.tc = rows > 16 && (tiles > 64 || tiles * keys > (1 << 17));
  pl.cluster = 1;
  if (pl.tc) {
    // A CTA costs its key blocks plus a fixed start and end.  CTAs start longest first on whichever SM is free: equal ones run in waves,
    // ragged ones (three quarters of the longest, taken on average) end about half a chunk unevenly; the estimate lies between the two.
    // Every chunk beyond the first writes and re-reads fp16 partials of all rows, and the merge is one more kernel.  us by 1 / 2 / 3 / 4 /
    // 6 chunks: one 60-node tree over 2k keys 34 / 27 / 23 / 21 / 20; 8-node trees over ragged 8k prefixes, 4 of them 79 / 49 / 38 / 34 /
    // 39, 16: 81 / 70 / 80 / 88 / 107, 64: 199 / 247 / 291 / 327 / 408; four full trees, 64 heads, over 32k keys 651 / 682 / 679 / 643 / 726.
    pl.grid_tiles = ceil_div(rows, 128);
    const int blocks = (int)((keys + 127) / 128) + (window > 0 ? 2 : 0) + 1;
    const double units = (double)kv->batch * kv->n_kv_heads * pl.grid_tiles;
    const double per_block = 1.28, fixed = 10.0;  // us
    const double partial = 2.0 * (double)total_q * tree->n_q_heads * kv->head_dim * 2.0 / 5e6;
    int best = 1;
    double best_cost = 0.0;
    const int most = num_splits > 0 ? 1 : (blocks < 64 ? blocks : 64);
    for (int s = 1; s <= most; ++s) {
      const double longest = ceil_div(blocks, s) * per_block + fixed;
      double cost = longest;
      if (units * s > sms) {
        const double even = ceil(units * s / sms) * longest;                                          // waves of equal chunks
        const double ragged = units * (0.75 * blocks * per_block + fixed * s) / sms + 0.5 * longest;  // of any length
        const double sum = 0.3 * even + 0.7 * ragged;
        if (sum > longest) cost = sum;
      }
      if (s > 1) cost += partial * s + 1.0 + 0.5 * s;
      if (s == 1 || cost < best_cost) {
        best = s;
        best_cost = cost;
      }
    }
    pl.outer = num_splits > 0 ? (num_splits < blocks ? num_splits : blocks) : best;
    return pl;
  }
  // Chunks per (sequence, KV head, tile), grouped into clusters of up to 8.  About 520 CTAs measured best (three fit on an SM; ragged
  // 4k prefixes, 8 KV heads, us by 1 / 2 / 3 / 4 / 6 / 8 chunks: 8 sequences 113 / 62 / 49 / 39 / 37 / 35, 16: 115 / 71 / 61 / 51 /
  // 54 / 64, 32: 150 / 89 / 89 / 94 / 103 / 124, 64: 159 / 138 / 156 / 164 / 183 / 227, 128: 263 / 285 / 329): a chunk per CTA
  // alone is bound by its own latency, every further CTA costs its start and its merge.  More than 8 chunks need the merge kernel, which
  // pays from about 5k keys on (32k: 67 us by 8, 29 by 32); then one wave of two CTAs per SM.
  pl.grid_tiles = ceil_div(rows, 16);
  const int groups = (int)((keys + 31) / 32) + (window > 0 ? 2 : 0) + ceil_div(tree->max_nodes, 16);
  const long long units = tiles;
  int s;
  if (num_splits > 0) {
    s = num_splits;
  } else {
    s = (int)((520 + units - 1) / units);
    // several tiles of rows: 32 of them over 2k keys 23 / 17 / 14 / 19 us by 2 / 4 / 6 / 8 chunks, 64: 24 / 19 / 19 / 33
    if (rows > 16 && units > 16) s = units > 32 ? 4 : 6;
    const int most = ceil_div(groups, 4);  // a group for each of the four warps
    if (s > most) s = most;
    if (s > kQuantMaxCluster) {
      s = groups > 160 ? (int)(2LL * sms / units) : kQuantMaxCluster;
      s = s < kQuantMaxCluster ? kQuantMaxCluster : (s > 64 ? 64 : s / kQuantMaxCluster * kQuantMaxCluster);
    } else if (s == 5 || s == 7) {
      --s;                                 // rows divide evenly among 4 or 6
    }
  }
  if (s > groups) s = groups;
  if (s < 1) s = 1;
  for (int c = kQuantMaxCluster; c >= 1; --c)
    if (s % c == 0) { pl.cluster = c; break; }
  pl.outer = s / pl.cluster;
  return pl;
}

static sb_status check_quant_call(const sb_quant_cache* kv, const sb_quant_tree* tree, int window, int sinks, int num_splits) {
  const sb_status st = check_quant_cache(kv);
  if (st != SB_OK) return st;
  if (!tree || !tree->prefix_len || !tree->node_offsets || !tree->parent || tree->n_q_heads < 1 ||
      tree->n_q_heads % kv->n_kv_heads != 0 || tree->total_nodes < 0 || tree->max_prefix < 0)
    return SB_ERR_INVALID_ARG;
  if (window < 0 || sinks < 0 || (window == 0 && sinks != 0) || num_splits < 0) return SB_ERR_INVALID_ARG;
  if (tree->n_q_heads / kv->n_kv_heads > 16) return SB_ERR_UNSUPPORTED;
  if (tree->max_nodes < 1 || tree->max_nodes > SB_MAX_NODES) return SB_ERR_UNSUPPORTED;
  if (kv->batch > 65535 || tree->max_prefix > 0x7fffffff - 256 || window > 0x7fffffff - 256) return SB_ERR_UNSUPPORTED;
  return SB_OK;
}

static size_t quant_workspace_bytes(const sb_quant_cache* kv, const sb_quant_tree* tree, int total_q, int outer) {
  if (outer <= 1) return 0;
  const size_t rows = (size_t)total_q * tree->n_q_heads;
  const size_t o = (size_t)outer * rows * kv->head_dim * sizeof(float), l = (size_t)outer * rows * sizeof(float);
  return ((o + 255) & ~(size_t)255) + ((l + 255) & ~(size_t)255);
}

}  // namespace sb

extern "C" size_t sb_tree_attention_quant_workspace_bytes(const sb_quant_cache* kv, const sb_quant_tree* tree,
                                                          int32_t total_q, int32_t window, int32_t sinks,
                                                          int32_t num_splits) {
  if (sb::check_quant_call(kv, tree, window, sinks, num_splits) != SB_OK || total_q < 0) return 0;
  return sb::quant_workspace_bytes(kv, tree, total_q, sb::plan_quant(kv, tree, total_q, window, sinks, num_splits).outer);
}

extern "C" sb_status sb_tree_attention_quant(const sb_quant_cache* kv, int32_t layer, const sb_quant_tree* tree,
                                             const void* k_nodes, const void* v_nodes, int64_t node_stride,
                                             const int32_t* q_node_begin, const int32_t* q_offsets, int32_t total_q,
                                             const void* q, int64_t q_stride, void* out, float* lse, float scale,
                                             int32_t window, int32_t sinks, int32_t num_splits, void* workspace,
                                             size_t workspace_bytes, int32_t* status, void* stream) {
  sb::TraceRange trace_range("sb_tree_attention_quant");
  using namespace sb;
  const sb_status st = check_quant_call(kv, tree, window, sinks, num_splits);
  if (st != SB_OK) return st;
  if (!k_nodes || !v_nodes || !q || !out || !status || total_q < 1 || !(scale >= 0.f) || layer < 0 || layer >= kv->n_layers)
    return SB_ERR_INVALID_ARG;
  if (q_node_begin && !q_offsets) return SB_ERR_INVALID_ARG;
  const int D = kv->head_dim;
  const int64_t node_width = (int64_t)kv->n_kv_heads * D, q_width = (int64_t)tree->n_q_heads * D;
  if (node_stride == 0) node_stride = node_width;
  if (q_stride == 0) q_stride = q_width;
  if (node_stride < node_width || node_stride % 8 != 0 || q_stride < q_width || q_stride % 8 != 0) return SB_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(k_nodes) |
       reinterpret_cast<uintptr_t>(v_nodes)) & 15)
    return SB_ERR_INVALID_ARG;
  QuantAttnParams p;
  p.kv = *kv;
  p.k_codes = static_cast<const uint8_t*>(kv->k_codes) + layer * kv->codes_layer_stride;
  p.v_codes = static_cast<const uint8_t*>(kv->v_codes) + layer * kv->codes_layer_stride;
  p.k_scale = kv->k_scale + layer * kv->scale_layer_stride;
  p.v_scale = kv->v_scale + layer * kv->scale_layer_stride;
  p.tree = *tree;
  p.k_nodes = static_cast<const bf16*>(k_nodes);
  p.v_nodes = static_cast<const bf16*>(v_nodes);
  p.node_stride = node_stride;
  p.q_node_begin = q_node_begin;
  p.q_offsets = q_offsets;
  p.total_q = total_q;
  p.q = static_cast<const bf16*>(q);
  p.q_stride = q_stride;
  p.out = static_cast<bf16*>(out);
  p.lse = lse;
  p.scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
  p.window = window;
  p.sinks = sinks;
  p.status = status;
  p.block_shift = 0;
  while ((1 << p.block_shift) < kv->scale_block) ++p.block_shift;
  p.G = tree->n_q_heads / kv->n_kv_heads;
  p.g_magic = (1u << 20) / (unsigned)p.G + 1u;
  p.part_o = nullptr;
  p.part_lse = nullptr;
  const QuantPlan pl = plan_quant(kv, tree, total_q, window, sinks, num_splits);
  p.num_splits = pl.cluster * pl.outer;
  p.outer = pl.outer;
  if (pl.outer > 1) {
    if (!workspace || workspace_bytes < quant_workspace_bytes(kv, tree, total_q, pl.outer) ||
        (reinterpret_cast<uintptr_t>(workspace) & 255))
      return SB_ERR_WORKSPACE;
    const size_t rows = (size_t)total_q * tree->n_q_heads;
    p.part_o = static_cast<float*>(workspace);
    p.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                          (((size_t)pl.outer * rows * D * sizeof(float) + 255) & ~(size_t)255));
  }
  const dim3 grid(p.num_splits, pl.grid_tiles * kv->n_kv_heads, kv->batch);
  if (grid.y > 65535) return SB_ERR_UNSUPPORTED;
  p.sort_seqs = kv->batch > 1 && kv->batch <= SB_MAX_NODES &&
                (long long)grid.x * grid.y * grid.z > (pl.tc ? 1LL : 2LL) * device_sms() ? 1 : 0;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const sb_status ls = pl.tc ? launch_quant_tc(p, grid, cs) : launch_quant_rows(p, grid, pl.cluster, device_sms(), cs);
  if (ls != SB_OK || pl.outer == 1) return ls;
  const int rows_max = tree->max_nodes * tree->n_q_heads;
  auto merge = [&](auto kernel, int rows_per_cta) {
    return launch_dependent(kernel, dim3(ceil_div(rows_max, rows_per_cta), kv->batch), dim3(256), cs, p);
  };
  if (pl.tc) return D == 64 ? merge(quant_merge_kernel<64, true>, 8 * 4) : merge(quant_merge_kernel<128, true>, 8 * 2);
  return D == 64 ? merge(quant_merge_kernel<64, false>, 8 * 2) : merge(quant_merge_kernel<128, false>, 8);
}
