// Pieces shared by the kernels of sb_tree_attention_quant: call parameters, per-sequence planning, visibility under a
// sliding window, and the list of key blocks that a sequence's nodes can see.
#pragma once

#include "quant_common.cuh"
#include "tc_common.cuh"

namespace sb {

struct QuantAttnParams {
  sb_quant_cache kv;
  const uint8_t* k_codes;  // the layer's
  const uint8_t* v_codes;
  const float* k_scale;
  const float* v_scale;
  sb_quant_tree tree;
  const bf16* k_nodes;
  const bf16* v_nodes;
  long long node_stride;
  const int* q_node_begin;
  const int* q_offsets;
  int total_q;
  const bf16* q;
  long long q_stride;
  bf16* out;
  float* lse;
  float scale_log2;
  int window, sinks;
  int num_splits;   // chunks of the key list per (sequence, KV head, row tile) = cluster size * outer
  int outer;        // clusters; > 1 needs the merge kernel
  float* part_o;    // [outer][total_q * Hq][D] normalised partial outputs (tcgen05 kernel: rows of kPartRow bytes)
  float* part_lse;  // [outer][total_q * Hq]    base-2 log-sum-exp of each
  int* status;
  int G;
  unsigned g_magic; // row / G = row * g_magic >> 20 for rows below 2^11
  int block_shift;  // log2 of the tokens per scale block
  int sort_seqs;    // 1: grid index z is the rank of a sequence by length, longest first
};

struct QuantSeq {
  int n, P, q0, q_off, nq, node_base;
  int err;
  bool can_write;  // the sequence's rows are inside q / out (zero-filled on an error)
};

__device__ inline QuantSeq load_quant_seq(const QuantAttnParams& p, int b) {
  QuantSeq s;
  const int o = p.tree.node_offsets[b];
  s.n = p.tree.node_offsets[b + 1] - o;
  s.P = p.tree.prefix_len[b];
  s.q0 = p.q_node_begin ? p.q_node_begin[b] : 0;
  s.q_off = p.q_offsets ? p.q_offsets[b] : o;
  s.nq = s.n - s.q0;
  s.node_base = o;
  s.err = 0;
  const bool tree_ok = s.n >= 0 && s.n <= p.tree.max_nodes && s.n <= SB_MAX_NODES && o >= 0 &&
                       (long long)o + s.n <= p.tree.total_nodes && s.q0 >= 0 && s.q0 <= s.n;
  const bool rows_ok = tree_ok && s.q_off >= 0 && (long long)s.q_off + s.nq <= p.total_q;
  const long long cap = p.kv.page_size == 0 ? p.kv.kv_capacity : (long long)p.kv.max_pages * p.kv.page_size;
  s.can_write = rows_ok;
  if (!tree_ok) s.err = SB_ERR_INVALID_TREE;
  else if (!rows_ok || s.P < 0 || s.P > p.tree.max_prefix || s.P > cap) s.err = SB_ERR_BOUNDS;
  if (!rows_ok) s.nq = 0;
  if (s.err) s.P = 0;
  return s;
}

// True when every page of the sequence's prefix is inside the pool.  Called by every thread of the group.
__device__ inline bool quant_pages_in_pool(const sb_quant_cache& kv, int b, int len, const ThreadGroup grp) {
  if (kv.page_size == 0) return true;
  __shared__ int s_bad_page;
  if (grp.tid == 0) s_bad_page = 0;
  grp.sync();
  const int need = (len + kv.page_size - 1) / kv.page_size;
  for (int i = grp.tid; i < need; i += grp.n) {
    const int page = kv.page_table[(long long)b * kv.max_pages + i];
    if (page < 0 || page >= kv.num_pages) s_bad_page = 1;
  }
  grp.sync();
  return s_bad_page == 0;
}

// The prefix blocks of `size` keys that some node of the sequence may see, as a list: `head` blocks from position 0
// (sinks), then the blocks from `tail` on (the window of a node at depth 0, which reaches back furthest).
struct BlockList {
  int head, tail, count;  // count = blocks in the list
  __device__ int at(int i) const { return i < head ? i : tail + (i - head); }
};
__device__ inline BlockList visible_blocks(int P, int window, int sinks, int size) {
  BlockList l;
  const int all = (P + size - 1) / size;
  l.head = 0;
  l.tail = 0;
  if (window > 0) {
    l.head = (min(sinks, P) + size - 1) / size;
    l.tail = max(l.head, max(0, P - window + 1) / size);
  }
  l.count = l.head + max(0, all - l.tail);
  return l;
}

// The prefix positions that no node of the sequence sees: [lo, hi), between the sinks and the window of a node at depth 0; empty
// without a window.  What a block of keys holds there may be anything, codes that are NaN included: V codes must not meet
// the zero probabilities.
struct UnseenKeys {
  int lo, hi;
  __device__ UnseenKeys(int P, int window, int sinks) : lo(sinks), hi(window > 0 ? P - window + 1 : 0) {}
  __device__ bool meets(int first, int last) const { return max(first, lo) < min(last, hi); }  // of the keys [first, last)
  __device__ bool has(int j) const { return j >= lo && j < hi; }
};

// Sequence with rank z by length, longest first (see sequence_of_rank in attention_common.cuh).  batch <= SB_MAX_NODES; s_len: 16-byte
// aligned scratch of SB_MAX_NODES ints, s_pick: one int.
__device__ inline int quant_sequence_of_rank(const QuantAttnParams& p, int z, int* s_len, int* s_pick) {
  const int B = p.kv.batch, tid = threadIdx.x;
  for (int i = tid; i < SB_MAX_NODES; i += blockDim.x) s_len[i] = i < B ? p.tree.prefix_len[i] : (int)0x80000000;
  __syncthreads();
  for (int i = tid; i < B; i += blockDim.x) {
    const int me = s_len[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < B; j += 4) {
      const int4 o = *reinterpret_cast<const int4*>(s_len + j);
      r += (o.x > me || (o.x == me && j < i)) + (o.y > me || (o.y == me && j + 1 < i)) + (o.z > me || (o.z == me && j + 2 < i)) +
           (o.w > me || (o.w == me && j + 3 < i));
    }
    if (r == z) *s_pick = i;
  }
  __syncthreads();
  const int b = *s_pick;
  __syncthreads();
  return b;
}

// A V scale as the kernels use it: tiny scales read as 2^-60 (their codes then count as zeros); NaN stays NaN.
constexpr float kMinVScale = 8.673617379884035e-19f;  // 2^-60
__device__ inline float v_scale_used(float s) { return s < kMinVScale ? kMinVScale : s; }

// bf16 magnitudes >= 0x7F80 are NaN or infinite
__device__ inline bool bf16x2_nonfinite(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Tensor maps of the codes: rank-4 view (d, KV head, row, page); a contiguous cache is one "page" of kv_capacity rows per sequence.  A box is
// one head's D bytes of *box_rows rows (a page's, at most `most`), swizzled by its row size.
template <int D>
inline sb_status make_code_maps(const QuantAttnParams& p, int most, CUtensorMap* kmap, CUtensorMap* vmap, int* box_rows) {
  *box_rows = p.kv.page_size == 0 || p.kv.page_size > most ? most : p.kv.page_size;
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return SB_ERR_CUDA;
  const uint8_t* codes[2] = {p.k_codes, p.v_codes};
  for (int i = 0; i < 2; ++i) {
    const cuuint64_t H = (cuuint64_t)p.kv.n_kv_heads, rows = (cuuint64_t)(p.kv.page_size == 0 ? p.kv.kv_capacity : p.kv.page_size);
    const cuuint64_t dims[4] = {(cuuint64_t)D, H, rows, (cuuint64_t)(p.kv.page_size == 0 ? p.kv.batch : p.kv.num_pages)};
    const cuuint64_t strides[3] = {(cuuint64_t)D, H * D, rows * H * D};
    const cuuint32_t box[4] = {(cuuint32_t)D, 1, (cuuint32_t)*box_rows, 1}, elem[4] = {1, 1, 1, 1};
    if (enc(i ? vmap : kmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t*>(codes[i]), dims, strides, box, elem,
            CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return SB_ERR_UNSUPPORTED;  // an extent or stride beyond what a tensor map holds
  }
  return SB_OK;
}

// Bytes of a partial row of the tcgen05 kernel: fp16 values, and the exponent of every eight of them (16 bytes; value = fp16 *
// 2^(exponent - 141)).
template <int D>
constexpr int kPartRow = 2 * D + 16;
constexpr int kQuantMaxCluster = 8;
sb_status launch_quant_rows(const QuantAttnParams& p, dim3 grid, int cluster, int sms, cudaStream_t cs);
sb_status launch_quant_tc(const QuantAttnParams& p, dim3 grid, cudaStream_t cs);

}  // namespace sb
