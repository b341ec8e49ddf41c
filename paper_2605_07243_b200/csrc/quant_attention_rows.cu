// Tree attention over an 8-bit prefix for few query rows (decoding, small trees): 16 packed (node, head) rows per CTA.
//
// The cost is the stream of codes: 2 D bytes per key and head.  At most 16 rows share it, far too few for a
// 128-row tcgen05 tile (its operands would have to be converted and written back to shared memory first, which
// costs more shared-memory traffic than the stream itself).  Here the codes go straight from a
// TMA-filled ring into the register fragments of mma.sync m16n8k16 and are converted there, two at a time.  (mma.sync on the
// codes themselves, with Q as two e4m3 terms, was slower: 191 against 150 us on a batch of 64 sequences of 4k tokens.)
//
// Each of the 4 warps owns every fourth group of 32 keys of the CTA's chunk and a ring of two groups, which one lane
// refills (address arithmetic of cp.async in every lane was a fifth of the instructions), so the main loop has no CTA
// barrier.  Three CTAs fit on an SM: 12 warps, each of which waits most of the time, keep up to 192 KB under way.  A contraction does not care for the order of its terms, so the fragments are defined by what
// one thread can load in 16 bytes (thread = 4 g + c of the fragment layouts):
//   S = Q K^T : thread (g, c) holds 16-byte chunks c and c + 4 of key row(g), and Q has the same order of d;
//   O = P V   : thread (g, c) holds chunk of column group g of the keys whose probabilities it already has, and
//               pairs bytes of two keys with one byte permutation; its output columns are 16 (or 2 x 16) in a row.
// TMA swizzles the rows of the ring by 16-byte chunks, which makes both access patterns free of bank conflicts (D = 128).
//
// Scales: a K scale multiplies the scores of its 16 or more keys; a V scale s enters the exponent: P' = 2^(score + log2 s -
// reference) goes into the product with the plain codes, and the denominator sums P' / s.  So no element of the stream is
// scaled.  The reference of a row is its largest exponent of the first keys that it sees and is raised only when a sum
// shows that an exponent lies far above it, so that the common step needs no maximum and no shuffle.
//
// The tree's nodes come first in the key list, in groups of 16 bf16 rows that go straight from global memory into bf16 products:
// the first codes are on their way meanwhile.
//
// Chunks of one tile are merged inside a cluster through distributed shared memory (up to 8), further clusters by
// quant_merge_kernel.
#include "quant_attention.cuh"

namespace sb {

constexpr int QR_WARPS = 4;
constexpr int QR_THREADS = QR_WARPS * 32;
constexpr int QR_ROWS = 16;
constexpr int QR_GROUP = 32;   // keys per warp step
constexpr int QR_NODES = 16;   // nodes per warp step
constexpr int QR_STAGES = 2;

template <int D>
struct QrLayout {
  static constexpr int STAGE = QR_GROUP * D * 2;                       // K then V codes
  static constexpr int RING = QR_WARPS * QR_STAGES * STAGE;
  static constexpr int RS = D + 8;                                     // floats per staged row
  static constexpr int MERGE_ROWS = QR_ROWS + 8;                       // S * ceil(16 / S) <= 23 slots for S <= 8
  static constexpr int MERGE = MERGE_ROWS * RS * 4 + 2 * MERGE_ROWS * 4;
  // Where the cluster's merge buffer lies: behind the rings, or, to fit a third CTA on the SM, over them (behind the warps' staged
  // rows), which then costs a wait for the cluster's slowest main loop.
  static constexpr int MERGE_OVER = 40 * 1024;
  static constexpr int BYTES_APART = 1024 + RING + MERGE;
  static constexpr int BYTES_OVER = 1024 + (RING > MERGE_OVER + MERGE ? RING : MERGE_OVER + MERGE);
};

__device__ inline uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ inline uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ inline void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ inline void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ inline uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ inline float weight_of(float m, float M) { return m == -INFINITY ? 0.f : fast_exp2(m - M); }

// Byte offset of 16-byte chunk `ch` of row `r` in a [32][D] code tile.
template <int D>
__device__ inline uint32_t code_off(int r, int ch) {
  return (uint32_t)(r * D + ((ch ^ (D == 128 ? (r & 7) : ((r >> 1) & 3))) << 4));
}
// Key (within 8) that column n of a score tile stands for.  D = 128: columns n and n + 1 are rows 4 apart, whose chunks
// c and c ^ 4 fall into different banks.  D = 64: neighbouring rows share a bank line already.
template <int D>
__device__ inline int key_of_col(int n) {
  return D == 128 ? ((n >> 1) | ((n & 1) << 2)) : n;
}

// This thread's share of one bf16 row: D / 4 elements in the fragment order, as D / 8 words.
template <int D>
__device__ inline void load_row_share(uint32_t (&w)[D / 8], const bf16* row, int c, bool on) {
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (on) v = *reinterpret_cast<const uint4*>(row + (h * 4 + c) * 16 + k * 8);
      w[h * 8 + k * 4 + 0] = v.x;
      w[h * 8 + k * 4 + 1] = v.y;
      w[h * 8 + k * 4 + 2] = v.z;
      w[h * 8 + k * 4 + 3] = v.w;
    }
}

// Zeros over the rows of a V tile (keys k0 .. k0 + 31) that no node sees, behind the prefix or before every window: what lies there (stale
// bytes, codes that are NaN) must not meet the zero probabilities.  One warp.
template <int D>
__device__ __forceinline__ void clear_unseen(uint32_t tile, int k0, int P, const UnseenKeys unseen, int lane) {
  for (int c = lane; c < QR_GROUP * (D / 16); c += 32) {
    const int j = k0 + c / (D / 16);
    if (j >= P || unseen.has(j)) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(tile + c * 16), "r"(0) : "memory");
  }
  fence_async_smem();  // a later load into the stage comes after these writes
  __syncwarp();
}

template <int D>
__global__ void __launch_bounds__(QR_THREADS, 3) quant_rows_kernel(const QuantAttnParams p, const __grid_constant__ CUtensorMap kmap,
                                                                   const __grid_constant__ CUtensorMap vmap, const int box_rows,
                                                                   const int merge_apart) {
  typedef QrLayout<D> L;
  constexpr int KS = D / 16;    // k steps of S = Q K^T
  constexpr int NT = D / 8;     // column tiles of O
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t s_full[QR_WARPS][QR_STAGES];
  __shared__ int s_abort, s_late;                    // a wait gave up; the same for the waits after that
  __shared__ int s_page[QR_WARPS][4][2];             // ids of the pages of the two halves of coming groups
  __shared__ __align__(16) int s_parent[SB_MAX_NODES];
  __shared__ uint32_t s_anc[SB_MAX_NODES * 4];
  __shared__ int s_depth[SB_MAX_NODES];
  __shared__ float s_scale[QR_WARPS][QR_STAGES][4];  // K, K, V, V scale of the two 16-key halves of a group
  __shared__ float s_m[QR_WARPS][QR_ROWS], s_l[QR_WARPS][QR_ROWS];

  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, fg = lane >> 2, fc = lane & 3;
  const int split = blockIdx.x;
  const int S = (int)cluster.num_blocks(), crank = (int)cluster.block_rank();
  const int Hq = p.tree.n_q_heads, Hkv = p.kv.n_kv_heads, G = p.G;
  const int g = blockIdx.y % Hkv, row0 = (blockIdx.y / Hkv) * QR_ROWS;
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap));
    s_abort = s_late = 0;
    for (int i = 0; i < QR_WARPS * QR_STAGES; ++i) mbar_init(&s_full[0][0] + i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (S > 1 && merge_apart) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // this CTA has started
  pdl_wait();
  pdl_release();
  const int b = p.sort_seqs ? quant_sequence_of_rank(p, blockIdx.z, s_parent, s_depth) : (int)blockIdx.z;
  const QuantSeq si = load_quant_seq(p, b);
  const int rows_total = si.nq * G;
  const bool designated = split == 0 && blockIdx.y == 0;
  if (!si.can_write || row0 >= rows_total) {  // the same for all CTAs of a cluster
    if (S > 1 && merge_apart) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (designated) {
      const bool pages_ok = si.err ? true : quant_pages_in_pool(p.kv, b, si.P, whole_cta());
      if (tid == 0) p.status[b] = si.err ? si.err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
    }
    return;
  }

  // the key list: groups of nodes, then groups of prefix keys that some node sees; cut into num_splits chunks
  const BlockList list = visible_blocks(si.P, p.window, p.sinks, QR_GROUP);
  const int node_groups = si.err ? 0 : ceil_div(si.n, QR_NODES);
  const int total = si.err ? 0 : node_groups + list.count;
  const int per = total / p.num_splits, rem = total % p.num_splits;
  const int chunk0 = split * per + min(split, rem);
  const int chunk_n = per + (split < rem ? 1 : 0);
  // this warp's groups: list positions first, first + 4, ...; the first nodes_mine of them are nodes
  const int first = chunk0 + warp;
  const int mine = chunk_n > warp ? (chunk_n - warp + QR_WARPS - 1) / QR_WARPS : 0;
  const int nodes_mine = max(0, min(mine, (node_groups - first + QR_WARPS - 1) / QR_WARPS));
  const int codes_mine = mine - nodes_mine;
  auto code_key = [&](int i) { return list.at(first + (nodes_mine + i) * QR_WARPS - node_groups) * QR_GROUP; };  // first key of the i-th of codes
  const uint32_t ring = smem_u32(smem) + warp * (QR_STAGES * L::STAGE);
  // Lanes 0-3 look after a group's loads: lane & 1 is the 16-key half, lane >> 1 K or V; TMA boxes, scales, page ids.  An id is fetched two
  // groups ahead, into shared memory, so that nothing waits for it.
  const bool paged = p.kv.page_size != 0;
  const int page_shift = paged ? 31 - __clz(p.kv.page_size) : 31;
  const int* table = p.kv.page_table + (long long)b * p.kv.max_pages;
  auto my_key = [&](int i) { return code_key(i) + 16 * (lane & 1); };
  auto fetch_page = [&](int i) {  // -> s_page[i & 3]
    if (paged && lane < 2 && i < codes_mine && my_key(i) < si.P)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(smem_u32(&s_page[warp][i & 3][lane])), "l"(table + (my_key(i) >> page_shift)));
  };
  auto issue = [&](int i, int page) {
    if (i < codes_mine && lane < 4) {
      const int key = my_key(i), st = i % QR_STAGES;
      const bool on = key < si.P;
      if (page < 0 || page >= p.kv.num_pages) page = 0;  // reported by the designated CTA; reads stay in the pool
      const int in_page = paged ? key & (p.kv.page_size - 1) : key;
      const int boxes = box_rows >= QR_GROUP || key - 16 * (lane & 1) + 16 >= si.P ? 1 : 2;
      if (lane == 0) mbar_expect_tx(&s_full[warp][st], 2 * boxes * box_rows * D);
      __syncwarp(0xF);
      const uint32_t stage = ring + st * L::STAGE + (lane & 1) * 16 * D;
      if (on && (lane & 1) < boxes) {  // lanes 0, 1: K; lanes 2, 3: V
        const CUtensorMap* map = lane < 2 ? &kmap : &vmap;
        tma_load_4d(stage + (lane < 2 ? 0 : QR_GROUP * D), map, 0, g, in_page, paged ? page : b, &s_full[warp][st]);
      }
      const long long crow = on ? (paged ? (long long)page << page_shift : (long long)b * p.kv.kv_capacity) + in_page : -1;
      float* dst = &s_scale[warp][st][lane];
      if (on && SB_CHECKED_ACCESS(crow + 15, quant_rows_total(p.kv), &p.status[b]))
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(smem_u32(dst)),
                     "l"((lane < 2 ? p.k_scale : p.v_scale) + (crow >> p.block_shift) * Hkv + g));
      else
        *dst = 1.f;
    }
    fetch_page(i + 2);
    asm volatile("cp.async.commit_group;\n" ::);
  };
  // the first groups are requested before anything else: they need the lengths only
  {
    int first_pages[QR_STAGES];
#pragma unroll
    for (int i = 0; i < QR_STAGES; ++i)
      first_pages[i] = paged && lane < 4 && i < codes_mine && my_key(i) < si.P ? __ldg(table + (my_key(i) >> page_shift)) : 0;
#pragma unroll
    for (int i = 0; i < QR_STAGES; ++i) issue(i, first_pages[i]);
  }

  // Q fragments: rows fg and fg + 8, as they are (for the nodes)
  bool row_on[2];
  int node[2];
  uint32_t qa[KS][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int R = row0 + fg + 8 * h;
    row_on[h] = R < rows_total;
    const int nl = row_on[h] ? (int)((unsigned)R * p.g_magic >> 20) : 0, hh = row_on[h] ? R - nl * G : 0;
    node[h] = si.q0 + nl;
    row_on[h] = row_on[h] && SB_CHECKED_ACCESS(si.q_off + nl, p.total_q, &p.status[b]);
    uint32_t w[D / 8];
    load_row_share<D>(w, p.q + (long long)(si.q_off + nl) * p.q_stride + (g * G + hh) * D, fc, row_on[h]);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) qa[i >> 1][(i & 1) * 2 + h] = w[i];
  }

  const bool tree_ok = build_ancestors_smem(p.tree.parent + si.node_base, si.err ? 0 : si.n, s_parent, s_anc, s_depth);
  int err = si.err;
  if (!err && !tree_ok) err = SB_ERR_INVALID_TREE;
  if (designated) {
    const bool pages_ok = err ? true : quant_pages_in_pool(p.kv, b, si.P, whole_cta());
    if (tid == 0) p.status[b] = err ? err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);  // reported; reads stay in the pool
  }
  const bool compute = err == 0;
  int pos[2];  // position of each row's node
#pragma unroll
  for (int h = 0; h < 2; ++h) pos[h] = si.P + (compute && row_on[h] ? s_depth[node[h]] : 0);

  float o[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[t][e] = 0.f;
  float ref[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};   // l: this thread's part of the row
  bool seen_any[2] = {false, false};               // the row has met a visible key, and `ref` is its reference

  // Exponents a[t][e] of two or four 8-key tiles (base 2, V scale folded in, relative to the reference, masked to -inf) -> probabilities.
  auto softmax_step = [&](auto& a, const float (&inv_v)[2]) {  // inv_v: of the two halves of the tiles
    constexpr int T = (int)(sizeof(a) / sizeof(a[0]));
    bool raise = !(seen_any[0] && seen_any[1]);
    float pr[T][4], sum[2][2];
    while (true) {
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float top = fmaxf(a[0][2 * h], a[0][2 * h + 1]);
#pragma unroll
          for (int t = 1; t < T; ++t) top = max3(top, a[t][2 * h], a[t][2 * h + 1]);
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          // the same in the four threads of a row
          const float delta = (seen_any[h] ? top > 0.f : top > -INFINITY) ? top : 0.f;
          const float f = seen_any[h] ? fast_exp2(-delta) : 1.f;  // nothing accumulated yet: nothing to scale
          seen_any[h] |= top > -INFINITY;
          ref[h] += delta;
          l[h] *= f;
#pragma unroll
          for (int t = 0; t < T; ++t) {
            a[t][2 * h] -= delta;
            a[t][2 * h + 1] -= delta;
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            o[t][2 * h] *= f;
            o[t][2 * h + 1] *= f;
          }
        }
      }
      raise = false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[h][0] = sum[h][1] = 0.f;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            pr[t][2 * h + e] = fast_exp2(a[t][2 * h + e]);
            sum[h][t * 2 / T] += pr[t][2 * h + e];
          }
        raise |= sum[h][0] + sum[h][1] > 2048.f;  // of at most 8 probabilities: an exponent above 8 (fp16 ends at 2^16)
      }
      if (!__any_sync(0xffffffffu, raise)) break;
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = pr[t][e];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (sum[h][u] != 0.f) l[h] = fmaf(sum[h][u], inv_v[u], l[h]);  // a NaN scale must not meet an empty half
  };

  // ---- nodes -------------------------------------------------------------------------------------------------------------
#pragma unroll 1
  for (int i = 0; i < (compute ? nodes_mine : 0); ++i) {
    const int n0 = (first + i * QR_WARPS) * QR_NODES;
    uint32_t kw[2][D / 8], vw[4][NT / 2];  // V: keys of columns 2c, 2c + 1 of the two tiles
    auto row_at = [&](const bf16* rows, int nd) { return rows + (long long)(si.node_base + (nd < si.n ? nd : 0)) * p.node_stride + g * D; };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int nd = n0 + 8 * t + key_of_col<D>(fg);
      load_row_share<D>(kw[t], row_at(p.k_nodes, nd), fc, nd < si.n);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int nd = n0 + 8 * (x >> 1) + key_of_col<D>(2 * fc + (x & 1));
      const bf16* src = row_at(p.v_nodes, nd) + (D == 128 ? ((fg >> 1) | ((fg & 1) << 2)) * 16 : fg * 8);
#pragma unroll
      for (int k = 0; k < NT / 8; ++k) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (nd < si.n) v = *reinterpret_cast<const uint4*>(src + k * 8);
        vw[x][4 * k] = v.x; vw[x][4 * k + 1] = v.y; vw[x][4 * k + 2] = v.z; vw[x][4 * k + 3] = v.w;
      }
    }
    float a[2][4];
    uint32_t bad = 0;  // nodes (bit per node of the group) with a NaN or an infinity
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      bool nf = false;
#pragma unroll
      for (int k = 0; k < D / 8; ++k) nf |= bf16x2_nonfinite(kw[t][k]);
      if (nf) bad |= 1u << (8 * t + key_of_col<D>(fg));
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) mma_bf16(a[t], qa[k], kw[t][2 * k], kw[t][2 * k + 1]);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      bool nf = false;
#pragma unroll
      for (int k = 0; k < NT / 2; ++k) nf |= bf16x2_nonfinite(vw[x][k]);
      if (nf) bad |= 1u << (8 * (x >> 1) + key_of_col<D>(2 * fc + (x & 1)));
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1, kk = 8 * t + key_of_col<D>(2 * fc + (e & 1)), nd = n0 + kk;
        bool seen = nd < si.n && row_on[h] && ((s_anc[4 * node[h] + (nd >> 5)] >> (nd & 31)) & 1u);
        if (seen && p.window > 0) {
          const int kp = si.P + s_depth[nd];
          seen = kp < p.sinks || pos[h] - kp < p.window;
        }
        a[t][e] = seen ? (((bad >> kk) & 1u) ? __uint_as_float(0x7FC00000u) : fmaf(a[t][e], p.scale_log2, -ref[h])) : -INFINITY;
      }
    const float one[2] = {1.f, 1.f};
    softmax_step(a, one);
    const uint32_t pa[4] = {pack_bf16(a[0][0], a[0][1]), pack_bf16(a[0][2], a[0][3]), pack_bf16(a[1][0], a[1][1]), pack_bf16(a[1][2], a[1][3])};
    // a bad row counts through its NaN probability; its elements must not meet the zeros of other rows
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if ((bad >> (8 * (x >> 1) + key_of_col<D>(2 * fc + (x & 1)))) & 1u)
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) vw[x][k] = 0;
#pragma unroll
    for (int k = 0; k < NT / 2; ++k) {
      mma_bf16(o[2 * k], pa, __byte_perm(vw[0][k], vw[1][k], 0x5410), __byte_perm(vw[2][k], vw[3][k], 0x5410));
      mma_bf16(o[2 * k + 1], pa, __byte_perm(vw[0][k], vw[1][k], 0x7632), __byte_perm(vw[2][k], vw[3][k], 0x7632));
    }
  }

  // ---- codes -------------------------------------------------------------------------------------------------------------
  // Q scaled by a power of two per row into the middle of fp16's range (bf16 has fewer bits of significand, so nothing is rounded
  // but elements 2^-21 and more below the row's largest).
  float qscale[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t amax = 0;
#pragma unroll
    for (int k = 0; k < KS; ++k) amax = __vmaxu2(amax, __vmaxu2(qa[k][h] & 0x7FFF7FFFu, qa[k][2 + h] & 0x7FFF7FFFu));
    amax = __vmaxu2(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = __vmaxu2(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const int ex = (int)(max(amax & 0xFFFFu, amax >> 16) >> 7);  // biased exponent
    const int e = ex == 255 ? 127 : min(max(ex - 7, 1), 253);    // the largest element becomes 2^7 .. 2^8
    qscale[h] = ex == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)e << 23) * p.scale_log2;  // NaN row: NaN throughout
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        qa[k][2 * x + h] = pack_half(__uint_as_float(qa[k][2 * x + h] << 16) * inv, __uint_as_float(qa[k][2 * x + h] & 0xFFFF0000u) * inv);
  }
  // A reference that comes from nodes knows nothing of the V scale that the codes' exponents contain: with small values (of 2^-7: scale
  // 2^-15) the fp16 probabilities of the prefix would lie that far below it.  It goes down by the scale of the first codes.
  if (nodes_mine > 0 && codes_mine > 0) {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(QR_STAGES - 1) : "memory");
    __syncwarp();
    const float down = fminf(__log2f(v_scale_used(fminf(s_scale[warp][0][2], s_scale[warp][0][3]))), 0.f);
    const float f = fast_exp2(-down);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ref[h] += down;
      l[h] *= f;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] *= f;
  }
  bool ok = true;
  for (int i = 0; i < codes_mine; ++i) {
    const int k0 = code_key(i);
    const uint32_t stage = ring + (i % QR_STAGES) * L::STAGE;
    if (ok) ok = mbar_wait(&s_full[warp][i % QR_STAGES], (i / QR_STAGES) & 1, &s_abort);
    asm volatile("cp.async.wait_group %0;\n" ::"n"(QR_STAGES - 1) : "memory");
    __syncwarp();
    const bool all_seen = k0 + QR_GROUP <= si.P &&
                          (p.window == 0 || k0 + QR_GROUP <= p.sinks || si.P + si.n - 1 - k0 < p.window);
    if (!all_seen) clear_unseen<D>(stage + QR_GROUP * D, k0, si.P, UnseenKeys(si.P, p.window, p.sinks), lane);
    float a[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = 0.f;
    // two tiles at a time, their products interleaved: a tile's own eight form a chain
#pragma unroll
    for (int t = 0; t < 4; t += 2) {
      uint32_t w[2][D / 16];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint4 v = lds128(stage + code_off<D>(8 * (t + x) + key_of_col<D>(fg), fc + 4 * h));
          w[x][4 * h] = v.x; w[x][4 * h + 1] = v.y; w[x][4 * h + 2] = v.z; w[x][4 * h + 3] = v.w;
        }
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          mma_f16(a[t + x], qa[k], half2_of_e4m3x2((uint16_t)w[x][k]), half2_of_e4m3x2((uint16_t)(w[x][k] >> 16)));
    }
    float lsv[2], inv_v[2], ks[2];
    bool v_tiny = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ks[u] = s_scale[warp][i % QR_STAGES][u];
      const float raw = s_scale[warp][i % QR_STAGES][2 + u];
      v_tiny |= raw < kMinVScale;
      const float sv = v_scale_used(raw);
      lsv[u] = __log2f(sv);
      inv_v[u] = __fdividef(1.f, sv);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1;
        a[t][e] = fmaf(a[t][e], qscale[h] * ks[t >> 1], lsv[t >> 1] - ref[h]);
        if (!all_seen) {
          const int j = k0 + 8 * t + key_of_col<D>(2 * fc + (e & 1));
          const bool seen = j < si.P && (p.window == 0 || j < p.sinks || pos[h] - j < p.window);
          if (!seen) a[t][e] = -INFINITY;
        }
      }
    softmax_step(a, inv_v);
    if (v_tiny) {  // a V block that reads as zeros (rare): its probabilities only enter the denominator
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (s_scale[warp][i % QR_STAGES][2 + (t >> 1)] < kMinVScale)
#pragma unroll
          for (int e = 0; e < 4; ++e) a[t][e] = 0.f;
    }
    const uint32_t vst = stage + QR_GROUP * D;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t pa[4] = {pack_half(a[2 * u][0], a[2 * u][1]), pack_half(a[2 * u][2], a[2 * u][3]),
                              pack_half(a[2 * u + 1][0], a[2 * u + 1][1]), pack_half(a[2 * u + 1][2], a[2 * u + 1][3])};
      uint32_t w[4][NT / 4];  // keys of columns 2c, 2c + 1 of the two tiles
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int r = 16 * u + 8 * (x >> 1) + key_of_col<D>(2 * fc + (x & 1));
        if (D == 128) {
          const uint4 v = lds128(vst + code_off<D>(r, (fg >> 1) | ((fg & 1) << 2)));
          w[x][0] = v.x; w[x][1] = v.y; w[x][NT / 4 - 2] = v.z; w[x][NT / 4 - 1] = v.w;
        } else {
          const uint2 v = lds64(vst + code_off<D>(r, fg >> 1) + (fg & 1) * 8);
          w[x][0] = v.x; w[x][1] = v.y;
        }
      }
#pragma unroll
      for (int k = 0; k < NT / 4; ++k) {
        const uint32_t lo0 = __byte_perm(w[0][k], w[1][k], 0x5140), lo1 = __byte_perm(w[0][k], w[1][k], 0x7362);
        const uint32_t hi0 = __byte_perm(w[2][k], w[3][k], 0x5140), hi1 = __byte_perm(w[2][k], w[3][k], 0x7362);
        mma_f16(o[4 * k + 0], pa, half2_of_e4m3x2((uint16_t)lo0), half2_of_e4m3x2((uint16_t)hi0));
        mma_f16(o[4 * k + 1], pa, half2_of_e4m3x2((uint16_t)(lo0 >> 16)), half2_of_e4m3x2((uint16_t)(hi0 >> 16)));
        mma_f16(o[4 * k + 2], pa, half2_of_e4m3x2((uint16_t)lo1), half2_of_e4m3x2((uint16_t)hi1));
        mma_f16(o[4 * k + 3], pa, half2_of_e4m3x2((uint16_t)(lo1 >> 16)), half2_of_e4m3x2((uint16_t)(hi1 >> 16)));
      }
    }
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) {  // nothing more is asked for; what is in flight is awaited, again with a limit, before shared memory has another use
      for (int k = i; k < min(i + QR_STAGES, codes_mine); ++k) mbar_wait(&s_full[warp][k % QR_STAGES], (k / QR_STAGES) & 1, &s_late);
      break;
    }
    issue(i + QR_STAGES, paged && lane < 4 ? s_page[warp][(i + QR_STAGES) & 3][lane & 1] : 0);
  }
  asm volatile("cp.async.wait_group 0;\n" ::: "memory");
  if (!ok) atomicMax(&p.status[b], (int)SB_ERR_CUDA);

  // ---- merge the warps, then the chunks of the cluster ----------------------------------------------------------------
  float m[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    m[h] = seen_any[h] ? ref[h] : -INFINITY;
    if (l[h] != l[h]) m[h] = INFINITY;  // a NaN outweighs every other chunk
    if (!compute) {
      l[h] = 0.f;
      m[h] = -INFINITY;
    }
  }
  __syncthreads();  // the rings are idle
  float* stage_o = reinterpret_cast<float*>(smem) + warp * (QR_ROWS * L::RS);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float* dst = stage_o + (fg + 8 * h) * L::RS;
#pragma unroll
    for (int t = 0; t < NT; t += 4) {
      // D = 128: columns 16 c + t and 16 (c + 4) + t; D = 64: columns 16 c + t and 16 c + 8 + t
      const int c0 = 16 * fc + t, c1 = c0 + (D == 128 ? 64 : 8);
      *reinterpret_cast<float4*>(dst + c0) = make_float4(o[t][2 * h], o[t + 1][2 * h], o[t + 2][2 * h], o[t + 3][2 * h]);
      *reinterpret_cast<float4*>(dst + c1) =
          make_float4(o[t][2 * h + 1], o[t + 1][2 * h + 1], o[t + 2][2 * h + 1], o[t + 3][2 * h + 1]);
    }
    if (fc == 0) {
      s_m[warp][fg + 8 * h] = m[h];
      s_l[warp][fg + 8 * h] = l[h];
    }
  }
  __syncthreads();

  const int rows_per = ceil_div(QR_ROWS, S);
  float* red = reinterpret_cast<float*>(smem + (merge_apart ? L::RING : L::MERGE_OVER));   // [S * rows_per][RS]
  float* red_m = red + L::MERGE_ROWS * L::RS;
  float* red_l = red_m + L::MERGE_ROWS;
  const long long rows_all = (long long)p.total_q * Hq;
  auto store = [&](int r, int c4, float4 acc, float M, float Lsum, int outer_idx) {
    const int R = row0 + r;
    if (R >= rows_total) return;
    const int nl = (int)((unsigned)R * p.g_magic >> 20);
    const long long grow = (long long)(si.q_off + nl) * Hq + g * G + (R - nl * G);
    if (!SB_CHECKED_ACCESS(grow, rows_all, &p.status[b])) return;
    const float inv = Lsum == 0.f ? 0.f : 1.f / Lsum;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    const float lse2 = Lsum == 0.f ? -INFINITY : M + log2f(Lsum);
    if (p.outer == 1) {
      uint2 packed;
      packed.x = pack_bf16(acc.x, acc.y);
      packed.y = pack_bf16(acc.z, acc.w);
      *reinterpret_cast<uint2*>(p.out + grow * D + c4 * 4) = packed;
      if (p.lse && c4 == 0) p.lse[grow] = Lsum == 0.f ? 0.f : lse2 * kLn2;
    } else {
      *reinterpret_cast<float4*>(p.part_o + (outer_idx * rows_all + grow) * D + c4 * 4) = acc;
      if (c4 == 0) p.part_lse[outer_idx * rows_all + grow] = lse2;
    }
  };
  if (S > 1) {
    if (merge_apart) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA of the cluster has started,
    else cluster.sync();                                                           // or is done with its rings
  }
#pragma unroll
  for (int idx = tid; idx < QR_ROWS * (D / 4); idx += QR_THREADS) {
    const int r = idx / (D / 4), c4 = idx % (D / 4);
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < QR_WARPS; ++w) M = fmaxf(M, s_m[w][r]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float Lsum = 0.f;
#pragma unroll
    for (int w = 0; w < QR_WARPS; ++w) {
      const float wt = weight_of(s_m[w][r], M);
      const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * QR_ROWS + r) * L::RS + c4 * 4);
      acc.x += wt * v.x; acc.y += wt * v.y; acc.z += wt * v.z; acc.w += wt * v.w;
      Lsum += wt * s_l[w][r];
    }
    if (S == 1) {
      store(r, c4, acc, M, Lsum, split);
    } else {
      const int owner = r / rows_per, slot = crank * rows_per + (r - owner * rows_per);
      *reinterpret_cast<float4*>(cluster.map_shared_rank(red, owner) + slot * L::RS + c4 * 4) = acc;
      if (c4 == 0) {
        cluster.map_shared_rank(red_m, owner)[slot] = M;
        cluster.map_shared_rank(red_l, owner)[slot] = Lsum;
      }
    }
  }
  if (S == 1) return;
  cluster.sync();
  const int r_begin = crank * rows_per, n_rows = max(0, min(QR_ROWS, r_begin + rows_per) - r_begin);
  for (int idx = tid; idx < n_rows * (D / 4); idx += QR_THREADS) {
    const int t = idx / (D / 4), c4 = idx % (D / 4);
    float mc[kQuantMaxCluster], M = -INFINITY;
#pragma unroll
    for (int c = 0; c < kQuantMaxCluster; ++c) {
      mc[c] = c < S ? red_m[c * rows_per + t] : -INFINITY;
      M = fmaxf(M, mc[c]);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float Lsum = 0.f;
#pragma unroll
    for (int c = 0; c < kQuantMaxCluster; ++c)
      if (c < S) {
        const float wt = weight_of(mc[c], M);
        const float4 v = *reinterpret_cast<const float4*>(red + (c * rows_per + t) * L::RS + c4 * 4);
        acc.x += wt * v.x; acc.y += wt * v.y; acc.z += wt * v.z; acc.w += wt * v.w;
        Lsum += wt * red_l[c * rows_per + t];
      }
    store(r_begin + t, c4, acc, M, Lsum, split / S);
  }
}

template <int D>
static sb_status launch_rows(const QuantAttnParams& p, dim3 grid, int cluster, int sms, cudaStream_t cs) {
  static PerDeviceOnce once;
  if (!once.run([]() {
        const bool ok = cudaFuncSetAttribute(quant_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             QrLayout<D>::BYTES_APART > QrLayout<D>::BYTES_OVER ? QrLayout<D>::BYTES_APART
                                                                                                : QrLayout<D>::BYTES_OVER) == cudaSuccess;
        if (!ok) cudaGetLastError();
        return ok;
      }))
    return SB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(QR_THREADS);
  // a merge buffer of its own costs the third CTA of an SM: only where two to an SM are enough
  const int merge_apart = cluster > 1 && (long long)grid.x * grid.y * grid.z <= 2LL * sms ? 1 : 0;
  cfg.dynamicSmemBytes = merge_apart ? QrLayout<D>::BYTES_APART : QrLayout<D>::BYTES_OVER;
  cfg.stream = cs;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  CUtensorMap kmap, vmap;
  int box_rows;
  const sb_status ms = make_code_maps<D>(p, QR_GROUP, &kmap, &vmap, &box_rows);
  if (ms != SB_OK) return ms;
  if (cudaLaunchKernelEx(&cfg, quant_rows_kernel<D>, p, kmap, vmap, box_rows, merge_apart) != cudaSuccess) {
    cudaGetLastError();
    return SB_ERR_CUDA;
  }
  return launch_check();
}

sb_status launch_quant_rows(const QuantAttnParams& p, dim3 grid, int cluster, int sms, cudaStream_t cs) {
  return p.kv.head_dim == 64 ? launch_rows<64>(p, grid, cluster, sms, cs) : launch_rows<128>(p, grid, cluster, sms, cs);
}

}  // namespace sb
