// Tree attention over an 8-bit prefix for few query rows (decoding, small trees): 16 packed (node, head) rows per CTA.
//
// The cost is the stream of codes: 2 D bytes per key and head.  At most 16 rows share it, far too few for a
// 128-row tcgen05 tile (its operands would have to be converted and written back to shared memory first, which
// costs more shared-memory traffic than the stream itself).  Here the codes go straight from a
// cp.async ring into the register fragments of mma.sync m16n8k16 and are converted there, two at a time.
//
// Each of the 4 warps owns every fourth group of 32 keys of the CTA's chunk and a ring of its own, so the main
// loop has no CTA barrier.  A contraction does not care for the order of its terms, so the fragments are defined by what
// one thread can load in 16 bytes (thread = 4 g + c of the fragment layouts):
//   S = Q K^T : thread (g, c) holds 16-byte chunks c and c + 4 of key row(g), and Q has the same order of d;
//   O = P V   : thread (g, c) holds chunk of column group g of the keys whose probabilities it already has, and
//               pairs bytes of two keys with one byte permutation; its output columns are 16 (or 2 x 16) in a row.
// Rows of the ring are XOR-swizzled by 16-byte chunks so that both access patterns are free of bank conflicts (D = 128).
//
// Scales: a K scale multiplies the scores of its 16 or more keys; a V scale s enters the exponent: the running reference is the
// maximum of score + log2 s, P' = 2^(score + log2 s - reference) goes into the product with the plain codes, and
// the denominator sums P' / s.  So no element of the stream is scaled, and P' is at most 1 for any mix of scales.
//
// Chunks of one tile are merged inside a cluster through distributed shared memory (up to 8), further clusters by
// quant_merge_kernel.
#include "quant_attention.cuh"

namespace sb {

constexpr int QR_WARPS = 4;
constexpr int QR_THREADS = QR_WARPS * 32;
constexpr int QR_ROWS = 16;
constexpr int QR_GROUP = 32;   // keys per warp step
constexpr int QR_STAGES = 3;

template <int D>
struct QrLayout {
  static constexpr int STAGE = QR_GROUP * D * 2;                       // K then V codes
  static constexpr int RING = QR_WARPS * QR_STAGES * STAGE;
  static constexpr int RS = D + 8;                                     // floats per staged row
  static constexpr int MERGE_ROWS = QR_ROWS + 8;                       // S * ceil(16 / S) <= 23 slots for S <= 8
  static constexpr int MERGE = MERGE_ROWS * RS * 4 + 2 * MERGE_ROWS * 4;
  static constexpr int BYTES = RING + MERGE;
};

__device__ inline void cp_async16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0));
}
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

template <int D>
__global__ void __launch_bounds__(QR_THREADS, 2) quant_rows_kernel(const QuantAttnParams p) {
  typedef QrLayout<D> L;
  constexpr int KS = D / 16;    // k steps of S = Q K^T
  constexpr int NT = D / 8;     // column tiles of O
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_parent[SB_MAX_NODES];
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
  pdl_wait();
  pdl_release();
  const int b = p.sort_seqs ? quant_sequence_of_rank(p, blockIdx.z, s_parent, s_depth) : (int)blockIdx.z;
  const QuantSeq si = load_quant_seq(p, b);
  const int rows_total = si.nq * G;
  const bool designated = split == 0 && blockIdx.y == 0;
  if (!si.can_write || row0 >= rows_total) {  // the same for all CTAs of a cluster
    if (designated) {
      const bool pages_ok = si.err ? true : quant_pages_in_pool(p.kv, b, si.P, whole_cta());
      if (tid == 0) p.status[b] = si.err ? si.err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
    }
    return;
  }

  // the key list: groups of prefix keys that some node sees, then groups of nodes; cut into num_splits chunks
  const BlockList list = visible_blocks(si.P, p.window, p.sinks, QR_GROUP);
  const int total = si.err ? 0 : list.count + ceil_div(si.n, QR_GROUP);
  const int per = total / p.num_splits, rem = total % p.num_splits;
  const int chunk0 = split * per + min(split, rem);
  const int chunk_n = per + (split < rem ? 1 : 0);
  const int mine = chunk_n > warp ? (chunk_n - warp + QR_WARPS - 1) / QR_WARPS : 0;  // groups of this warp
  auto group_at = [&](int i) { return chunk0 + warp + i * QR_WARPS; };               // position in the list

  const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + warp * (QR_STAGES * L::STAGE);
  // Row of the cache where each 16-key half of a group starts (both inside one page).  Halves past the prefix start at a
  // row that exists; they are not loaded.
  long long half_row[2];
  auto lookup = [&](int i) {
    half_row[0] = half_row[1] = 0;
    if (i >= mine) return;
    const int at = group_at(i);
    if (at >= list.count) return;
    const int k0 = list.at(at) * QR_GROUP;
    half_row[0] = quant_row(p.kv, b, k0);
    half_row[1] = k0 + 16 < si.P ? quant_row(p.kv, b, k0 + 16) : half_row[0];
  };
  auto issue = [&](int i) {
    if (i < mine && group_at(i) < list.count) {
      const int k0 = list.at(group_at(i)) * QR_GROUP;
      const uint32_t stage = ring + (i % QR_STAGES) * L::STAGE;
      constexpr int CPR = D / 16;            // chunks per row
      constexpr int RPI = 32 / CPR;          // rows per step of the warp
      const int ch = lane % CPR, r_in = lane / CPR;
      const long long step = (long long)Hkv * D;
#pragma unroll
      for (int s = 0; s < QR_GROUP / RPI; ++s) {
        const int r = s * RPI + r_in;
        const bool on = k0 + r < si.P && SB_CHECKED_ACCESS(half_row[r >> 4] + (r & 15), quant_rows_total(p.kv), &p.status[b]);
        const long long off = on ? (half_row[r >> 4] + (r & 15)) * step + g * D + ch * 16 : 0;
        cp_async16(stage + code_off<D>(r, ch), p.k_codes + off, on);
        cp_async16(stage + QR_GROUP * D + code_off<D>(r, ch), p.v_codes + off, on);
      }
      if (lane < 4) {
        const int h = lane & 1;
        const long long off = ((h == 0 ? half_row[0] : half_row[1]) >> p.block_shift) * Hkv + g;
        const float* src = (lane < 2 ? p.k_scale : p.v_scale) + off;
        const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(&s_scale[warp][i % QR_STAGES][lane]));
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src));
      }
    }
    asm volatile("cp.async.commit_group;\n" ::);
  };
  // the first groups are requested before anything else: they need the lengths only
#pragma unroll
  for (int i = 0; i < QR_STAGES - 1; ++i) {
    lookup(i);
    issue(i);
  }
  lookup(QR_STAGES - 1);

  // Q fragments: rows fg and fg + 8, scaled by a power of two per row into the middle of fp16's range (bf16 has fewer bits of
  // significand, so nothing is rounded but elements 2^-14 and more below the row's largest).
  const bf16* qrow[2];
  bool row_on[2];
  int node[2];
  float qscale[2];
  uint32_t qa[KS][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int R = row0 + fg + 8 * h;
    row_on[h] = R < rows_total;
    const int nl = row_on[h] ? R / G : 0, hh = row_on[h] ? R - nl * G : 0;
    node[h] = si.q0 + nl;
    row_on[h] = row_on[h] && SB_CHECKED_ACCESS(si.q_off + nl, p.total_q, &p.status[b]);
    qrow[h] = p.q + (long long)(si.q_off + nl) * p.q_stride + (long long)(g * G + hh) * D;
    uint32_t w[D / 8];
    load_row_share<D>(w, qrow[h], fc, row_on[h]);
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) amax = max(amax, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const int ex = (int)(amax >> 7);  // biased exponent
    const int e = ex == 0 || ex == 255 ? 127 : min(ex, 253);
    qscale[h] = __uint_as_float((uint32_t)e << 23) * p.scale_log2;
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const uint32_t v = pack_half(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xFFFF0000u) * inv);
      qa[i >> 1][(i & 1) * 2 + h] = v;
    }
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
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  // Scores a[t][e] (base 2, V scale folded in, masked to -inf) of four 8-key tiles -> probabilities; rescales what was
  // accumulated when a row's reference grows.
  auto softmax_step = [&](float (&a)[4][4], const float (&inv_v)[2]) {
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      top[0] = max3(top[0], a[t][0], a[t][1]);
      top[1] = max3(top[1], a[t][2], a[t][3]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
    }
    const bool grow = top[0] > m[0] || top[1] > m[1];
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float mn = fmaxf(m[h], top[h]);
        const float f = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - mn);  // nothing was accumulated before
        l[h] *= f;
        m[h] = mn;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          o[t][2 * h] *= f;
          o[t][2 * h + 1] *= f;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float ref = m[h] == -INFINITY ? 0.f : m[h];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float sum = 0.f;
#pragma unroll
        for (int t = 2 * u; t < 2 * u + 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float pr = fast_exp2(a[t][2 * h + e] - ref);
            a[t][2 * h + e] = pr;
            sum += pr;
          }
        if (sum != 0.f) l[h] = fmaf(sum, inv_v[u], l[h]);  // a NaN scale must not meet an empty half
      }
    }
  };

  for (int i = 0; i < mine; ++i) {
    const int at = group_at(i);
    if (at >= list.count) break;  // the rest are node groups
    asm volatile("cp.async.wait_group %0;\n" ::"n"(QR_STAGES - 2) : "memory");
    __syncwarp();
    issue(i + QR_STAGES - 1);     // into the stage that the previous step has finished with
    lookup(i + QR_STAGES);
    const int k0 = list.at(at) * QR_GROUP;
    const uint32_t stage = ring + (i % QR_STAGES) * L::STAGE;
    float a[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = 0.f;
      const int r = 8 * t + key_of_col<D>(fg);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const uint4 w4 = lds128(stage + code_off<D>(r, fc + 4 * h));
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_f16(a[t], qa[4 * h + k], half2_of_e4m3x2((uint16_t)w[k]), half2_of_e4m3x2((uint16_t)(w[k] >> 16)));
      }
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
    const bool all_seen = k0 + QR_GROUP <= si.P &&
                          (p.window == 0 || k0 + QR_GROUP <= p.sinks || si.P + si.n - 1 - k0 < p.window);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1;
        a[t][e] = fmaf(a[t][e], qscale[h] * ks[t >> 1], lsv[t >> 1]);
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
    __syncwarp();
  }
  asm volatile("cp.async.wait_group 0;\n" ::: "memory");

  // ---- node groups: bf16 rows, straight from global memory, bf16 products --------------------------------------------
  if (compute && mine > 0 && group_at(mine - 1) >= list.count) {
    uint32_t qb[KS][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[D / 8];
      load_row_share<D>(w, qrow[h], fc, row_on[h]);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) qb[i >> 1][(i & 1) * 2 + h] = w[i];
    }
    float qs[2] = {p.scale_log2, p.scale_log2};
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      const int at = group_at(i);
      if (at < list.count) continue;
      const int n0 = (at - list.count) * QR_GROUP;
      uint32_t bad = 0;  // keys (bit per key of the group) with a NaN or an infinity
      float a[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[t][e] = 0.f;
        const int nd = n0 + 8 * t + key_of_col<D>(fg);
        const bool on = nd < si.n && SB_CHECKED_ACCESS(si.node_base + nd, p.tree.total_nodes, &p.status[b]);
        uint32_t w[D / 8];
        load_row_share<D>(w, p.k_nodes + (long long)(si.node_base + (on ? nd : 0)) * p.node_stride + g * D, fc, on);
        bool nf = false;
#pragma unroll
        for (int k = 0; k < D / 8; ++k) nf |= bf16x2_nonfinite(w[k]);
        if (nf) bad |= 1u << (8 * t + key_of_col<D>(fg));
#pragma unroll
        for (int k = 0; k < KS; ++k) mma_bf16(a[t], qb[k], w[2 * k], w[2 * k + 1]);
      }
      // V rows of the keys whose probabilities this thread holds: keys of columns 2c and 2c + 1 of each tile
      auto v_row = [&](int t, int x, uint32_t (&w)[NT / 2]) {
        const int kk = 8 * t + key_of_col<D>(2 * fc + x), nd = n0 + kk;
        const bool on = nd < si.n && SB_CHECKED_ACCESS(si.node_base + nd, p.tree.total_nodes, &p.status[b]);
        const bf16* src = p.v_nodes + (long long)(si.node_base + (on ? nd : 0)) * p.node_stride + g * D +
                          (D == 128 ? ((fg >> 1) | ((fg & 1) << 2)) * 16 : fg * 8);
#pragma unroll
        for (int k = 0; k < NT / 8; ++k) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (on) v = *reinterpret_cast<const uint4*>(src + k * 8);
          w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
        }
        bool nf = false;
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) nf |= bf16x2_nonfinite(w[k]);
        return nf;
      };
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t w[NT / 2];
          if (v_row(t, x, w)) bad |= 1u << (8 * t + key_of_col<D>(2 * fc + x));
        }
      bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int h = e >> 1, kk = 8 * t + key_of_col<D>(2 * fc + (e & 1)), nd = n0 + kk;
          bool seen = nd < si.n && row_on[h] && ((s_anc[4 * node[h] + (nd >> 5)] >> (nd & 31)) & 1u);
          if (seen && p.window > 0) {
            const int kp = si.P + s_depth[nd];
            seen = kp < p.sinks || pos[h] - kp < p.window;
          }
          a[t][e] = seen ? (((bad >> kk) & 1u) ? __uint_as_float(0x7FC00000u) : a[t][e] * qs[h]) : -INFINITY;
        }
      const float one[2] = {1.f, 1.f};
      softmax_step(a, one);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t pa[4] = {pack_bf16(a[2 * u][0], a[2 * u][1]), pack_bf16(a[2 * u][2], a[2 * u][3]),
                                pack_bf16(a[2 * u + 1][0], a[2 * u + 1][1]), pack_bf16(a[2 * u + 1][2], a[2 * u + 1][3])};
        uint32_t w[4][NT / 2];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          v_row(2 * u + (x >> 1), x & 1, w[x]);
          // a bad row counts through its NaN probability; its elements must not meet the zeros of other rows
          if ((bad >> (16 * u + 8 * (x >> 1) + key_of_col<D>(2 * fc + (x & 1)))) & 1u)
#pragma unroll
            for (int k = 0; k < NT / 2; ++k) w[x][k] = 0;
        }
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) {
          mma_bf16(o[2 * k], pa, __byte_perm(w[0][k], w[1][k], 0x5410), __byte_perm(w[2][k], w[3][k], 0x5410));
          mma_bf16(o[2 * k + 1], pa, __byte_perm(w[0][k], w[1][k], 0x7632), __byte_perm(w[2][k], w[3][k], 0x7632));
        }
      }
    }
  }

  // ---- merge the warps, then the chunks of the cluster ----------------------------------------------------------------
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
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
  float* red = reinterpret_cast<float*>(smem + L::RING);            // [S * rows_per][RS]
  float* red_m = red + L::MERGE_ROWS * L::RS;
  float* red_l = red_m + L::MERGE_ROWS;
  const long long rows_all = (long long)p.total_q * Hq;
  auto store = [&](int r, int c4, float4 acc, float M, float Lsum, int outer_idx) {
    const int R = row0 + r;
    if (R >= rows_total) return;
    const int nl = R / G;
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
  if (S > 1) cluster.sync();  // every CTA of the cluster has started: its shared memory may be written
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
    float M = -INFINITY;
    for (int c = 0; c < S; ++c) M = fmaxf(M, red_m[c * rows_per + t]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float Lsum = 0.f;
    for (int c = 0; c < S; ++c) {
      const float wt = weight_of(red_m[c * rows_per + t], M);
      const float4 v = *reinterpret_cast<const float4*>(red + (c * rows_per + t) * L::RS + c4 * 4);
      acc.x += wt * v.x; acc.y += wt * v.y; acc.z += wt * v.z; acc.w += wt * v.w;
      Lsum += wt * red_l[c * rows_per + t];
    }
    store(r_begin + t, c4, acc, M, Lsum, split / S);
  }
}

template <int D>
static sb_status launch_rows(const QuantAttnParams& p, dim3 grid, int cluster, cudaStream_t cs) {
  static PerDeviceOnce once;
  if (!once.run([]() {
        const bool ok = cudaFuncSetAttribute(quant_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             QrLayout<D>::BYTES) == cudaSuccess;
        if (!ok) cudaGetLastError();
        return ok;
      }))
    return SB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(QR_THREADS);
  cfg.dynamicSmemBytes = QrLayout<D>::BYTES;
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
  if (cudaLaunchKernelEx(&cfg, quant_rows_kernel<D>, p) != cudaSuccess) {
    cudaGetLastError();
    return SB_ERR_CUDA;
  }
  return launch_check();
}

sb_status launch_quant_rows(const QuantAttnParams& p, dim3 grid, int cluster, cudaStream_t cs) {
  return p.kv.head_dim == 64 ? launch_rows<64>(p, grid, cluster, cs) : launch_rows<128>(p, grid, cluster, cs);
}

}  // namespace sb
