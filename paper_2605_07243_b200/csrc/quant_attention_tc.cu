// Tree attention over an 8-bit prefix on the tensor cores (tcgen05 + TMEM, sm_100a), for tiles of 128 packed rows.
//
// tcgen05 takes operands of one width only, and Q and P would lose what bf16 outputs need as e4m3.  So the codes become
// fp16 on their way into shared memory (exact: every e4m3 value is an fp16 value): four converter warps load 16
// codes per thread from global memory, convert them in registers and store them in the operand layout.  The
// next block's codes wait in registers meanwhile, so global latency hides behind the conversion of the present one,
// and shared memory holds fp16 tiles only (two of K, two of V).
// Scales never touch an element of the stream: a K scale multiplies the scores of its 16 or more columns, a V scale enters the
// exponent (P' = 2^(s + log2 v - reference), denominator sum P' / v), which the fused multiply-add that forms
// the exponent does for nothing.  Q is scaled per row by a power of two into fp16's range.
//
// A CTA owns one KV head's chunk of the key list and two "streams" t = 0, 1, each with its own score buffer and
// accumulator in tensor memory (2 x 128 + 2 x D columns) and its own softmax warpgroup with one thread per row:
//   two row tiles (mode A): stream t is tile t, every key block is used twice;
//   one row tile (mode B): stream t takes every second key block; the two accumulators are merged at the end.
// The first thread of a stream's warpgroup issues its MMAs, O += P_n V then S_{n+1} = Q K^T, when the warpgroup has
// written P_n: it has nothing else to do until S_{n+1} is there, and the tensor pipe works for one stream while
// the other stream's threads compute exponentials.  MMAs of one thread complete in order, so a completed S_{n+1} also means
// that P_n has been read and the accumulator holds it.  (No warp of its own for the issue: 12 warps leave
// 168 registers a thread, 13 would leave 128, and the scores would spill.)
//
// The softmax thread walks its row's 128 scores in quarters of 32 columns, the next quarter's load in flight.  The
// reference is raised only when a score exceeds it by 2^8 (P' is fp16: up to 2^15 would do), a rare event that rescales
// the accumulator and the quarters already written; so the maximum of a whole block is never needed first.
//
// Prefix blocks come from the window's block list (128 keys); the tree's nodes are one last block of their own, whose bf16
// rows are brought into fp16 by a power of two per 16 rows, as if they were codes.
#include "quant_attention.cuh"
#include "tc_common.cuh"

namespace sb {

constexpr int QT_SOFTMAX = 256;       // warps 0-3: stream 0, warps 4-7: stream 1
constexpr int QT_CVT_WARP = 8;        // warps 8-11; warp 8 also owns the tensor memory allocation
constexpr int QT_THREADS = 384;
constexpr int QT_TMEM_COLS = 512;
constexpr int QT_SMALL = 8192;
constexpr float kQuantStep = 8.f;     // the reference follows the maximum in steps of at least 2^8

enum QtBar { QB_K_FULL0, QB_K_FULL1, QB_K_EMPTY0, QB_K_EMPTY1, QB_V_FULL0, QB_V_FULL1, QB_V_EMPTY0, QB_V_EMPTY1,
             QB_S_FULL0, QB_S_FULL1, QB_SC0, QB_SC1, QB_SC2, QB_SC3, QB_O_DONE0, QB_O_DONE1, QB_COUNT };

template <int D>
constexpr int quant_tc_smem() { return 1024 + QT_SMALL + 6 * TC_BM * D * 2; }

__device__ inline uint32_t tc_idesc_f16(int M, int N, int b_mn_major) {
  return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ inline uint32_t low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
__device__ inline uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// 32 columns without the wait
__device__ inline void tmem_ld32_async(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// The wait names the registers that the load fills: the compiler must not move their uses above it.
__device__ inline void tmem_wait_ld(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

template <int D>
__global__ void __launch_bounds__(QT_THREADS, 1) quant_tc_kernel(const QuantAttnParams p) {
  constexpr int TILE = TC_BN * D * 2;   // one fp16 tile of 128 rows
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint32_t* s_anc = reinterpret_cast<uint32_t*>(base);               // 2048 B
  int* s_parent = reinterpret_cast<int*>(base + 2048);               // 512 B
  int* s_depth = reinterpret_cast<int*>(base + 2560);                // 512 B
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(base + 3072);        // QB_COUNT * 8
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(base + 3328);
  volatile int* s_abort = reinterpret_cast<volatile int*>(base + 3332);   // [0] a wait gave up; [1] the same for the last wait
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(base + 3344);          // [4]: node rows with a NaN or an infinity
  float* s_ks = reinterpret_cast<float*>(base + 3392);               // [4 slots][8 groups of 16 keys] K scale
  float* s_lsv = s_ks + 32;                                          // log2 of the V scale
  float* s_isv = s_lsv + 32;                                         // 1 / V scale
  float* s_qs = reinterpret_cast<float*>(base + 3840);               // [256 rows] scale of a Q row
  float* s_ml = reinterpret_cast<float*>(base + 4864);               // [2][128] reference and sum of stream 1 (mode B)
  uint8_t* sQ = base + QT_SMALL;
  uint8_t* sK = sQ + 2 * TILE;
  uint8_t* sV = sK + 2 * TILE;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = blockIdx.x;
  const int Hq = p.tree.n_q_heads, Hkv = p.kv.n_kv_heads, G = p.G;
  if (warp == QT_CVT_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(QT_TMEM_COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  pdl_release();

  const int pairs = (int)gridDim.y / Hkv;
  const int g = blockIdx.y / pairs, pair = blockIdx.y % pairs;   // the pairs of a KV head are neighbours: they share its codes in L2
  const int b = p.sort_seqs ? quant_sequence_of_rank(p, blockIdx.z, reinterpret_cast<int*>(s_anc), s_parent) : (int)blockIdx.z;
  const QuantSeq si = load_quant_seq(p, b);
  const int rows_total = si.nq * G;
  const int row0 = pair * 2 * TC_BM;
  const bool designated = split == 0 && blockIdx.y == 0;
  if (!si.can_write || row0 >= rows_total) {
    if (designated) {
      const bool pages_ok = si.err ? true : quant_pages_in_pool(p.kv, b, si.P, whole_cta());
      if (tid == 0) p.status[b] = si.err ? si.err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
    }
    if (warp == QT_CVT_WARP)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*s_tmem), "r"(QT_TMEM_COLS));
    return;
  }
  const bool two = row0 + TC_BM < rows_total;   // mode A
  if (tid == 0) {
    s_abort[0] = s_abort[1] = 0;
    for (int i = 0; i < 4; ++i) s_bad[i] = 0;
    for (int i = 0; i < QB_COUNT; ++i) {
      const bool full = i == QB_K_FULL0 || i == QB_K_FULL1 || i == QB_V_FULL0 || i == QB_V_FULL1 || (i >= QB_SC0 && i <= QB_SC3);
      const bool empty = i == QB_K_EMPTY0 || i == QB_K_EMPTY1 || i == QB_V_EMPTY0 || i == QB_V_EMPTY1;
      mbar_init(&s_bar[i], full ? 4 : empty && two ? 2 : 1);  // a stage is free when its last reader, of one or two streams, is done
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const long long rows_all = (long long)p.total_q * Hq;

  const BlockList list = visible_blocks(si.P, p.window, p.sinks, TC_BN);
  const int total = si.err ? 0 : list.count + (si.n > 0 ? 1 : 0);   // the tree is the last block
  const int per = total / p.num_splits, rem = total % p.num_splits;
  const int blk0 = split * per + min(split, rem);
  const int nb = per + (split < rem ? 1 : 0);
  const int nv = two ? 2 * nb : nb;
  const uint32_t tmem = *s_tmem;
  const uint32_t tmem_o = tmem + 2 * TC_BN;

  // state of the softmax threads
  const int t_mine = warp >> 2, row = (warp & 3) * 32 + lane;
  const uint32_t lane_base = ((uint32_t)((warp & 3) * 32)) << 16;
  float ref = 0.f, l_run = 0.f;
  bool seen_any = false, ok = true, compute = false;

  if (tid < QT_SOFTMAX) {
    // ---- Q: 16-byte pieces, D / 8 lanes to a row ---------------------------------------------------------------
    constexpr int LPR = D / 8, RPP = QT_SOFTMAX / LPR;
    const int n_rows = two ? 2 * TC_BM : TC_BM;
#pragma unroll 4
    for (int r0 = 0; r0 < n_rows; r0 += RPP) {
      const int r = r0 + tid / LPR, ch = tid % LPR;
      const int R = row0 + r;
      const int nl = R / G;
      const bool on = R < rows_total && SB_CHECKED_ACCESS(si.q_off + nl, p.total_q, &p.status[b]);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (on) v = *reinterpret_cast<const uint4*>(p.q + (long long)(si.q_off + nl) * p.q_stride + (long long)(g * G + R - nl * G) * D + ch * 8);
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t amax = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) amax = max(amax, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
#pragma unroll
      for (int d = 1; d < LPR; d <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, d));
      const int ex = (int)(amax >> 7);
      const int e = ex == 0 || ex == 255 ? 127 : min(ex, 253);
      const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = pack_f16(__uint_as_float(w[k] << 16) * inv, __uint_as_float(w[k] & 0xFFFF0000u) * inv);
      *reinterpret_cast<uint4*>(sQ + (r / TC_BM) * TILE + sw128_chunk_off(r % TC_BM, ch, TC_BM)) = make_uint4(w[0], w[1], w[2], w[3]);
      if (ch == 0) s_qs[r] = __uint_as_float((uint32_t)e << 23) * p.scale_log2;
    }
    fence_async_smem();
    const ThreadGroup grp = first_threads(QT_SOFTMAX);
    const bool tree_ok = build_ancestors_smem(p.tree.parent + si.node_base, si.err ? 0 : si.n, s_parent, s_anc, s_depth, grp);
    int err = si.err;
    if (!err && !tree_ok) err = SB_ERR_INVALID_TREE;
    if (designated) {
      const bool pages_ok = err ? true : quant_pages_in_pool(p.kv, b, si.P, grp);
      if (tid == 0) p.status[b] = err ? err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
    }
    compute = err == 0;

    // ---- softmax --------------------------------------------------------------------------------------------------
    const int R = row0 + (two ? t_mine * TC_BM : 0) + row;
    const int node = (R < rows_total && compute) ? si.q0 + R / G : -1;
    const int pos = si.P + (node >= 0 ? s_depth[node] : 0);
    const float qs = s_qs[(two ? t_mine * TC_BM : 0) + row];
    const uint32_t s_addr = tmem + lane_base + t_mine * TC_BN;
    bool poison = false;

    const bool leader = (tid & 127) == 0;     // issues the MMAs of its stream
    const uint32_t hi = tc_desc_hi(1024);
    const uint32_t q_lo = tc_desc_lo(smem_u32(sQ) + (two ? t_mine * TILE : 0), 16), k_lo = tc_desc_lo(smem_u32(sK), 16);
    const uint32_t v_lo = tc_desc_lo(smem_u32(sV), TC_BN * 128);
    auto issue_s = [&](int n) {               // S of this stream's n-th block
      const int j = two ? n : 2 * n + t_mine;
      if (ok) ok = mbar_wait(&s_bar[QB_K_FULL0 + (j & 1)], (j >> 1) & 1, s_abort);
      if (!ok) return;
      tc_fence_after();
      const uint32_t kb = k_lo + (j & 1) * (TILE >> 4), idesc = tc_idesc_f16(TC_BM, TC_BN, 0);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const uint32_t koff = ((ks >> 2) * (TC_BM * 128) + (ks & 3) * 32) >> 4;
        tc_mma_h(tmem + t_mine * TC_BN, q_lo + koff, kb + koff, hi, idesc, ks > 0);
      }
      tc_commit(&s_bar[QB_S_FULL0 + t_mine]);
      tc_commit(&s_bar[QB_K_EMPTY0 + (j & 1)]);
    };
    auto issue_pv = [&](int n) {
      const int j = two ? n : 2 * n + t_mine;
      if (ok) ok = mbar_wait(&s_bar[QB_V_FULL0 + (j & 1)], (j >> 1) & 1, s_abort);
      if (!ok) return;
      tc_fence_after();
      const uint32_t vb = v_lo + (j & 1) * (TILE >> 4), pb = tmem + t_mine * TC_BN, idesc = tc_idesc_f16(TC_BM, D, 1);
#pragma unroll
      for (int ks = 0; ks < TC_BN / 16; ++ks)
        tc_mma_ts_h(tmem_o + t_mine * D, pb + ks * 8, vb + ks * (2048 >> 4), hi, idesc, (n > 0 || ks > 0) ? 1u : 0u);
      tc_commit(&s_bar[QB_V_EMPTY0 + (j & 1)]);
    };
    const int my_blocks = nv > t_mine ? (nv - t_mine + 1) / 2 : 0;
    if (leader && my_blocks > 0) issue_s(0);
    // A wait that gives up leaves `ok` false; the loop still runs to its end, so that the warpgroup's barriers match.
    for (int n = 0; n < my_blocks; ++n) {
      const int v = 2 * n + t_mine;
      const int j = two ? n : v;
      const int at = blk0 + j, slot = (j & 3) * 8;
      const bool is_tree = at >= list.count;
      const int k0 = is_tree ? 0 : list.at(at) * TC_BN;
      // blocks that every row sees whole need no mask
      const bool masked = is_tree || k0 + TC_BN > si.P ||
                          (p.window > 0 && k0 + TC_BN > p.sinks && si.P + si.n - 1 - k0 >= p.window);
      if (ok) ok = mbar_wait(&s_bar[QB_SC0 + (j & 3)], (j >> 2) & 1, s_abort) && mbar_wait(&s_bar[QB_S_FULL0 + t_mine], n & 1, s_abort);
      __syncwarp();
      tc_fence_after();
      uint32_t sr[2][32];
      tmem_ld32_async(s_addr, sr[0]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t(&x)[32] = sr[q & 1];
        tmem_wait_ld(x);
        if (q < 3) tmem_ld32_async(s_addr + 32 * (q + 1), sr[(q + 1) & 1]);
        const float2 ks = *reinterpret_cast<const float2*>(s_ks + slot + 2 * q);
        const float2 lsv = *reinterpret_cast<const float2*>(s_lsv + slot + 2 * q);
        const float2 isv = *reinterpret_cast<const float2*>(s_isv + slot + 2 * q);
        // exponents relative to the present reference
        const float f0 = qs * ks.x, f1 = qs * ks.y, c0 = lsv.x - ref, c1 = lsv.y - ref;
        unsigned long long mul[2] = {pack_f32x2(f0, f0), pack_f32x2(f1, f1)}, add[2] = {pack_f32x2(c0, c0), pack_f32x2(c1, c1)};
        float d[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2)
          unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), mul[i >> 4], add[i >> 4]), d[i], d[i + 1]);
        if (masked) {
          uint32_t word;
          if (is_tree) {
            word = node >= 0 ? s_anc[4 * node + q] : 0u;
            if (p.window > 0) {
              for (uint32_t w = word; w; w &= w - 1) {
                const int bit = __ffs(w) - 1, kp = si.P + s_depth[32 * q + bit];
                if (!(kp < p.sinks || pos - kp < p.window)) word &= ~(1u << bit);
              }
            }
            poison |= (word & s_bad[q]) != 0;
          } else {
            const int kq = k0 + 32 * q;
            word = low_bits(si.P - kq);
            if (p.window > 0) word &= low_bits(p.sinks - kq) | ~low_bits(pos - p.window + 1 - kq);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!((word >> i) & 1u)) d[i] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 32; i += 2) top = max3(top, d[i], d[i + 1]);
        const bool step = seen_any ? top > kQuantStep : top > -INFINITY;
        if (__any_sync(0xffffffffu, step)) {
          const float delta = step ? top : 0.f;
          const float factor = step && seen_any ? fast_exp2(-delta) : 1.f;
#pragma unroll
          for (int i = 0; i < 32; ++i) d[i] -= delta;
          ref += delta;
          l_run *= factor;
          seen_any |= step;
          if (n > 0) {  // PV of this stream's previous block is complete (see above)
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t r[16];
              tmem_ld16(tmem_o + t_mine * D + lane_base + c * 16, r);
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * factor);
              tmem_st16(tmem_o + t_mine * D + lane_base + c * 16, r);
            }
          }
          if (q > 0) tmem_wait_st();  // the quarters already written are read back
#pragma unroll 1
          for (int c = 0; c < q; ++c) {
            uint32_t r[16];
            tmem_ld16(s_addr + 16 * c, r);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r[i]));
              r[i] = pack_f16(f.x * factor, f.y * factor);
            }
            tmem_st16(s_addr + 16 * c, r);
          }
          tmem_wait_st();
        }
        uint32_t pk[16];
        unsigned long long sum2[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          const float p0 = fast_exp2(d[i]), p1 = fast_exp2(d[i + 1]);
          sum2[i >> 4] = add_f32x2(sum2[i >> 4], pack_f32x2(p0, p1));
          pk[i >> 1] = pack_f16(p0, p1);
        }
        float a0, a1, b0, b1;
        unpack_f32x2(sum2[0], a0, a1);
        unpack_f32x2(sum2[1], b0, b1);
        a0 += a1;
        b0 += b1;
        if (a0 != 0.f) l_run = fmaf(a0, isv.x, l_run);  // a NaN scale must not meet an empty group
        if (b0 != 0.f) l_run = fmaf(b0, isv.y, l_run);
        tmem_st16(s_addr + 16 * q, pk);
      }
      tmem_wait_st();
      tc_fence_before();
      asm volatile("bar.sync %0, 128;" ::"r"(2 + t_mine) : "memory");
      if (leader) {
        issue_pv(n);
        if (n + 1 < my_blocks) issue_s(n + 1);
      }
      __syncwarp();
    }
    if (leader) tc_commit(&s_bar[QB_O_DONE0 + t_mine]);
    if (!ok) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
    if (poison) l_run = __uint_as_float(0x7FC00000u);
    if (!compute) {
      l_run = 0.f;
      seen_any = false;
    }
  } else {
    // ---- converters ---------------------------------------------------------------------------------------------------
    const int cw = warp - QT_CVT_WARP;          // rows [32 cw, 32 cw + 32) of every block
    constexpr int CPR = D / 16, RPI = 32 / CPR, NI = 32 / RPI;
    const int ch = lane % CPR, r_in = lane / CPR;
    const long long width = (long long)Hkv * D;
    long long half_row[2] = {0, 0};             // cache rows of this warp's two 16-key halves, of the block looked up last
    int k0 = 0;
    float ks_raw = 1.f, vs_raw = 1.f;           // lanes 0 and 1: scales of half `lane` of the block loaded last
    bool v_zero[2] = {false, false};
    uint4 kx[NI], vx[NI];
    auto lookup = [&](int j) {
      if (j >= nb || blk0 + j >= list.count) return;
      k0 = list.at(blk0 + j) * TC_BN + 32 * cw;
      half_row[0] = k0 < si.P ? quant_row(p.kv, b, k0) : 0;
      half_row[1] = k0 + 16 < si.P ? quant_row(p.kv, b, k0 + 16) : 0;
    };
    auto load = [&](const uint8_t* codes, uint4 (&x)[NI]) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int r = i * RPI + r_in;
        const long long crow = (i * RPI < 16 ? half_row[0] : half_row[1]) + (r & 15);
        x[i] = make_uint4(0, 0, 0, 0);
        if (k0 + r < si.P && SB_CHECKED_ACCESS(crow, quant_rows_total(p.kv), &p.status[b]))
          x[i] = __ldg(reinterpret_cast<const uint4*>(codes + crow * width + g * D + ch * 16));
      }
    };
    auto load_scales = [&]() {
      ks_raw = vs_raw = 1.f;
      if (lane < 2 && k0 + 16 * lane < si.P) {
        const long long off = (lane == 0 ? half_row[0] : half_row[1]) / p.kv.scale_block * Hkv + g;
        ks_raw = p.k_scale[off];
        vs_raw = p.v_scale[off];
      }
    };
    auto store_pair = [&](uint8_t* stage, int r, const uint4 (&h)[2]) {
      // Two 16-byte chunks of one row.  D = 128: the lanes of a row's upper half, whose tile repeats the banks of the lower
      // one, store them in the other order.
      const bool swap = D == 128 && (lane & 4);
      const uint4 a = swap ? h[1] : h[0], b2 = swap ? h[0] : h[1];
      *reinterpret_cast<uint4*>(stage + sw128_chunk_off(r, 2 * ch + (swap ? 1 : 0), TC_BN)) = a;
      *reinterpret_cast<uint4*>(stage + sw128_chunk_off(r, 2 * ch + (swap ? 0 : 1), TC_BN)) = b2;
    };
    auto convert = [&](uint8_t* stage, const uint4 (&x)[NI], bool z0, bool z1) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const bool z = i * RPI < 16 ? z0 : z1;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint32_t h[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          h[2 * k] = z ? 0u : half2_of_e4m3x2((uint16_t)w[k]);
          h[2 * k + 1] = z ? 0u : half2_of_e4m3x2((uint16_t)(w[k] >> 16));
        }
        const uint4 o[2] = {make_uint4(h[0], h[1], h[2], h[3]), make_uint4(h[4], h[5], h[6], h[7])};
        store_pair(stage, 32 * cw + i * RPI + r_in, o);
      }
    };
    auto put_scales = [&](int j, float ks, float vs) {
      const int at = (j & 3) * 8 + 2 * cw + lane;
      s_ks[at] = ks;
      s_lsv[at] = log2f(vs);
      s_isv[at] = 1.f / vs;
    };
    auto publish = [&](uint64_t* bar) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    // The tree: bf16 rows -> fp16 with a power of two per 16 rows.  Rows that hold a NaN or an infinity become zeros.
    auto node_rows = [&](const bf16* src, int half, uint4 (&x)[NI]) {  // x: this lane's 16 elements of NI / 2 rows
#pragma unroll
      for (int i = 0; i < NI / 2; ++i) {
        const int nd = 32 * cw + 16 * half + i * RPI + r_in;
        x[2 * i] = x[2 * i + 1] = make_uint4(0, 0, 0, 0);
        if (nd < si.n && SB_CHECKED_ACCESS(si.node_base + nd, p.tree.total_nodes, &p.status[b])) {
          const uint4* s4 = reinterpret_cast<const uint4*>(src + (long long)(si.node_base + nd) * p.node_stride + g * D + ch * 16);
          x[2 * i] = s4[0];
          x[2 * i + 1] = s4[1];
        }
      }
    };
    auto bad_rows = [&](uint4 (&x)[NI], int half) {  // bits (row of the warp) of rows with a NaN or an infinity, which are zeroed
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < NI / 2; ++i) {
        const uint32_t w[8] = {x[2 * i].x, x[2 * i].y, x[2 * i].z, x[2 * i].w, x[2 * i + 1].x, x[2 * i + 1].y, x[2 * i + 1].z, x[2 * i + 1].w};
        bool nf = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) nf |= bf16x2_nonfinite(w[k]);
        const uint32_t votes = __ballot_sync(0xffffffffu, nf);
        const uint32_t mine = (votes >> (r_in * CPR)) & ((1u << CPR) - 1u);
        if (mine) x[2 * i] = x[2 * i + 1] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < RPI; ++r)
          if ((votes >> (r * CPR)) & ((1u << CPR) - 1u)) bits |= 1u << (16 * half + i * RPI + r);
      }
      return bits;
    };
    auto node_convert = [&](const bf16* src, uint8_t* stage, float (&scale)[2], bool is_v) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint4 x[NI];
        node_rows(src, half, x);
        bad_rows(x, half);
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) amax = max(amax, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        int e = (int)(amax >> 7) - 8;              // biased exponent of the scale: the largest value becomes 2^8 .. 2^9
        e = amax < 0x80u ? 127 : max(e, is_v ? 127 - 60 : 1);
        e = min(e, 253);
        scale[half] = __uint_as_float((uint32_t)e << 23);
        const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
        for (int i = 0; i < NI / 2; ++i) {
          uint4 o[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint4 v = x[2 * i + k];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t h[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) h[c] = pack_f16(__uint_as_float(w[c] << 16) * inv, __uint_as_float(w[c] & 0xFFFF0000u) * inv);
            o[k] = make_uint4(h[0], h[1], h[2], h[3]);
          }
          store_pair(stage, 32 * cw + 16 * half + i * RPI + r_in, o);
        }
      }
    };
    auto is_prefix = [&](int j) { return j < nb && blk0 + j < list.count; };
    lookup(0);
    if (is_prefix(0)) {
      load(p.k_codes, kx);
      load_scales();
      load(p.v_codes, vx);
    }
    for (int j = 0; j < nb && ok; ++j) {
      uint8_t* ks_stage = sK + (j & 1) * TILE;
      uint8_t* vs_stage = sV + (j & 1) * TILE;
      const bool prefix = is_prefix(j);
      const float ks = ks_raw, vs = vs_raw;
      lookup(j + 1);
      if (j >= 2) ok = mbar_wait(&s_bar[QB_K_EMPTY0 + (j & 1)], ((j >> 1) - 1) & 1, s_abort);
      if (!ok) break;
      if (prefix) {
        const uint32_t tiny = __ballot_sync(0xffffffffu, vs < kMinVScale);
        v_zero[0] = tiny & 1;
        v_zero[1] = (tiny >> 1) & 1;
        if (lane < 2) put_scales(j, ks, v_scale_used(vs));
        convert(ks_stage, kx, false, false);
        publish(&s_bar[QB_K_FULL0 + (j & 1)]);
        if (lane == 0) mbar_arrive(&s_bar[QB_SC0 + (j & 3)]);
        if (is_prefix(j + 1)) {
          load(p.k_codes, kx);
          load_scales();
        }
        if (j >= 2) ok = mbar_wait(&s_bar[QB_V_EMPTY0 + (j & 1)], ((j >> 1) - 1) & 1, s_abort);
        if (!ok) break;
        convert(vs_stage, vx, v_zero[0], v_zero[1]);
        publish(&s_bar[QB_V_FULL0 + (j & 1)]);
        if (is_prefix(j + 1)) load(p.v_codes, vx);
      } else {
        float kscale[2], vscale[2];
        uint32_t bits = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint4 x[NI];
          node_rows(p.k_nodes, half, x);
          bits |= bad_rows(x, half);
        }
        node_convert(p.k_nodes, ks_stage, kscale, false);
        if (j >= 2) ok = mbar_wait(&s_bar[QB_V_EMPTY0 + (j & 1)], ((j >> 1) - 1) & 1, s_abort);
        if (!ok) break;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint4 x[NI];
          node_rows(p.v_nodes, half, x);
          bits |= bad_rows(x, half);
        }
        node_convert(p.v_nodes, vs_stage, vscale, true);
        if (lane < 2) put_scales(j, lane == 0 ? kscale[0] : kscale[1], lane == 0 ? vscale[0] : vscale[1]);
        if (lane == 0) s_bad[cw] = bits;
        publish(&s_bar[QB_K_FULL0 + (j & 1)]);
        if (lane == 0) {
          mbar_arrive(&s_bar[QB_V_FULL0 + (j & 1)]);
          mbar_arrive(&s_bar[QB_SC0 + (j & 3)]);
        }
      }
    }
    if (!ok) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
  }

  // ---- store ----------------------------------------------------------------------------------------------------------
  // One thread per row: normalised by its own sum.  In mode B the second stream hands its row over in shared memory.
  const bool have = nb > 0;
  if (tid < QT_SOFTMAX) {
    // awaited even after a wait that gave up: tensor memory is idle before it is freed
    if (!mbar_wait(&s_bar[QB_O_DONE0 + t_mine], 0, s_abort + 1)) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
    __syncwarp();
    tc_fence_after();
    if (l_run != l_run) {  // a NaN outweighs everything it is merged with
      ref = INFINITY;
      seen_any = true;
    }
    const int streams = two ? 1 : (nv > 1 ? 2 : 1);   // accumulators per row
    constexpr int RS = D + 4;                         // floats per row handed over (over the idle K and V tiles)
    float* hand = reinterpret_cast<float*>(sK);
    softmax_group_sync();                             // the MMAs of both streams are done
    if (streams == 2 && t_mine == 1) {
#pragma unroll 1
      for (int c = 0; c < D / 16; ++c) {
        uint32_t r[16];
        tmem_ld16(tmem_o + D + lane_base + c * 16, r);
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<uint4*>(hand + row * RS + c * 16 + i) = make_uint4(r[i], r[i + 1], r[i + 2], r[i + 3]);
      }
      s_ml[row] = seen_any ? ref : -INFINITY;
      s_ml[128 + row] = l_run;
    }
    softmax_group_sync();
    if (two || t_mine == 0) {
      float m = seen_any ? ref : -INFINITY, w0 = 1.f, w1 = 0.f, l = l_run;
      if (streams == 2) {
        const float m1 = s_ml[row], l1 = s_ml[128 + row], M = fmaxf(m, m1);
        w0 = m == -INFINITY ? 0.f : fast_exp2(m - M);
        w1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - M);
        l = w0 * l + w1 * l1;
        m = M;
      }
      const int R = row0 + (two ? t_mine * TC_BM : 0) + row;
      const int nl = R / G;
      const long long grow = (long long)(si.q_off + nl) * Hq + g * G + (R - nl * G);
      const bool on = R < rows_total && SB_CHECKED_ACCESS(grow, rows_all, &p.status[b]);
      const bool empty = !have || l == 0.f;
      const float inv = empty ? 0.f : 1.f / l;
      w0 *= inv;
      w1 *= inv;
#pragma unroll 1
      for (int c = 0; c < D / 16; ++c) {
        float f[16];
        if (have) {
          uint32_t r[16];
          tmem_ld16(tmem_o + (two ? t_mine * D : 0) + lane_base + c * 16, r);
#pragma unroll
          for (int i = 0; i < 16; ++i) f[i] = w0 == 0.f ? 0.f : __uint_as_float(r[i]) * w0;
          if (streams == 2 && w1 != 0.f)
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = fmaf(hand[row * RS + c * 16 + i], w1, f[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) f[i] = 0.f;
        }
        if (!on) continue;
        if (p.outer == 1) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + grow * D + c * 16);
          dst[0] = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
          dst[1] = make_uint4(pack_bf16(f[8], f[9]), pack_bf16(f[10], f[11]), pack_bf16(f[12], f[13]), pack_bf16(f[14], f[15]));
        } else {
          float4* dst = reinterpret_cast<float4*>(p.part_o + ((long long)split * rows_all + grow) * D + c * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) dst[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        }
      }
      if (on) {
        const float lse2 = empty ? -INFINITY : m + log2f(l);
        if (p.outer == 1) {
          if (p.lse) p.lse[grow] = empty ? 0.f : lse2 * kLn2;
        } else {
          p.part_lse[(long long)split * rows_all + grow] = lse2;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == QT_CVT_WARP) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(QT_TMEM_COLS));
  }
}

template <int D>
static sb_status launch_quant_tc_d(const QuantAttnParams& p, dim3 grid, cudaStream_t cs) {
  static PerDeviceOnce once;
  if (!once.run([]() {
        const bool ok = cudaFuncSetAttribute(quant_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, quant_tc_smem<D>()) == cudaSuccess;
        if (!ok) cudaGetLastError();
        return ok;
      }))
    return SB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(QT_THREADS);
  cfg.dynamicSmemBytes = quant_tc_smem<D>();
  cfg.stream = cs;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, quant_tc_kernel<D>, p) != cudaSuccess) {
    cudaGetLastError();
    return SB_ERR_CUDA;
  }
  return launch_check();
}

// grid = (chunks, KV heads x tile pairs, sequences)
sb_status launch_quant_tc(const QuantAttnParams& p, dim3 grid, cudaStream_t cs) {
  return p.kv.head_dim == 64 ? launch_quant_tc_d<64>(p, grid, cs) : launch_quant_tc_d<128>(p, grid, cs);
}

}  // namespace sb
