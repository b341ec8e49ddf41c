// Tree attention over an 8-bit prefix on the tensor cores (tcgen05 + TMEM, sm_100a), for tiles of 128 packed rows.
//
// S = Q K^T runs on the codes as they are (kind::f8f6f4, K straight from a TMA tile in shared memory): a bf16 number scaled by its
// row's power of two is the sum of two e4m3 numbers (eight significant bits are four and a signed four; elements 2^-10
// and more below the row's largest lose what is below 2^-18 of it), so Q is held as two e4m3 terms and S costs two
// products at twice the 16-bit rate.  P would need a range that two e4m3 terms do not have (a sink with most of the weight
// beside thousands of small ones), so O = P V runs in fp16: two converter warps turn the V codes into an fp16 tile (exact:
// every e4m3 value is an fp16 value).  Converting K as well, and loading both through the converters' registers, took longer
// than everything else in the kernel: 3000 instructions a block in warps that issue one every eight clocks.
// Scales never touch an element of the stream: a K scale multiplies the scores of its 16 or more columns, a V scale enters the
// exponent (P' = 2^(s + log2 v - reference), denominator sum P' / v), which the fused multiply-add that forms
// the exponent does for nothing.
//
// A CTA owns one row tile of a KV head and a chunk of its key list, and works as two "streams" t = 0, 1: stream t takes half t (64
// keys) of every key block, with its own accumulator and two score buffers in tensor memory (2 x D + 4 x 64 columns) and its
// own softmax warpgroup of one thread per row; the two accumulators are merged at the end.  The MMA warp issues, for
// block i, O_t += P_i V of both streams and then S_{i+2} = Q K^T, 128 keys at once, into the buffers that P_i was read from.  So a
// softmax warp always has the next 64 scores waiting while the tensor pipe is busy with the buffer it has just left: with
// one buffer per stream the warps spent half of their time waiting for PV and S of their own stream.
// (One tile per CTA, although two tiles could share a key block's loads and conversions: both are off the critical path, which
// is the exponentials, and the smaller units fill the SMs more evenly: 191 us against 150 on 16 ragged trees,
// which take 131 now.)
//
// The softmax thread does not compute a maximum after its row's first visible key: the reference is raised when the sum of 64
// probabilities shows that an exponent is far above it (P' is fp16, which ends at 2^16), a rare event that
// rescales the accumulator.
//
// The tree's nodes are one block of their own, the first of the list: the softmax warps bring it into the first stages before anything
// else, scaled by a power of two per row as if they were codes (K as two e4m3 terms, V as fp16).  Its step has a function of its
// own in front of the loop, since its columns have a scale each; in the loop the same test cost 2 % of the long trees.  Then come the prefix
// blocks of 128 keys that the window leaves.
#include "quant_attention.cuh"

namespace sb {

constexpr int QT_SOFTMAX = 256;       // warps 0-3: stream 0, warps 4-7: stream 1
constexpr int QT_MMA_WARP = 8;
constexpr int QT_LOAD_WARP = 9;       // K and V tiles by TMA, scales
constexpr int QT_CVT_WARP = 10;       // warps 10, 11: V codes -> fp16
constexpr int QT_THREADS = 384;       // 12 warps leave 168 registers a thread
constexpr int QT_TMEM_COLS = 512;
constexpr int QT_SMALL = 8192;
constexpr float kQuantLimit = 8192.f; // sum of a step's 64 probabilities relative to the reference beyond which it is raised

enum QtBar { QB_P_FULL0, QB_P_FULL1,                                                          // 8 arrivals: the softmax warps
             QB_V_FULL0, QB_V_FULL1, QB_VR_EMPTY0, QB_VR_EMPTY1, QB_VR_EMPTY2,                // 2: the converter warps
             QB_K_FULL0, QB_K_FULL1, QB_K_FULL2, QB_VR_FULL0, QB_VR_FULL1, QB_VR_FULL2, QB_SC0, QB_SC_LAST = QB_SC0 + 7,
             QB_K_EMPTY0, QB_K_EMPTY1, QB_K_EMPTY2,
             QB_V_EMPTY0, QB_V_EMPTY1, QB_S_FULL0, QB_S_FULL1, QB_PV, QB_O_DONE,
             QB_Q_FULL, QB_COUNT };

// Q terms (2 x 128 D), K codes (3 stages), the tree's second K term, V codes (3 stages), V fp16 (2 stages).  Three stages of codes: a
// stage is free, asked for again and filled within the time of one block less than the ring holds, and a load takes longer than a block.
template <int D>
constexpr int quant_tc_smem() { return 1024 + QT_SMALL + TC_BM * D * (2 + 3 + 1 + 3 + 4); }

__device__ inline uint32_t tc_idesc_f16(int M, int N, int b_mn_major) {
  return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ inline uint32_t low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
__device__ inline uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two bf16 values times a factor, as fp16.
__device__ inline uint32_t scaled_f16(uint32_t w, float f) { return pack_f16(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xFFFF0000u) * f); }
// kind::f8f6f4, e4m3 A and B, both K-major: the same bits with other meanings of the type fields (0 = e4m3)
__device__ inline uint32_t tc_idesc_e4m3(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }
// One lane of the (converged) warp.
__device__ inline uint32_t elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(r));
  return r;
}
// The MMA forms of tc_common.cuh for a whole warp of which one lane issues: the operands are the same in every lane, so the
// compiler keeps them in uniform registers (a lane of its own would move each of them there for every MMA, which
// costs more issue time than the tensor pipe takes for the MMA).
__device__ inline void warp_mma_f8(uint32_t elected, uint32_t d_tmem, uint32_t alo, uint32_t blo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 ad, bd;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 ad, {%1, %3};\n\tmov.b64 bd, {%2, %3};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, p;\n\t}\n" ::"r"(d_tmem),
      "r"(alo), "r"(blo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
__device__ inline void warp_mma_ts(uint32_t elected, uint32_t d_tmem, uint32_t a_tmem, uint32_t blo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 bd;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 bd, {%2, %3};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, p;\n\t}\n" ::"r"(d_tmem),
      "r"(a_tmem), "r"(blo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
__device__ inline void warp_commit(uint32_t elected, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(smem_u32(bar)), "r"(elected)
      : "memory");
}
// 2^x for two values by the FMA pipe: x = n + f, |f| <= 1/2 (adding 1.5 * 2^23 rounds x to an integer, which the low bits of the sum then
// hold), 2^f by a polynomial of degree 4 fitted for equal relative error by Remez exchange (2.6e-6), 2^n by the exponent
// bits.  Below -126 the result is 2^-126; above 126 it means nothing.
__device__ inline void exp2_by_fma(float x0, float x1, float& y0, float& y1) {
  auto both = [](float v) { return pack_f32x2(v, v); };
  const unsigned long long x = pack_f32x2(fmaxf(x0, -126.f), fmaxf(x1, -126.f));
  const unsigned long long t = add_f32x2(x, both(12582912.f)), n = add_f32x2(t, both(-12582912.f)), f = fma_f32x2(n, both(-1.f), x);
  unsigned long long q = fma_f32x2(both(0.009570102f), f, both(0.05591786f));
  q = fma_f32x2(q, f, both(0.24024744f));
  q = fma_f32x2(q, f, both(0.6931218f));
  q = fma_f32x2(q, f, both(0.9999993f));
  float q0, q1, t0, t1;
  unpack_f32x2(q, q0, q1);
  unpack_f32x2(t, t0, t1);
  y0 = __uint_as_float(__float_as_uint(q0) + (__float_as_uint(t0) << 23));
  y1 = __uint_as_float(__float_as_uint(q1) + (__float_as_uint(t1) << 23));
}
__device__ inline float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
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

__device__ inline float4 lds_float4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}

// Rescales a row's accumulator in tensor memory.  Rare, and out of line: its registers and code stay out of the main loop.
template <int D>
static __device__ __noinline__ void rescale_row(uint32_t o_addr, float factor) {
#pragma unroll 1
  for (int c = 0; c < D / 16; ++c) {
    uint32_t r[16];
    tmem_ld16(o_addr + c * 16, r);
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * factor);
    tmem_st16(o_addr + c * 16, r);
  }
  tmem_wait_st();
}

// log2, exact for powers of two
__device__ inline float log2_of_scale(float s) {
  const uint32_t u = __float_as_uint(s);
  return (float)((int)(u >> 23) - 127) + __log2f(__uint_as_float((u & 0x7FFFFFu) | 0x3F800000u));
}
// Byte offset of 16-byte chunk `ch` of row `r` in a tile of D-byte rows, as TMA and the tensor core swizzle them (128-byte rows: XOR with
// the row's low three bits; 64-byte rows: with bits 1 and 2).
template <int D>
__device__ inline uint32_t code_tile_off(int r, int ch) {
  return (uint32_t)(r * D + ((ch ^ (D == 128 ? (r & 7) : ((r >> 1) & 3))) << 4));
}
// Lane -> (row, 16-element chunk) when a warp moves rows of D elements, 32 / (D / 16) rows at a time.  D = 128: eight neighbouring
// lanes hold four chunks of one row and the other four of the next: 16-byte codes that lie in different banks, and so do the fp16 halves
// that they become (a row's two fp16 column halves share their banks, two neighbouring rows do not).
template <int D>
__device__ inline int lane_chunk(int lane) { return D == 128 ? (lane & 3) | (((lane ^ (lane >> 1)) & 4)) : lane & 3; }
template <int D>
__device__ inline int lane_row(int lane) { return D == 128 ? ((lane >> 2) & 1) | ((lane >> 3) & 2) : lane >> 2; }

// 16 node rows (from row 16 * grp of `src`, n of them exist): this lane's 16 elements of each of its rows.
template <int D>
__device__ inline void load_node_rows(const bf16* src, long long stride, int n, int grp, int lane, uint4 (&x)[D / 16]) {
  constexpr int RPI = 512 / D, NI = 16 / RPI;
  const int ch = lane_chunk<D>(lane), r_in = lane_row<D>(lane);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int nd = 16 * grp + i * RPI + r_in;
    x[2 * i] = x[2 * i + 1] = make_uint4(0, 0, 0, 0);
    if (nd < n) {
      const uint4* s4 = reinterpret_cast<const uint4*>(src + nd * stride + ch * 16);
      x[2 * i] = s4[0];
      x[2 * i + 1] = s4[1];
    }
  }
}
// Rows that hold a NaN or an infinity become zeros; their bits (of 16) are returned.
template <int D>
__device__ inline uint32_t drop_bad_rows(int lane, uint4 (&x)[D / 16]) {
  constexpr int RPI = 512 / D, NI = 16 / RPI;
  const int r_in = lane_row<D>(lane);
  uint32_t mine = 0;  // bit i: this lane's part of its i-th row
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const uint32_t w[8] = {x[2 * i].x, x[2 * i].y, x[2 * i].z, x[2 * i].w, x[2 * i + 1].x, x[2 * i + 1].y, x[2 * i + 1].z, x[2 * i + 1].w};
    bool nf = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) nf |= bf16x2_nonfinite(w[k]);
    if (nf) mine |= 1u << (i * RPI + r_in);
  }
  const uint32_t bits = __reduce_or_sync(0xffffffffu, mine);
  if (bits)
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if ((bits >> (i * RPI + r_in)) & 1u) x[2 * i] = x[2 * i + 1] = make_uint4(0, 0, 0, 0);
  return bits;
}
// For each of this lane's rows the biased exponent e of the power of two 2^(e - 127) that takes the row's magnitudes below 2^(up + 1).  A row has
// an exponent of its own: of a tree's nodes only ancestors see each other, and a common one would let a large row cost the bits of
// rows beside it (one for 16 rows: a sibling 2^12 times larger moved scores by 0.07, one 2^16 times larger by 1.2).
template <int D>
__device__ inline void node_exponents(const uint4 (&x)[D / 16], int up, int least, int (&e)[D / 32]) {
  constexpr int NI = D / 32;
#pragma unroll
  for (int i = 0; i < NI; i += 2) {
    uint32_t m[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint4 a = x[2 * (i + k)], b = x[2 * (i + k) + 1];
      const uint32_t w = __vmaxu2(__vmaxu2(__vmaxu2(a.x & 0x7FFF7FFFu, a.y & 0x7FFF7FFFu), __vmaxu2(a.z & 0x7FFF7FFFu, a.w & 0x7FFF7FFFu)),
                                  __vmaxu2(__vmaxu2(b.x & 0x7FFF7FFFu, b.y & 0x7FFF7FFFu), __vmaxu2(b.z & 0x7FFF7FFFu, b.w & 0x7FFF7FFFu)));
      m[k] = max(w & 0xFFFFu, w >> 16);
    }
    uint32_t both = m[0] | (m[1] << 16);
    both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 1));
    both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 2));
    if (D == 128) both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 8));  // (see lane_row)
    e[i] = max((int)((both & 0xFFFFu) >> 7) - up, least);
    e[i + 1] = max((int)(both >> 23) - up, least);
  }
}
// What the step over the tree needs of a node's rows: 2^e of K and the exponent of V's power of two.
struct NodeScales {
  float *k, *log_v;
};
// 16 rows of the tree (group grp), one warp: V as fp16, or K as two e4m3 terms, and their scales.
template <int D>
__device__ inline void put_node_v(int grp, int lane, const uint4 (&x)[D / 16], uint8_t* v16, NodeScales scales) {
  constexpr int RPI = 512 / D, NI = 16 / RPI;
  const int ch = lane_chunk<D>(lane), r_in = lane_row<D>(lane);
  int ev[NI];
  node_exponents<D>(x, 8, 127 - 60, ev);  // (see v_scale_used)
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = 16 * grp + i * RPI + r_in;
    const float inv = __uint_as_float((uint32_t)(254 - ev[i]) << 23);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t w[4] = {x[2 * i + k].x, x[2 * i + k].y, x[2 * i + k].z, x[2 * i + k].w};
      uint32_t h[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) h[c] = scaled_f16(w[c], inv);
      *reinterpret_cast<uint4*>(v16 + sw128_chunk_off(r, 2 * ch + k, TC_BN)) = make_uint4(h[0], h[1], h[2], h[3]);
    }
    if (ch == 0) scales.log_v[r] = (float)(ev[i] - 127);
  }
}
template <int D>
__device__ inline void put_node_k(int grp, int lane, const uint4 (&y)[D / 16], uint8_t* k1, uint8_t* k2, NodeScales scales) {
  constexpr int RPI = 512 / D, NI = 16 / RPI;
  const int ch = lane_chunk<D>(lane), r_in = lane_row<D>(lane);
  int ek[NI];
  node_exponents<D>(y, 7, 1, ek);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = 16 * grp + i * RPI + r_in;
    const float inv = __uint_as_float((uint32_t)(254 - ek[i]) << 23);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t w[4] = {y[2 * i + k].x, y[2 * i + k].y, y[2 * i + k].z, y[2 * i + k].w};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint16_t h0, l0, h1, l1;
        split_e4m3(scaled_f16(w[2 * c], inv), h0, l0);
        split_e4m3(scaled_f16(w[2 * c + 1], inv), h1, l1);
        hi[2 * k + c] = h0 | ((uint32_t)h1 << 16);
        lo[2 * k + c] = l0 | ((uint32_t)l1 << 16);
      }
    }
    const uint32_t off = code_tile_off<D>(r, ch);
    *reinterpret_cast<uint4*>(k1 + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(k2 + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if (ch == 0) scales.k[r] = __uint_as_float((uint32_t)ek[i] << 23);
  }
}

// A row's step over the tree: 64 scores of nodes, of which those count whose bit of `words` is set, become probabilities.  A node's
// exponent is its score times the scales of Q and K, plus the logarithm of V's power of two; the reference is the largest of them.
// scales: shared address of the nodes' K scales, SB_MAX_NODES floats before the logarithms.  -> reference (-inf: no node is visible),
// denominator relative to it.  The denominator is summed on its own, from scores: the columns have no common V scale.
__device__ __forceinline__ float2 tree_step(uint32_t addr, uint2 words, float qs, uint32_t scales) {
  float most = -INFINITY, ref = -INFINITY, sum = 0.f;
  if (!__any_sync(0xffffffffu, (words.x | words.y) != 0)) {
    const uint32_t none[16] = {};
    tmem_st16(addr, none);
    tmem_st16(addr + 16, none);
    return make_float2(ref, sum);
  }
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {  // both halves for the largest, both for the probabilities (stored over scores that are done with)
    const int q = pass & 1;
    const uint32_t word = q ? words.y : words.x, at = scales + q * 128;
    uint32_t x[32];
    tmem_ld32(addr + 32 * q, x);
    float s[32], d[32];
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const float4 k = lds_float4(at + e * 4), v = lds_float4(at + (SB_MAX_NODES + e) * 4);
      const float f[4] = {qs * k.x, qs * k.y, qs * k.z, qs * k.w}, lv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool on = (word >> (e + c)) & 1u;
        s[e + c] = on ? __uint_as_float(x[e + c]) * f[c] : -INFINITY;
        d[e + c] = on ? s[e + c] + lv[c] : -INFINITY;
      }
    }
    if (pass < 2) {
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        most = max3(most, s[e], s[e + 1]);
        ref = max3(ref, d[e], d[e + 1]);
      }
    } else {
      const float m = most == -INFINITY ? 0.f : most, r = ref == -INFINITY ? 0.f : ref;
      uint32_t pk[16];
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        sum += fast_exp2(s[e] - m) + fast_exp2(s[e + 1] - m);
        pk[e >> 1] = pack_f16(fast_exp2(d[e] - r), fast_exp2(d[e + 1] - r));
      }
      tmem_st16(addr + 16 * q, pk);
    }
  }
  return make_float2(ref, ref == -INFINITY ? sum : sum * fast_exp2(most - ref));
}

// Scores of 32 columns whose bit is not set become -inf.
static __device__ __noinline__ void mask_scores(uint32_t addr, uint32_t word) {
  uint32_t x[32];
  tmem_ld32(addr, x);
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!((word >> e) & 1u)) x[e] = 0xff800000u;
  tmem_st32(addr, x);
  tmem_wait_st();
}

// The CTA's sequence, KV head and row tile when CTAs are handed out in order: sequences longest first, for each its heads, for each head
// the tiles that it has (at least one).  False for the CTAs behind the last.  A grid of the longest tree's tiles for every sequence, run as
// it is, starts CTAs without work before others with much (16 windowed trees of 5 to 33 nodes 36.3 us; so, 35.6).  batch <= SB_MAX_NODES;
// s_len: 16-byte aligned scratch of 2 * SB_MAX_NODES ints, s_pick: two ints.
__device__ inline bool quant_unit_of_rank(const QuantAttnParams& p, int most, int* s_len, int* s_pick, int& b, int& g, int& tile) {
  const int B = p.kv.batch, tid = threadIdx.x;
  int* s_tiles = s_len + SB_MAX_NODES;
  for (int i = tid; i < SB_MAX_NODES; i += blockDim.x) {
    int len = (int)0x80000000, n = 0;
    if (i < B) {
      len = p.tree.prefix_len[i];
      n = p.tree.node_offsets[i + 1] - p.tree.node_offsets[i] - (p.q_node_begin ? p.q_node_begin[i] : 0);
      n = min(max(ceil_div(min(max(n, 0), SB_MAX_NODES) * p.G, TC_BM), 1), most);
    }
    s_len[i] = len;
    s_tiles[i] = n;
  }
  if (tid == 0) s_pick[0] = -1;
  __syncthreads();
  const int unit = blockIdx.z * gridDim.y + blockIdx.y, Hkv = p.kv.n_kv_heads;
  for (int i = tid; i < B; i += blockDim.x) {
    const int me = s_len[i];
    int start = 0;
#pragma unroll 4
    for (int j = 0; j < B; j += 4) {
      const int4 o = *reinterpret_cast<const int4*>(s_len + j), t = *reinterpret_cast<const int4*>(s_tiles + j);
      start += (o.x > me || (o.x == me && j < i) ? t.x : 0) + (o.y > me || (o.y == me && j + 1 < i) ? t.y : 0) +
               (o.z > me || (o.z == me && j + 2 < i) ? t.z : 0) + (o.w > me || (o.w == me && j + 3 < i) ? t.w : 0);
    }
    if (unit >= start * Hkv && unit < (start + s_tiles[i]) * Hkv) {
      s_pick[0] = i;
      s_pick[1] = start;
    }
  }
  __syncthreads();
  b = s_pick[0];
  if (b >= 0) {
    const int mine = unit - s_pick[1] * Hkv;
    g = mine / s_tiles[b];
    tile = mine - g * s_tiles[b];
  }
  __syncthreads();
  return b >= 0;
}

// After a wait that gave up: shared memory must not be given back under copies in flight.  The last one of every stage is awaited, again with
// a limit.
static __device__ __noinline__ void await_loads(uint64_t* bars, const int* asked, int first_k, volatile int* abort_flag) {
  for (int k = max(first_k, asked[0] - 3); k < asked[0]; ++k) mbar_wait(&bars[QB_K_FULL0 + k % 3], (k / 3) & 1, abort_flag);
  for (int k = max(0, asked[1] - 3); k < asked[1]; ++k) mbar_wait(&bars[QB_VR_FULL0 + k % 3], (k / 3) & 1, abort_flag);
}

template <int D>
__global__ void __launch_bounds__(QT_THREADS, 1) quant_tc_kernel(const QuantAttnParams p, const __grid_constant__ CUtensorMap kmap,
                                                                 const __grid_constant__ CUtensorMap vmap, const int box_rows) {
  constexpr int TILE8 = TC_BN * D;      // 128 rows of codes
  constexpr int TILE = 2 * TILE8;       // 128 rows of fp16
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint32_t* s_anc = reinterpret_cast<uint32_t*>(base);               // 2048 B
  int* s_parent = reinterpret_cast<int*>(base + 2048);               // 512 B
  int* s_depth = reinterpret_cast<int*>(base + 2560);                // 512 B
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(base + 4352);        // QB_COUNT * 8 <= 512
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(base + 3328);
  volatile int* s_abort = reinterpret_cast<volatile int*>(base + 3332);   // [0] a wait gave up; [1] the same for the last wait
  int* s_err = reinterpret_cast<int*>(base + 3340);
  int* s_asked = reinterpret_cast<int*>(base + 3392);                // blocks of K and of V codes that the loader has asked for
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(base + 3344);        // [4]: node rows with a NaN or an infinity
  uint32_t* s_flag = reinterpret_cast<uint32_t*>(base + 3360);       // [8 slots]: bits 0-7 the groups with a NaN scale, bits 8-15 those whose V reads as zeros
  // Eight slots: the loader writes block j's when S of block j - 3 is done, i.e. the softmax with block j - 5.
  float* s_ks = reinterpret_cast<float*>(base + 7168);               // [8 slots][8 groups of 16 keys] K scale
  float* s_lsv = s_ks + 64;                                          // log2 of the V scale
  float* s_isv = s_lsv + 64;                                         // 1 / V scale
  float* s_qs = reinterpret_cast<float*>(base + 3840);               // [128 rows] scale of a Q row
  float* s_ml = reinterpret_cast<float*>(base + 4864);               // [2 streams][reference, sum][128 rows]
  float* s_node = s_ml;                                              // [2][128 nodes]: NodeScales; read before the first P V, s_ml written after the last
  uint8_t* sQ = base + QT_SMALL;      // [2 terms]
  uint8_t* sK = sQ + 2 * TILE8;       // [3 stages] codes
  uint8_t* sK2 = sK + 3 * TILE8;      // second term of the tree's K
  uint8_t* sVr = sK2 + TILE8;         // [3 stages] codes
  uint8_t* sV = sVr + 3 * TILE8;      // [2 stages] fp16

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;  // (known to be uniform)
  const int split = blockIdx.x;
  const int Hq = p.tree.n_q_heads, Hkv = p.kv.n_kv_heads, G = p.G;
  if (tid == 0) {
    s_abort[0] = s_abort[1] = 0;
    for (int i = 0; i < 4; ++i) s_bad[i] = 0;
    s_flag[0] = 0;
    for (int i = 0; i < QB_COUNT; ++i)
      mbar_init(&s_bar[i], i <= QB_P_FULL1 ? 8 : i <= QB_VR_EMPTY2 ? 2 : i == QB_Q_FULL ? QT_SOFTMAX : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == QT_MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(QT_TMEM_COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  pdl_release();

  // The tiles of a KV head are neighbours: they share its codes in L2.
  const int tiles = (int)gridDim.y / Hkv;
  int b = blockIdx.z, g = blockIdx.y / tiles, tile = blockIdx.y % tiles;
  if (p.sort_seqs && !quant_unit_of_rank(p, tiles, reinterpret_cast<int*>(s_anc), s_parent, b, g, tile)) {
    if (warp == QT_MMA_WARP)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*s_tmem), "r"(QT_TMEM_COLS));
    return;
  }
  const int row0 = tile * TC_BM;
  const QuantSeq si = load_quant_seq(p, b);
  const int rows_total = si.nq * G;
  const bool designated = split == 0 && g == 0 && tile == 0;
  if (!si.can_write || row0 >= rows_total) {
    if (designated) {
      const bool pages_ok = si.err ? true : quant_pages_in_pool(p.kv, b, si.P, whole_cta());
      if (tid == 0) p.status[b] = si.err ? si.err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
    }
    if (warp == QT_MMA_WARP)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*s_tmem), "r"(QT_TMEM_COLS));
    return;
  }
  const long long rows_all = (long long)p.total_q * Hq;

  const BlockList list = visible_blocks(si.P, p.window, p.sinks, TC_BN);
  const int total = si.err ? 0 : list.count + 1;                    // the tree is the first block
  const int per = total / p.num_splits, rem = total % p.num_splits;
  const int blk0 = split * per + min(split, rem);
  const int nb = per + (split < rem ? 1 : 0);
  const int tree_blocks = nb > 0 && blk0 == 0 ? 1 : 0;              // this CTA's first block is the tree
  auto prefix_key = [&](int i) { return list.at(blk0 + i - 1) * TC_BN; };  // first key of this CTA's i-th block
  const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0);
  const uint32_t tmem_o = tmem + 4 * 64;                            // accumulator of stream t at tmem_o + t * D

  // state of the softmax threads
  const int t_mine = warp >> 2, row = (warp & 3) * 32 + lane;
  const uint32_t lane_base = ((uint32_t)((warp & 3) * 32)) << 16;
  float ref = 0.f, l_run = 0.f;
  bool seen_any = false;  // the row has met a visible key, and `ref` is its reference
  bool ok = true, compute = false;

  if (warp < QT_SOFTMAX / 32) {
    const int groups = tree_blocks ? (si.n + 15) >> 4 : 0;
    // Q: 16-byte pieces, D / 8 lanes to a row
    constexpr int LPR = D / 8, RPP = QT_SOFTMAX / LPR, NQ = TC_BM / RPP;
    const int ch = tid % LPR;
    uint4 xq[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int R = row0 + i * RPP + tid / LPR;
      const int nl = (int)((unsigned)R * p.g_magic >> 20), hh = R - nl * G;
      xq[i] = make_uint4(0, 0, 0, 0);
      if (R < rows_total && SB_CHECKED_ACCESS(si.q_off + nl, p.total_q, &p.status[b]))
        xq[i] = __ldg(reinterpret_cast<const uint4*>(p.q + (long long)(si.q_off + nl) * p.q_stride + (g * G + hh) * D + ch * 8));
    }
    // Nodes: warp w takes V (w even) or K (odd) of groups w / 2 and 4 + w / 2 of 16 nodes.  (Rolled: this code runs once, and costs its
    // instruction fetches: unrolled twice 16 trees take 134.5 us, so 133.2.)
    const NodeScales scales = {s_node, s_node + SB_MAX_NODES};
#pragma unroll 1
    for (int grp = warp >> 1; grp < groups; grp += 4) {
      uint4 xn[D / 16];
      load_node_rows<D>((warp & 1 ? p.k_nodes : p.v_nodes) + (long long)si.node_base * p.node_stride + g * D, p.node_stride, si.n,
                        grp, lane, xn);
      const uint32_t bits = drop_bad_rows<D>(lane, xn);
      if (bits && lane == 0) atomicOr(&s_bad[grp >> 1], bits << (16 * (grp & 1)));
      if (warp & 1) put_node_k<D>(grp, lane, xn, sK, sK2, scales);
      else put_node_v<D>(grp, lane, xn, sV, scales);
    }
    if (tree_blocks) {  // groups without nodes: K may be anything (masked), V has to be finite
      for (int i = groups * 2 * D + tid; i < TC_BN * D / 8; i += QT_SOFTMAX)
        *reinterpret_cast<uint4*>(sV + sw128_chunk_off(i / (D / 8), i % (D / 8), TC_BN)) = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int r = i * RPP + tid / LPR;
      const uint32_t w[4] = {xq[i].x, xq[i].y, xq[i].z, xq[i].w};
      uint32_t amax = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
#pragma unroll
      for (int d = 1; d < LPR; d <<= 1) amax = __vmaxu2(amax, __shfl_xor_sync(0xffffffffu, amax, d));
      const int ex = (int)(max(amax & 0xFFFFu, amax >> 16) >> 7);
      const int e = ex == 255 ? 127 : min(max(ex - 7, 1), 253);   // the largest element becomes 2^7 .. 2^8
      const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
      uint16_t hi[4], lo[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) split_e4m3(scaled_f16(w[k], inv), hi[k], lo[k]);
      uint8_t* dst = sQ + code_tile_off<D>(r, ch >> 1) + (ch & 1) * 8;
      *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0] | ((uint32_t)hi[1] << 16), hi[2] | ((uint32_t)hi[3] << 16));
      *reinterpret_cast<uint2*>(dst + TILE8) = make_uint2(lo[0] | ((uint32_t)lo[1] << 16), lo[2] | ((uint32_t)lo[3] << 16));
      // a row with a NaN or an infinity is NaN throughout (e4m3 has no infinity)
      if (ch == 0) s_qs[r] = ex == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)e << 23) * p.scale_log2;
    }
    fence_async_smem();
    mbar_arrive(&s_bar[QB_Q_FULL]);
    asm volatile("bar.sync 3, 320;" ::: "memory");   // the converters have planned the tree, s_qs is complete
    compute = *s_err == 0;
    if (tree_blocks && tid == 0) {  // every writer has fenced its part before the barrier
      mbar_arrive(&s_bar[QB_K_FULL0]);
      mbar_arrive(&s_bar[QB_V_FULL0]);
      mbar_arrive(&s_bar[QB_V_FULL0]);
      mbar_arrive(&s_bar[QB_SC0]);
    }

    // ---- softmax --------------------------------------------------------------------------------------------------
    const int R = row0 + row;
    const int node = (R < rows_total && compute) ? si.q0 + (int)((unsigned)R * p.g_magic >> 20) : -1;
    const int pos = si.P + (node >= 0 ? s_depth[node] : 0);
    const float qs = s_qs[row];
    bool poison = false;

    // One step's 64 scores of this row -> probabilities.  The two halves have no branch between them, so that one fills the
    // gaps of the other (a check of the reference after each half: 16 trees 148 us; one check: 136).
    auto walk = [&](int i, int group, uint32_t s_addr) {
      const float4 ks = *reinterpret_cast<const float4*>(s_ks + group), ls = *reinterpret_cast<const float4*>(s_lsv + group);
      const float4 is = *reinterpret_cast<const float4*>(s_isv + group);
      // exponents relative to the present reference
      // (a factor that underflows would turn the -inf of an invisible key into NaN; a NaN factor stays)
      const float f[4] = {max_nan(qs * ks.x, 1.17549435e-38f), max_nan(qs * ks.y, 1.17549435e-38f), max_nan(qs * ks.z, 1.17549435e-38f),
                          max_nan(qs * ks.w, 1.17549435e-38f)};
      const float c[4] = {ls.x - ref, ls.y - ref, ls.z - ref, ls.w - ref};
      const float inv_v[4] = {is.x, is.y, is.z, is.w};
      float d[64], part[4], most = 0.f;  // most: of the exponents whose exponential would not show by its size how large they are
      uint32_t pk[2][16];
      auto exponents = [&](int h, const uint32_t (&x)[32]) {
#pragma unroll
        for (int e = 0; e < 32; e += 2)
          unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), pack_f32x2(f[2 * h + (e >> 4)], f[2 * h + (e >> 4)]),
                                 pack_f32x2(c[2 * h + (e >> 4)], c[2 * h + (e >> 4)])), d[32 * h + e], d[32 * h + e + 1]);
      };
      auto probabilities = [&](int h) {
        unsigned long long sum2[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          // some exponentials go to the FMA pipe: the other pipe does 16 a clock (of 64 columns 4 / 8 / 12 / 16: 134 / 136 / 136 / 138
          // us on 16 trees; on long ones 12 and 16 take 0.5 and 2 % longer than 8)
          float p0, p1;
          const float d0 = d[32 * h + e], d1 = d[32 * h + e + 1];
          if ((e & 15) == 14) {
            exp2_by_fma(d0, d1, p0, p1);
            most = max3(most, d0, d1);
          } else {
            p0 = fast_exp2(d0);
            p1 = fast_exp2(d1);
          }
          sum2[e >> 4] = add_f32x2(sum2[e >> 4], pack_f32x2(p0, p1));
          pk[h][e >> 1] = pack_f16(p0, p1);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float u, v;
          unpack_f32x2(sum2[k], u, v);
          part[2 * h + k] = u + v;
        }
      };
      {
        uint32_t x0[32], x1[32];
        tmem_ld32_async(s_addr, x0);
        tmem_wait_ld(x0);
        tmem_ld32_async(s_addr + 32, x1);
        exponents(0, x0);
        tmem_wait_ld(x1);
        exponents(1, x1);
      }
      // The reference stays while no exponent is far above it.  That shows in the sums, which are needed anyway: a sum
      // beyond 2^13 (or infinite) means an exponent above 7, and the step is done again with a new reference.
      bool raise = !seen_any;
      while (true) {
        if (__any_sync(0xffffffffu, raise)) {
          float top = -INFINITY;
#pragma unroll
          for (int e = 0; e < 64; e += 2) top = max3(top, d[e], d[e + 1]);
          const float delta = raise && top > -INFINITY ? top : 0.f;
          const float factor = seen_any ? fast_exp2(-delta) : 1.f;  // nothing accumulated yet: nothing to scale
          seen_any |= raise && top > -INFINITY;
#pragma unroll
          for (int e = 0; e < 64; ++e) d[e] -= delta;
          ref += delta;
          l_run *= factor;
          // the accumulator holds the steps before this one: the last of them may still be under way
          if (i > 0) {
            if (ok) ok = mbar_wait(&s_bar[QB_PV], (i - 1) & 1, s_abort);
            __syncwarp();
            tc_fence_after();
            rescale_row<D>(tmem_o + t_mine * D + lane_base, factor);
          }
        }
        most = 0.f;
        probabilities(0);
        probabilities(1);
        raise = (part[0] + part[1]) + (part[2] + part[3]) > kQuantLimit || most > 14.f;
        if (!__any_sync(0xffffffffu, raise)) break;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) l_run = fmaf(part[k], inv_v[k], l_run);
      tmem_st16(s_addr, pk[0]);
      tmem_st16(s_addr + 16, pk[1]);
    };
    // A wait that gives up leaves `ok` false; the steps still run to their end, so that every barrier gets its arrivals.
    auto await_scores = [&](int i) {
      if (ok) ok = mbar_wait(&s_bar[QB_SC0 + (i & 7)], (i >> 3) & 1, s_abort) &&
                   mbar_wait(&s_bar[QB_S_FULL0 + (i & 1)], (i >> 1) & 1, s_abort);
      __syncwarp();
      tc_fence_after();
      return tmem + lane_base + (2 * (i & 1) + t_mine) * 64;
    };
    auto hand_over = [&](int i) {
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_bar[QB_P_FULL0 + (i & 1)]);
    };
    if (tree_blocks) {
      const uint32_t s_addr = await_scores(0);
      uint2 words = make_uint2(0u, 0u);
#pragma unroll 1
      for (int q = 0; q < 2; ++q) {
        const int w0 = 2 * t_mine + q;         // the nodes 32 w0 .. + 31
        uint32_t word = node >= 0 ? s_anc[4 * node + w0] : 0u;
        if (p.window > 0 && p.window < si.n) {  // (a node's ancestors lie less than n positions back)
          for (uint32_t w = word; w; w &= w - 1) {
            const int bit = __ffs(w) - 1, kp = si.P + s_depth[32 * w0 + bit];
            if (!(kp < p.sinks || pos - kp < p.window)) word &= ~(1u << bit);
          }
        }
        poison |= (word & s_bad[w0]) != 0;
        if (q) words.y = word;
        else words.x = word;
      }
      const float2 r = tree_step(s_addr, words, qs, smem_u32(s_node + 64 * t_mine));
      seen_any = r.x > -INFINITY;
      if (seen_any) ref = r.x;
      l_run = r.y;
      hand_over(0);
    }
    for (int i = tree_blocks; i < nb; ++i) {
      const int group = (i & 7) * 8 + t_mine * 4;
      const int k0 = prefix_key(i) + 64 * t_mine;
      // steps that every row sees whole need no mask
      const bool masked = k0 + 64 > si.P || (p.window > 0 && k0 + 64 > p.sinks && si.P + si.n - 1 - k0 >= p.window);
      const uint32_t s_addr = await_scores(i);
      const uint32_t flags = (s_flag[i & 7] >> (4 * t_mine)) & 15u;   // poisoned 16-key groups of the step
      if (masked || flags) {
        // invisible scores become -inf in tensor memory before the walk
#pragma unroll 1
        for (int q = 0; q < 2; ++q) {
          const int kq = k0 + 32 * q;
          uint32_t word = low_bits(si.P - kq);
          if (p.window > 0) word &= low_bits(p.sinks - kq) | ~low_bits(pos - p.window + 1 - kq);
          poison |= ((flags >> (2 * q)) & 1u && (word & 0xFFFFu)) || ((flags >> (2 * q + 1)) & 1u && (word >> 16));
          if (__any_sync(0xffffffffu, word != ~0u)) mask_scores(s_addr + 32 * q, word);
        }
      }
      walk(i, group, s_addr);
      hand_over(i);
    }
    if (!ok) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
    if (poison) l_run = __uint_as_float(0x7FC00000u);
    if (!compute) {
      l_run = 0.f;
      seen_any = false;
    }
  } else if (warp == QT_MMA_WARP) {
    // ---- MMA issuer -------------------------------------------------------------------------------------------------
    const uint32_t elected = elect_one();
    const uint32_t hi = tc_desc_hi(1024);
    // 8-bit tiles: 128-byte rows and swizzle (eight rows = 1024 bytes), or 64-byte ones (512; layout type 4)
    const uint32_t hi8 = D == 128 ? tc_desc_hi(1024) : ((512u >> 4) | (1u << 14) | (4u << 29));
    const uint32_t q_lo = tc_desc_lo(smem_u32(sQ), 16), k_lo = tc_desc_lo(smem_u32(sK), 16), k2_lo = tc_desc_lo(smem_u32(sK2), 16);
    const uint32_t v_lo = tc_desc_lo(smem_u32(sV), TC_BN * 128);
    const uint32_t idesc_s = tc_idesc_e4m3(TC_BM, TC_BN), idesc_pv = tc_idesc_f16(TC_BM, D, 1);
    auto issue_s = [&](int i) {  // both streams: score buffers 2 (i & 1) and 2 (i & 1) + 1 are neighbours
      ok = ok && mbar_wait(&s_bar[QB_K_FULL0 + i % 3], (i / 3) & 1, s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      tc_fence_after();
      const uint32_t d = tmem + (i & 1) * 128;
      uint32_t kb = k_lo + (i % 3) * (TILE8 >> 4);
      // (Q1 + Q2) K, and for the tree (Q1 + Q2) (K1 + K2); 32 elements a step
      const int terms = i < tree_blocks ? 2 : 1;
#pragma unroll 1
      for (int c = 0; c < terms; ++c) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          warp_mma_f8(elected, d, q_lo + (ks / (D / 32)) * (TILE8 >> 4) + (ks % (D / 32)) * 2, kb + (ks % (D / 32)) * 2, hi8, idesc_s, c + ks > 0);
        kb = k2_lo;
      }
      warp_commit(elected, &s_bar[QB_S_FULL0 + (i & 1)]);
      warp_commit(elected, &s_bar[QB_K_EMPTY0 + i % 3]);
    };
    auto issue_pv = [&](int i) {
      ok = ok && mbar_wait(&s_bar[QB_V_FULL0 + (i & 1)], (i >> 1) & 1, s_abort) && mbar_wait(&s_bar[QB_P_FULL0 + (i & 1)], (i >> 1) & 1, s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      tc_fence_after();
      const uint32_t vb = v_lo + (i & 1) * (TILE >> 4), pb = tmem + (i & 1) * 128;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          warp_mma_ts(elected, tmem_o + t * D, pb + t * 64 + ks * 8, vb + (t * 4 + ks) * (2048 >> 4), hi, idesc_pv, (i > 0 || ks > 0) ? 1u : 0u);
      warp_commit(elected, &s_bar[QB_PV]);
      warp_commit(elected, &s_bar[QB_V_EMPTY0 + (i & 1)]);
    };
    if (nb > 0) ok = __all_sync(0xffffffffu, mbar_wait(&s_bar[QB_Q_FULL], 0, s_abort));
    // (the first two rounds only issue S; rolled, so that the code is there once)
#pragma unroll 1
    for (int i = -2; i < nb; ++i) {
      if (i >= 0) issue_pv(i);
      if (i + 2 < nb) issue_s(i + 2);
    }
    warp_commit(elected, &s_bar[QB_O_DONE]);
    if (!ok && lane == 0) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
  } else if (warp == QT_LOAD_WARP) {
    // ---- loader: lane l < 8 looks after keys 16 l .. + 15 of every block -----------------------------------------------
    const bool paged = p.kv.page_size != 0;
    const int page_shift = paged ? 31 - __clz(p.kv.page_size) : 31;
    const int* table = paged ? p.kv.page_table + (long long)b * p.kv.max_pages : nullptr;
    auto my_key = [&](int j) { return prefix_key(j) + 16 * lane; };
    auto my_page = [&](int j) {  // page id of this lane's keys, unchecked (nothing waits for it here)
      if (!paged || lane >= 8 || j >= nb || my_key(j) >= si.P) return 0;
      return __ldg(table + (my_key(j) >> page_shift));
    };
    int page = my_page(tree_blocks);
    int asked_k = tree_blocks, asked_v = 0;  // blocks asked for
    for (int j = tree_blocks; j < nb; ++j) {
      const int r = j - tree_blocks;                            // the stages of V codes are used from the first prefix block on
      const int key = my_key(j);
      const bool on = lane < 8 && key < si.P;
      if (page < 0 || page >= p.kv.num_pages) page = 0;  // reported by the designated CTA; reads stay in the pool
      const int in_page = paged ? key & (p.kv.page_size - 1) : key;
      const long long crow = (paged ? (long long)page << page_shift : (long long)b * p.kv.kv_capacity) + in_page;
      float ks = 1.f, vs = 1.f;
      if (on && SB_CHECKED_ACCESS(crow + 15, quant_rows_total(p.kv), &p.status[b])) {
        ks = __ldg(p.k_scale + (crow >> p.block_shift) * Hkv + g);
        vs = __ldg(p.v_scale + (crow >> p.block_shift) * Hkv + g);
      }
      const bool piece = on && (16 * lane & (box_rows - 1)) == 0;     // this lane's keys begin a TMA box
      const uint32_t pieces = __popc(__ballot_sync(0xffffffffu, piece));
      const int c2 = in_page, c3 = paged ? page : b;
      page = my_page(j + 1);
      const int ks_at = j % 3, vs_at = r % 3;
      if (j >= 3) ok = ok && mbar_wait(&s_bar[QB_K_EMPTY0 + ks_at], (j / 3 - 1) & 1, s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(&s_bar[QB_K_FULL0 + ks_at], pieces * box_rows * D);
      __syncwarp();
      if (piece) tma_load_4d(smem_u32(sK) + ks_at * TILE8 + 16 * lane * D, &kmap, 0, g, c2, c3, &s_bar[QB_K_FULL0 + ks_at]);
      asked_k = j + 1;
      if (r >= 3) ok = ok && mbar_wait(&s_bar[QB_VR_EMPTY0 + vs_at], (r / 3 - 1) & 1, s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(&s_bar[QB_VR_FULL0 + vs_at], pieces * box_rows * D);
      __syncwarp();
      if (piece) tma_load_4d(smem_u32(sVr) + vs_at * TILE8 + 16 * lane * D, &vmap, 0, g, c2, c3, &s_bar[QB_VR_FULL0 + vs_at]);
      asked_v = r + 1;
      // A NaN scale poisons the rows that see one of its keys; it is noted, and 1 takes its place, so that it meets no other row.
      const uint32_t nan = __ballot_sync(0xffffffffu, ks != ks || vs != vs), tiny = __ballot_sync(0xffffffffu, vs < kMinVScale);
      if (ks != ks || vs != vs) ks = vs = 1.f;
      vs = v_scale_used(vs);
      if (lane < 8) {
        const int at = (j & 7) * 8 + lane;
        s_ks[at] = ks;
        s_lsv[at] = log2_of_scale(vs);
        s_isv[at] = __fdividef(1.f, vs);
      }
      if (lane == 0) s_flag[j & 7] = nan | (tiny << 8);
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_bar[QB_SC0 + (j & 7)]);
    }
    if (lane == 0) {
      s_asked[0] = asked_k;
      s_asked[1] = asked_v;
    }
    if (!ok && lane == 0) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
  } else {
    // ---- converters: warp cw owns rows 64 cw .. + 63 of every V block ----------------------------------------------------
    // Before the first block arrives they plan the tree for the softmax warps, which are busy with Q.
    {
      const ThreadGroup grp{tid - QT_CVT_WARP * 32, 64, false};
      const bool tree_ok = build_ancestors_smem(p.tree.parent + si.node_base, si.err ? 0 : si.n, s_parent, s_anc, s_depth, grp);
      int err = si.err;
      if (!err && !tree_ok) err = SB_ERR_INVALID_TREE;
      if (designated) {
        const bool pages_ok = err ? true : quant_pages_in_pool(p.kv, b, si.P, grp);
        if (grp.tid == 0) p.status[b] = err ? err : (pages_ok ? 0 : (int)SB_ERR_BOUNDS);
      }
      if (grp.tid == 0) *s_err = err;
      asm volatile("bar.sync 3, 320;" ::: "memory");
    }
    const int cw = warp - QT_CVT_WARP;
    constexpr int CPR = D / 16, RPI = 32 / CPR, NI = 32 / RPI;
    const int ch = lane_chunk<D>(lane), r_in = lane_row<D>(lane);
    const UnseenKeys unseen(si.P, p.window, p.sinks);
    for (int j = tree_blocks; j < nb; ++j) {
      const int st = (j - tree_blocks) % 3, use = (j - tree_blocks) / 3;
      uint8_t* stage = sV + (j & 1) * TILE;
      ok = mbar_wait(&s_bar[QB_VR_FULL0 + st], use & 1, s_abort) && mbar_wait(&s_bar[QB_SC0 + (j & 7)], (j >> 3) & 1, s_abort);
      if (ok && j >= 2) ok = mbar_wait(&s_bar[QB_V_EMPTY0 + (j & 1)], ((j >> 1) - 1) & 1, s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const uint8_t* raw = sVr + st * TILE8;
      const int k0 = prefix_key(j), left = si.P - k0;
      const bool gap = unseen.meets(k0, k0 + TC_BN);
      const uint32_t tiny = (s_flag[j & 7] >> 8) & 255u;
#pragma unroll 1
      for (int q = 0; q < 2; ++q) {
        const int r0 = 64 * cw + 32 * q;
        uint4 x[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) x[i] = *reinterpret_cast<const uint4*>(raw + code_tile_off<D>(r0 + i * RPI + r_in, ch));
        if (left < r0 + 32 || tiny || gap) {  // rows past the prefix (stale bytes) or before every window, and blocks that read as zeros
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const int r = r0 + i * RPI + r_in;
            if (r >= left || ((tiny >> (r >> 4)) & 1u) || unseen.has(k0 + r)) x[i] = make_uint4(0, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t h[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            h[2 * k] = half2_of_e4m3x2((uint16_t)w[k]);
            h[2 * k + 1] = half2_of_e4m3x2((uint16_t)(w[k] >> 16));
          }
          const int r = r0 + i * RPI + r_in;
          *reinterpret_cast<uint4*>(stage + sw128_chunk_off(r, 2 * ch, TC_BN)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(stage + sw128_chunk_off(r, 2 * ch + 1, TC_BN)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s_bar[QB_VR_EMPTY0 + st]);
        mbar_arrive(&s_bar[QB_V_FULL0 + (j & 1)]);
      }
    }
    if (!ok && lane == 0) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
  }

  // ---- store ----------------------------------------------------------------------------------------------------------
  // The two streams merge their accumulators: thread (stream t, row) takes half t of the row's columns, for which the other stream
  // hands its part over in shared memory.  Rows are staged with their number and log-sum-exp (over the idle Q and K
  // tiles); then half a warp per row writes whole rows.  A row that is final is bf16.  One that will be merged with other chunks' is fp16
  // with an exponent for every eight values, at half the bytes of fp32 (one 60-node tree over 2k keys in 6 chunks: 21.0 us and an error
  // of 0.0016 of the result, the output's own rounding; bf16 20.0 us and 0.0023).
  constexpr int ROWB = D * 2 + 48;                    // [row | exponents | base-2 log-sum-exp | pad | global row or -1 | pad (banks)]
  constexpr int DH = D / 2, RS = DH + 4;              // floats per half row handed over
  const bool have = nb > 0;
  if (warp < QT_SOFTMAX / 32) {
    // awaited even after a wait that gave up: tensor memory is idle before it is freed
    if (!mbar_wait(&s_bar[QB_O_DONE], 0, s_abort + 1)) atomicMax(&p.status[b], (int)SB_ERR_CUDA);
    __syncwarp();
    tc_fence_after();
    if (l_run != l_run) {  // a NaN outweighs everything it is merged with
      ref = INFINITY;
      seen_any = true;
    }
    float* hand0 = reinterpret_cast<float*>(sV + 2 * TILE - 2 * TC_BM * RS * 4);  // over the idle V tiles and the end of the codes before them
    float* hand = hand0 + (t_mine * TC_BM + row) * RS;
    if (have)
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) {
        uint32_t r[32];
        tmem_ld32(tmem_o + t_mine * D + lane_base + (t_mine ^ 1) * DH + c * 32, r);
#pragma unroll
        for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(hand + c * 32 + i) = make_uint4(r[i], r[i + 1], r[i + 2], r[i + 3]);
      }
    s_ml[t_mine * 256 + row] = seen_any ? ref : -INFINITY;
    s_ml[t_mine * 256 + 128 + row] = l_run;
    softmax_group_sync();
    const float m_me = seen_any ? ref : -INFINITY, m_other = s_ml[(t_mine ^ 1) * 256 + row], l_other = s_ml[(t_mine ^ 1) * 256 + 128 + row];
    const float m = fmaxf(m_me, m_other);
    float w_me = m_me == -INFINITY ? 0.f : fast_exp2(m_me - m), w_other = m_other == -INFINITY ? 0.f : fast_exp2(m_other - m);
    const float l = w_me * l_run + w_other * l_other;
    const bool empty = l == 0.f;
    const float inv = empty ? 0.f : 1.f / l;
    w_me *= inv;
    w_other *= inv;
    const float* theirs = hand0 + ((t_mine ^ 1) * TC_BM + row) * RS;
    uint8_t* dst = sQ + row * ROWB;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) {
      uint32_t r[32];
      if (have) tmem_ld32(tmem_o + t_mine * D + lane_base + t_mine * DH + c * 32, r);
#pragma unroll
      for (int i = 0; i < 32; i += 8) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = have && w_me != 0.f ? __uint_as_float(r[i + k]) * w_me : 0.f;  // (weight 0: nothing was written there)
        if (have && w_other != 0.f) {
          const float4 o0 = *reinterpret_cast<const float4*>(theirs + c * 32 + i), o1 = *reinterpret_cast<const float4*>(theirs + c * 32 + i + 4);
          f[0] = fmaf(o0.x, w_other, f[0]); f[1] = fmaf(o0.y, w_other, f[1]); f[2] = fmaf(o0.z, w_other, f[2]); f[3] = fmaf(o0.w, w_other, f[3]);
          f[4] = fmaf(o1.x, w_other, f[4]); f[5] = fmaf(o1.y, w_other, f[5]); f[6] = fmaf(o1.z, w_other, f[6]); f[7] = fmaf(o1.w, w_other, f[7]);
        }
        uint4& at = *reinterpret_cast<uint4*>(dst + (t_mine * DH + c * 32 + i) * 2);
        if (p.outer == 1) {
          at = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        } else {
          uint32_t amax = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) amax = max(amax, __float_as_uint(f[k]) & 0x7FFFFFFFu);
          const uint32_t ex = max(amax >> 23, 16u);   // the largest becomes 2^14 .. 2^15
          const float up = __uint_as_float((268u - ex) << 23);
          at = make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up), pack_f16(f[6] * up, f[7] * up));
          dst[D * 2 + (t_mine * DH + c * 32 + i) / 8] = (uint8_t)ex;
        }
      }
    }
    if (t_mine == 0) {
      const int R = row0 + row;
      const int nl = (int)((unsigned)R * p.g_magic >> 20);
      const long long grow = (long long)(si.q_off + nl) * Hq + g * G + (R - nl * G);
      const bool on = R < rows_total && SB_CHECKED_ACCESS(grow, rows_all, &p.status[b]);
      *reinterpret_cast<float*>(dst + D * 2 + 16) = empty ? -INFINITY : m + log2f(l);
      *reinterpret_cast<long long*>(dst + D * 2 + 24) = on ? grow : -1ll;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == QT_MMA_WARP) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(QT_TMEM_COLS));
  }
  const int col8 = lane & 15;
  if (col8 < D / 8) {
#pragma unroll 6
    for (int r = 2 * warp + (lane >> 4); r < TC_BM; r += 2 * (QT_THREADS / 32)) {
      const uint8_t* rowp = sQ + r * ROWB;
      const long long grow = *reinterpret_cast<const long long*>(rowp + D * 2 + 24);
      const float lse2 = *reinterpret_cast<const float*>(rowp + D * 2 + 16);
      const uint4 raw = *reinterpret_cast<const uint4*>(rowp + col8 * 16);
      if (grow < 0) continue;
      if (p.outer == 1) {
        *reinterpret_cast<uint4*>(p.out + grow * D + col8 * 8) = raw;
        if (p.lse && col8 == 0) p.lse[grow] = lse2 == -INFINITY ? 0.f : lse2 * kLn2;
      } else {
        uint4* po = reinterpret_cast<uint4*>(reinterpret_cast<char*>(p.part_o) + ((long long)split * rows_all + grow) * kPartRow<D>);
        po[col8] = raw;
        if (col8 == 0) po[D / 8] = *reinterpret_cast<const uint4*>(rowp + D * 2);
        if (col8 == 0) p.part_lse[(long long)split * rows_all + grow] = lse2;
      }
    }
  }
  if (warp == QT_LOAD_WARP && s_abort[0]) await_loads(s_bar, s_asked, tree_blocks, s_abort + 1);
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
  CUtensorMap kmap, vmap;
  int box_rows;
  const sb_status ms = make_code_maps<D>(p, TC_BN, &kmap, &vmap, &box_rows);
  if (ms != SB_OK) return ms;
  if (cudaLaunchKernelEx(&cfg, quant_tc_kernel<D>, p, kmap, vmap, box_rows) != cudaSuccess) {
    cudaGetLastError();
    return SB_ERR_CUDA;
  }
  return launch_check();
}

// grid = (chunks, KV heads x row tiles, sequences)
sb_status launch_quant_tc(const QuantAttnParams& p, dim3 grid, cudaStream_t cs) {
  return p.kv.head_dim == 64 ? launch_quant_tc_d<64>(p, grid, cs) : launch_quant_tc_d<128>(p, grid, cs);
}

}  // namespace sb
