// sb_kv_append_quant: bf16 rows become codes and scales of an 8-bit cache.
//
// For every block of scale_block tokens and KV head that receives rows
//   s = 2^ceil(log2(max|x| / 448)) over the new rows, at least 2^-100, at least the scale of older tokens in the block;
//   code = round_e4m3(x / s);   older code = round_e4m3(code * old / s) where s grew.
// e4m3 keeps four significant bits at every exponent, so a power of two loses nothing against max/448 but range at
// the bottom, and dividing by it is exact: a code is rounded once, and a later growth of the scale moves
// the older codes by whole exponents (they lose bits only below 2^-6).
//
// Bound by memory for prompts: 2 bytes read and 1 written per element.  A unit of work is one (block, head, K or V): the maximum
// needs the whole block before the first code can be written, so the new rows stay in registers between the two
// steps, 64 elements a thread.  Prompts: 2 * scale_block threads per unit, and many units on an SM hide one
// another's chain of dependent loads (lengths, rows and page ids, old scale).  Four prompts of 2000 to 8192 tokens: 31 us, 4.0 TB/s;
// without the stores 21 us, the launch alone 9.  Up to 16 rows (a verified step): one warp per unit; there the chain is all there
// is, and a commit has thousands of units of a few hundred bytes: 16 sequences, 32 layers 11.4 us, of which the launch and the chain up
// to the rows take 5.  (One warp for both blocks that a path may touch, instead of a warp each of which the second mostly finds
// nothing to do: 12.6.)  Row loads go out before the page ids are looked at.  Elements past the new rows are never touched.
#include "quant_common.cuh"

namespace sb {

struct AppendParams {
  sb_quant_cache kv;
  const uint16_t* rows[2];  // K, V
  long long row_stride, rows_layer_stride;
  const int* row_offsets;
  int total_rows;
  const int* path_nodes;
  const int* accept_len;
  int max_depth, max_rows;
  int block_shift;          // log2 of the tokens per block
  const int* len;
  int* new_len;
  int* status;
};

// The scale exponent of a maximum given as fp32 bits: smallest e with amax <= 448 * 2^e = 1.75 * 2^(e+8), >= -100.
__device__ inline int scale_exponent(uint32_t amax_bits) {
  const int ex = (int)(amax_bits >> 23) - 127;  // a subnormal maximum lands far below -100
  const int e = ex - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < -100 ? -100 : e;
}

// Eight bf16 values times a factor (or over a divisor) -> eight codes.
__device__ inline uint2 codes_times(const uint4& x, float f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) c[k] = e4m3x2_of(__uint_as_float(w[k] << 16) * f, __uint_as_float(w[k] & 0xFFFF0000u) * f);
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
static __device__ __noinline__ uint2 codes_over(uint4 x, float s) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) c[k] = e4m3x2_of(__uint_as_float(w[k] << 16) / s, __uint_as_float(w[k] & 0xFFFF0000u) / s);
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
// Eight codes under another scale.
static __device__ __noinline__ uint2 rescaled(uint2 v, float old, float s) {
  const uint32_t w[2] = {v.x, v.y};
  uint32_t out[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float2 a = float2_of_e4m3x2((uint16_t)w[k]), b = float2_of_e4m3x2((uint16_t)(w[k] >> 16));
    out[k] = e4m3x2_of(a.x * old / s, a.y * old / s) | ((uint32_t)e4m3x2_of(b.x * old / s, b.y * old / s) << 16);
  }
  return make_uint2(out[0], out[1]);
}

// UT threads to a unit.  A CTA has 256 threads whatever the unit: 20,000 prompt tokens in blocks of 64 are 5000 units of 128 threads, and
// starting a CTA for each took 9 of 33 us (31 so; 384 and 512 threads 35.6 and 33).
constexpr int kAppendThreads = 256;
template <int D, int UT>
__global__ void __launch_bounds__(kAppendThreads, 4) kv_append_quant_kernel(const AppendParams p) {
  constexpr int LPR = D / 8;              // lanes per row: 8 elements (16 bytes of bf16) each
  constexpr int RPP = UT / LPR;           // rows per pass
  constexpr int ROWS = UT == 32 ? 16 : UT / 2;
  constexpr int PASSES = ROWS / RPP;
  constexpr int UNITS = kAppendThreads / UT;
  __shared__ int s_path[UNITS][SB_MAX_DEPTH + 1];
  __shared__ uint32_t s_max[UNITS][UT / 32];
  const int H = p.kv.n_kv_heads, sb = p.kv.scale_block;
  const int tid = threadIdx.x % UT, slot = threadIdx.x / UT;
  auto sync = [slot]() {
    if (UT == 32) __syncwarp();
    else asm volatile("barrier.sync %0, %1;" ::"r"(slot + 1), "n"(UT) : "memory");
  };
  // the same value in every thread of the unit; shared memory that the unit wrote before is complete behind it
  auto any = [slot](bool v) {
    if (UT == 32) {
      __syncwarp();  // a vote alone orders no memory
      return __any_sync(0xffffffffu, v) != 0;
    }
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(r)
        : "r"((uint32_t)v), "r"(slot + 1), "n"(UT)
        : "memory");
    return r != 0;
  };
  pdl_wait();
  pdl_release();
  const int b = blockIdx.y, layer = blockIdx.z;
  const int unit = blockIdx.x * UNITS + slot, which = unit & 1, g = (unit >> 1) % H, nth = (unit >> 1) / H;
  const int start = p.len[b];
  const int o = p.row_offsets[b];
  const int avail = p.row_offsets[b + 1] - o;
  const int n = p.path_nodes ? p.accept_len[b] + 1 : avail;
  int err = 0;
  if (o < 0 || avail < 0 || (long long)o + avail > p.total_rows || n < 0 || n > p.max_rows ||
      (p.path_nodes && (n < 1 || n > p.max_depth + 1)))
    err = SB_ERR_INVALID_TREE;
  const long long cap = p.kv.page_size == 0 ? p.kv.kv_capacity : (long long)p.kv.max_pages * p.kv.page_size;
  if (!err && (start < 0 || (long long)start + n > cap)) err = SB_ERR_BOUNDS;
  const bool first_unit = unit == 0 && layer == 0;
  const int block = err ? 0 : (start >> p.block_shift) + nth; // block of tokens of this sequence
  const long long t0 = (long long)block << p.block_shift;
  const bool mine = !err && t0 < (long long)start + n;
  if (!mine && !first_unit) return;                           // (the first unit has the sequence's status to write)
  if (!err && p.path_nodes) {
    const int* path = p.path_nodes + (long long)b * (p.max_depth + 1);
    bool bad = false;
    for (int i = tid; i < n; i += UT) {
      const int self = path[i];
      s_path[slot][i] = self;
      bad |= self < 0 || self >= avail || (i > 0 && path[i - 1] >= self);
    }
    if (any(bad)) err = SB_ERR_INVALID_TREE;                  // (s_path is complete from here on)
  }
  const int lo = (int)(t0 > start ? t0 : start) - (int)t0;    // new rows of the block: [lo, hi)
  const int hi = mine ? (int)min((long long)start + n - t0, (long long)sb) : 0;
  const int r_in = tid / LPR, col = (tid % LPR) * 8;
  // Registers hold rows base + i * RPP + r_in; a warp's 16 rows start at the first new one.
  const int base = UT == 32 ? lo : 0;
  const uint16_t* src = p.rows[which] + layer * p.rows_layer_stride;

  const unsigned n_new = !err && hi > lo ? hi - lo : 0;       // row r of the block is new iff r - lo < n_new
  uint4 x[PASSES];
  if (p.path_nodes) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = base + i * RPP + r_in;
      x[i] = make_uint4(0, 0, 0, 0);
      if ((unsigned)(r - lo) < n_new) {
        const long long row = o + s_path[slot][(int)(t0 - start) + r];
        if (SB_CHECKED_ACCESS(row, p.total_rows, &p.status[b]))
          x[i] = __ldcs(reinterpret_cast<const uint4*>(src + row * p.row_stride + (long long)g * D + col));
      }
    }
  } else {
    const long long row_a = o + (t0 - start) + base + r_in;
    const uint16_t* from = src + row_a * p.row_stride + (long long)g * D + col;
    const long long pass = RPP * p.row_stride;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      x[i] = make_uint4(0, 0, 0, 0);
      if ((unsigned)(base + i * RPP + r_in - lo) < n_new && SB_CHECKED_ACCESS(row_a + i * RPP, p.total_rows, &p.status[b]))
        x[i] = __ldcs(reinterpret_cast<const uint4*>(from + i * pass));
    }
  }
  if (!err && p.kv.page_size > 0 && n > 0) {
    const int shift = 31 - __clz(p.kv.page_size);
    bool bad = false;
    for (int lp = (start >> shift) + tid; lp <= (start + n - 1) >> shift; lp += UT) {
      const int page = p.kv.page_table[(long long)b * p.kv.max_pages + lp];
      bad |= page < 0 || page >= p.kv.num_pages;
    }
    if (any(bad)) err = SB_ERR_BOUNDS;
  }
  if (first_unit && tid == 0) {
    p.status[b] = err;
    p.new_len[b] = err ? start : start + n;
  }
  if (err || !mine || hi <= lo) return;

  const long long row0 = quant_row(p.kv, b, (int)t0);         // the block lies inside one page
  uint8_t* codes = static_cast<uint8_t*>(which ? p.kv.v_codes : p.kv.k_codes) + layer * p.kv.codes_layer_stride;
  float* scale = (which ? p.kv.v_scale : p.kv.k_scale) + layer * p.kv.scale_layer_stride + (row0 >> p.block_shift) * H + g;
  const float old = lo > 0 ? *scale : 0.f;                    // older tokens share the block
  // magnitudes order like integers; a NaN or an infinity is >= 0x7F80
  auto unit_max = [&]() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) m = __vmaxu2(m, w[k] & 0x7FFF7FFFu);  // both halves at once
    }
    m = __reduce_max_sync(0xffffffffu, max(m & 0xFFFFu, m >> 16));
    if (UT > 32) {
      sync();
      if ((tid & 31) == 0) s_max[slot][tid >> 5] = m;
      sync();
#pragma unroll
      for (int i = 0; i < UT / 32; ++i) m = max(m, s_max[slot][i]);
    }
    return m;
  };
  uint32_t amax = unit_max();
  const bool bad = amax >= 0x7F80u;
  if (bad) {  // rare: the finite elements still get a scale of their own
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((w[k] & 0x7F80u) == 0x7F80u) w[k] &= 0xFFFF0000u;
        if ((w[k] & 0x7F800000u) == 0x7F800000u) w[k] &= 0xFFFFu;
      }
      x[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    amax = unit_max();
  }
  float s = __uint_as_float((uint32_t)(scale_exponent(amax << 16) + 127) << 23);
  const bool was_bad = old != old;
  if (!was_bad && old > s) s = old;
  sync();                                   // every thread has read the old scale
  if (tid == 0) *scale = (bad || was_bad) ? __uint_as_float(0x7FC00000u) : s;
  // Powers of two divide exactly by their reciprocal; an older scale of another writer may be any number.
  const float inv = 1.f / s;
  const bool exact = (__float_as_uint(s) & 0x7FFFFFu) == 0;
  uint8_t* dst = codes + ((row0 + base + r_in) * H + g) * (long long)D + col;
  const long long pass_bytes = (long long)RPP * H * D;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = base + i * RPP + r_in;
    if ((unsigned)(r - lo) < n_new && SB_CHECKED_ACCESS(((row0 + r) * H + g) * D + col + 7, quant_rows_total(p.kv) * H * D, &p.status[b]))
      *reinterpret_cast<uint2*>(dst + i * pass_bytes) = exact ? codes_times(x[i], inv) : codes_over(x[i], s);
  }
  if (lo > 0 && !was_bad && old != s) {     // the scale grew: the older codes follow
#pragma unroll 4
    for (int r = r_in; r < lo; r += RPP) {
      const long long off = ((row0 + r) * H + g) * (long long)D + col;
      if (!SB_CHECKED_ACCESS(off + 7, quant_rows_total(p.kv) * H * D, &p.status[b])) continue;
      uint2* at = reinterpret_cast<uint2*>(codes + off);
      *at = rescaled(*at, old, s);
    }
  }
}

}  // namespace sb

extern "C" sb_status sb_kv_append_quant(const sb_quant_cache* kv, const void* k_rows, const void* v_rows,
                                        int64_t row_stride, int64_t rows_layer_stride, const int32_t* row_offsets,
                                        int32_t total_rows, const int32_t* path_nodes, const int32_t* accept_len,
                                        int32_t max_depth, int32_t max_rows, const int32_t* len, int32_t* new_len,
                                        int32_t* status, void* stream) {
  sb::TraceRange trace_range("sb_kv_append_quant");
  using namespace sb;
  const sb_status st = check_quant_cache(kv);
  if (st != SB_OK) return st;
  if (!k_rows || !v_rows || !row_offsets || !len || !new_len || !status || new_len == len || total_rows < 0 || max_rows < 1)
    return SB_ERR_INVALID_ARG;
  if ((path_nodes == nullptr) != (accept_len == nullptr)) return SB_ERR_INVALID_ARG;
  if (path_nodes && (max_depth < 0 || max_depth > SB_MAX_DEPTH)) return SB_ERR_UNSUPPORTED;
  const int64_t width = (int64_t)kv->n_kv_heads * kv->head_dim;
  if (row_stride == 0) row_stride = width;
  if (row_stride < width || row_stride % 8 != 0 || rows_layer_stride < 0 || rows_layer_stride % 8 != 0) return SB_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_rows) & 15) || (reinterpret_cast<uintptr_t>(v_rows) & 15)) return SB_ERR_INVALID_ARG;
  // layers that overlap would be written by several CTAs at once
  if (kv->n_layers > 1 && (kv->codes_layer_stride < quant_rows_total(*kv) * width ||
                           kv->scale_layer_stride < quant_rows_total(*kv) / kv->scale_block * kv->n_kv_heads))
    return SB_ERR_INVALID_ARG;
  AppendParams p;
  p.kv = *kv;
  p.rows[0] = static_cast<const uint16_t*>(k_rows);
  p.rows[1] = static_cast<const uint16_t*>(v_rows);
  p.row_stride = row_stride;
  p.rows_layer_stride = rows_layer_stride;
  p.row_offsets = row_offsets;
  p.total_rows = total_rows;
  p.path_nodes = path_nodes;
  p.accept_len = accept_len;
  p.max_depth = max_depth;
  p.max_rows = max_rows;
  p.block_shift = 31 - __builtin_clz((unsigned)kv->scale_block);
  p.len = len;
  p.new_len = new_len;
  p.status = status;
  if (kv->n_layers > 65535 || kv->batch > 65535) return SB_ERR_UNSUPPORTED;
  const int most = path_nodes && max_depth + 1 < max_rows ? max_depth + 1 : max_rows;
  const int sb = kv->scale_block;
  // blocks that `most` rows can touch, whatever the offset of the first
  const long long units = (((long long)most + sb - 2) / sb + 1) * 2 * kv->n_kv_heads;
  if (units > 0x7fffffffLL) return SB_ERR_UNSUPPORTED;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  auto launch = [&](auto kernel, int unit_threads) {
    const int per_cta = kAppendThreads / unit_threads;
    return launch_dependent(kernel, dim3((unsigned)((units + per_cta - 1) / per_cta), kv->batch, kv->n_layers), dim3(kAppendThreads), cs, p);
  };
  const bool d64 = kv->head_dim == 64;
  if (most <= 16 || sb == 16) return d64 ? launch(kv_append_quant_kernel<64, 32>, 32) : launch(kv_append_quant_kernel<128, 32>, 32);
  if (sb == 32) return d64 ? launch(kv_append_quant_kernel<64, 64>, 64) : launch(kv_append_quant_kernel<128, 64>, 64);
  if (sb == 64) return d64 ? launch(kv_append_quant_kernel<64, 128>, 128) : launch(kv_append_quant_kernel<128, 128>, 128);
  return d64 ? launch(kv_append_quant_kernel<64, 256>, 256) : launch(kv_append_quant_kernel<128, 256>, 256);
}
