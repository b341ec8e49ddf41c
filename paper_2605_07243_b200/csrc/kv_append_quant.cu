// sb_kv_append_quant: bf16 rows become codes and scales of an 8-bit cache.
//
// For every block of scale_block tokens and KV head that receives rows
//   s = 2^ceil(log2(max|x| / 448)) over the new rows, at least 2^-100, at least the scale of older tokens in the block;
//   code = round_e4m3(x / s);   older code = round_e4m3(code * old / s) where s grew.
// e4m3 keeps four significant bits at every exponent, so a power of two loses nothing against max/448 but range at
// the bottom, and dividing by it is exact: a code is rounded once, and a later growth of the scale moves
// the older codes by whole exponents (they lose bits only below 2^-6).
//
// Bound by memory: 2 bytes read and 1 written per element.  One CTA owns one (block, head, K or V): the maximum
// needs the whole block before the first code can be written, and 128 tokens x 128 elements are 64 values a
// thread, which stay in registers between the two steps.  Elements past the new rows are never touched.
#include "quant_common.cuh"

namespace sb {

constexpr int AP_THREADS = 256;

struct AppendParams {
  sb_quant_cache kv;
  const uint16_t* rows[2];  // K, V
  long long row_stride, rows_layer_stride;
  const int* row_offsets;
  int total_rows;
  const int* path_nodes;
  const int* accept_len;
  int max_depth, max_rows;
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

template <int D>
__global__ void __launch_bounds__(AP_THREADS) kv_append_quant_kernel(const AppendParams p) {
  constexpr int LPR = D / 8;              // lanes per row: 8 elements (16 bytes of bf16) each
  constexpr int RPP = AP_THREADS / LPR;   // rows per pass
  constexpr int PASSES = 128 / RPP;
  __shared__ int s_path[SB_MAX_DEPTH + 1];
  __shared__ int s_err;
  __shared__ uint32_t s_max[AP_THREADS / 32];
  pdl_wait();
  pdl_release();
  const int H = p.kv.n_kv_heads, sb = p.kv.scale_block;
  const int tid = threadIdx.x;
  const int b = blockIdx.z % p.kv.batch, layer = blockIdx.z / p.kv.batch;
  const int which = blockIdx.y & 1, g = blockIdx.y >> 1;
  const int start = p.len[b];
  const int o = p.row_offsets[b];
  const int avail = p.row_offsets[b + 1] - o;
  int n = p.path_nodes ? p.accept_len[b] + 1 : avail;
  int err = 0;
  if (o < 0 || avail < 0 || (long long)o + avail > p.total_rows || n < 0 || n > p.max_rows ||
      (p.path_nodes && (n < 1 || n > p.max_depth + 1)))
    err = SB_ERR_INVALID_TREE;
  const long long cap = p.kv.page_size == 0 ? p.kv.kv_capacity : (long long)p.kv.max_pages * p.kv.page_size;
  if (!err && (start < 0 || (long long)start + n > cap)) err = SB_ERR_BOUNDS;
  if (tid == 0) s_err = err;
  __syncthreads();
  if (!err) {
    if (p.path_nodes && tid < n) {
      const int* path = p.path_nodes + (long long)b * (p.max_depth + 1);
      const int self = path[tid];
      s_path[tid] = self;
      if (self < 0 || self >= avail || (tid > 0 && path[tid - 1] >= self)) s_err = SB_ERR_INVALID_TREE;
    }
    if (p.kv.page_size > 0 && n > 0) {
      const int first = start / p.kv.page_size, last = (start + n - 1) / p.kv.page_size;
      for (int lp = first + tid; lp <= last; lp += AP_THREADS) {
        const int page = p.kv.page_table[(long long)b * p.kv.max_pages + lp];
        if (page < 0 || page >= p.kv.num_pages) atomicMax(&s_err, (int)SB_ERR_BOUNDS);
      }
    }
  }
  __syncthreads();
  err = s_err;
  if (blockIdx.x == 0 && blockIdx.y == 0 && layer == 0 && tid == 0) {
    p.status[b] = err;
    p.new_len[b] = err ? start : start + n;
  }
  if (err || n == 0) return;
  const int block = start / sb + blockIdx.x;                 // block of tokens of this sequence
  const long long t0 = (long long)block * sb;
  if (t0 >= (long long)start + n) return;
  const int lo = (int)(t0 > start ? t0 : start) - (int)t0;    // new rows of the block: [lo, hi)
  const int hi = (int)min((long long)start + n - t0, (long long)sb);

  const long long row0 = quant_row(p.kv, b, (int)t0);         // the block lies inside one page
  uint8_t* codes = static_cast<uint8_t*>(which ? p.kv.v_codes : p.kv.k_codes) + layer * p.kv.codes_layer_stride;
  float* scale = (which ? p.kv.v_scale : p.kv.k_scale) + layer * p.kv.scale_layer_stride + (row0 / sb) * H + g;
  const uint16_t* src = p.rows[which] + layer * p.rows_layer_stride;
  const int r_in = tid / LPR, col = (tid % LPR) * 8;

  uint4 x[PASSES];
  uint32_t amax = 0;  // magnitudes order like integers; a NaN or an infinity is >= 0x7F80
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * RPP + r_in;
    x[i] = make_uint4(0, 0, 0, 0);
    if (r >= lo && r < hi) {
      const int j = (int)(t0 + r - start);
      const long long row = o + (p.path_nodes ? s_path[j] : j);
      if (SB_CHECKED_ACCESS(row, p.total_rows, &p.status[b]))
        x[i] = *reinterpret_cast<const uint4*>(src + row * p.row_stride + (long long)g * D + col);
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        amax = max(amax, w[k] & 0x7FFFu);
        amax = max(amax, (w[k] >> 16) & 0x7FFFu);
      }
    }
  }
  amax = __reduce_max_sync(0xffffffffu, amax);
  if ((tid & 31) == 0) s_max[tid >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < AP_THREADS / 32; ++i) amax = max(amax, s_max[i]);
  const bool bad = amax >= 0x7F80u;
  if (bad) {  // rare: the finite elements still get a scale of their own
    uint32_t fin = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((w[k] & 0x7F80u) == 0x7F80u) w[k] &= 0xFFFF0000u;
        if ((w[k] & 0x7F800000u) == 0x7F800000u) w[k] &= 0xFFFFu;
        fin = max(fin, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
      }
      x[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    fin = __reduce_max_sync(0xffffffffu, fin);
    __syncthreads();
    if ((tid & 31) == 0) s_max[tid >> 5] = fin;
    __syncthreads();
    amax = 0;
#pragma unroll
    for (int i = 0; i < AP_THREADS / 32; ++i) amax = max(amax, s_max[i]);
  }
  float s = __uint_as_float((uint32_t)(scale_exponent(amax << 16) + 127) << 23);
  const float old = lo > 0 ? *scale : 0.f;  // older tokens share the block
  const bool was_bad = old != old;
  if (!was_bad && old > s) s = old;
  __syncthreads();                          // every thread has read the old scale
  if (tid == 0) *scale = (bad || was_bad) ? __uint_as_float(0x7FC00000u) : s;
  // Powers of two divide exactly by their reciprocal; an older scale of another writer may be any number.
  const float inv = 1.f / s;
  const bool exact_inv = (__float_as_uint(s) & 0x7FFFFFu) == 0;
  const bool grow = lo > 0 && !was_bad && old != s;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * RPP + r_in;
    if (r >= hi) break;
    const long long off = ((row0 + r) * H + g) * (long long)D + col;
    if (!SB_CHECKED_ACCESS(off + 7, quant_rows_total(p.kv) * H * D, &p.status[b])) continue;
    if (r >= lo) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint16_t c[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a0 = __uint_as_float(w[k] << 16), a1 = __uint_as_float(w[k] & 0xFFFF0000u);
        c[k] = exact_inv ? e4m3x2_of(a0 * inv, a1 * inv) : e4m3x2_of(a0 / s, a1 / s);
      }
      *reinterpret_cast<uint2*>(codes + off) = make_uint2(c[0] | ((uint32_t)c[1] << 16), c[2] | ((uint32_t)c[3] << 16));
    } else if (grow) {
      const uint2 was = *reinterpret_cast<const uint2*>(codes + off);
      const uint32_t w[2] = {was.x, was.y};
      uint32_t out[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint16_t c[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 v = float2_of_e4m3x2((uint16_t)(w[k] >> (16 * e)));
          c[e] = e4m3x2_of(v.x * old / s, v.y * old / s);
        }
        out[k] = c[0] | ((uint32_t)c[1] << 16);
      }
      *reinterpret_cast<uint2*>(codes + off) = make_uint2(out[0], out[1]);
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
  p.len = len;
  p.new_len = new_len;
  p.status = status;
  const long long zs = (long long)kv->batch * kv->n_layers, ys = 2LL * kv->n_kv_heads;
  if (zs > 65535 || ys > 65535) return SB_ERR_UNSUPPORTED;
  const int most = path_nodes && max_depth + 1 < max_rows ? max_depth + 1 : max_rows;
  // blocks that `most` rows can touch, whatever the offset of the first
  const dim3 grid(((unsigned)most + kv->scale_block - 2) / kv->scale_block + 1, (unsigned)ys, (unsigned)zs);
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  return kv->head_dim == 64 ? launch_dependent(kv_append_quant_kernel<64>, grid, dim3(AP_THREADS), cs, p)
                            : launch_dependent(kv_append_quant_kernel<128>, grid, dim3(AP_THREADS), cs, p);
}
