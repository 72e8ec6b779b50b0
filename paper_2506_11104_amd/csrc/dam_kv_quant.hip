// dam_kv_quantize, dam_kv_dequantize: rows of K and V into a cache of 8-bit codes as they are made, and back.
//
// Mathematics: dam_quant.h. For a block of rows with the largest finite magnitude a among the new ones,
//   s = max(smallest s' with a <= c_max 2^(s' - 127), the block's scale if it holds rows in front of the new ones),
//   code = round(x 2^(127 - s)); the rows in front become round(code 2^(s_old - s)) where s has grown.
// Both are bound by HBM: 2 d (sizeof(T) + 1) bytes a row against a handful of operations per element.
//
// One workgroup writes one block of rows of K or V of one (sequence, KV head): the new rows are read once into registers
// (a row by d / 8 adjacent lanes), the largest magnitude goes through one barrier, and the codes are written from the
// registers. No two workgroups share a block, so nothing is atomic and the result does not depend on any order.
#include <hip/hip_bf16.h>

#include <algorithm>

#include "dam_internal.h"
#include "dam_mfma.h"
#include "dam_quant.h"
#include "dam_span.h"

namespace {
using namespace dam;

struct QuantArgs {
  int B, Hkv, cap, n_rows, pos;
  int n_blocks;         // blocks of the cache that n_rows rows can touch
  int64_t n_units;      // workgroups' items: (sequence, KV head, K or V, block)
  int64_t x_sb[2], x_sh[2], x_ss[2];  // element strides of k and v
  int64_t c_sb, c_sh, c_ss, s_sb, s_sh;
};

// Where the rows of sequence b go.
__device__ __forceinline__ Span span_of(const QuantArgs &a, int b, const int *start_at, const int *count_at) {
  return dam::span_of(start_at ? start_at[b] : a.pos, count_at ? count_at[b] : a.n_rows, a.n_rows, a.cap);
}

// Eight elements of a row as read, their largest magnitude (fp32 bits) and their codes.
template <typename T>
struct Part;

template <>
struct Part<float> {
  float4 v[2] = {};
  __device__ void load(const float *p) { v[0] = reinterpret_cast<const float4 *>(p)[0], v[1] = reinterpret_cast<const float4 *>(p)[1]; }
  __device__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) x[4 * i] = v[i].x, x[4 * i + 1] = v[i].y, x[4 * i + 2] = v[i].z, x[4 * i + 3] = v[i].w;
  }
  __device__ unsigned top() const {
    float x[8];
    values(x);
    unsigned t = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    return t;
  }
};

template <>
struct Part<__hip_bfloat16> {
  u32x4 v = {0u, 0u, 0u, 0u};
  __device__ void load(const __hip_bfloat16 *p) { v = *reinterpret_cast<const u32x4 *>(p); }
  __device__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
  __device__ unsigned top() const {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    u16x2 t = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned m = v[i] & 0x7FFF7FFFu;
      t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, m));
    }
    return (unsigned)max(t[0], t[1]) << 16;
  }
};

// x, divided by its scale s (not 0), as codes.
template <int FORMAT, typename T>
__device__ __forceinline__ uint2 encode(const Part<T> &x, unsigned s) {
  if constexpr (FORMAT == DAM_KV_E4M3 && sizeof(T) == 2) {
    if (s < Code<FORMAT>::kHuge) {  // (the whole block) two bf16 numbers at a time, divided on the way
      typedef __attribute__((ext_vector_type(2))) short s16x2;
      unsigned w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned lo = x.v[2 * i], hi = x.v[2 * i + 1];
        s16x2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, lo), scale_value(s), false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, hi), scale_value(s), true);
        w[i] = __builtin_bit_cast(unsigned, r);
      }
      return make_uint2(w[0], w[1]);
    }
  }
  float v[8];
  x.values(v);
  const float down = __uint_as_float((254u - s) << 23);  // 2^(127 - s)
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= down;
  return pack8<FORMAT>(v, s);
}

// The largest over the LPR adjacent lanes of a row, and over the rows of a wave from those.
template <int CTRL>
__device__ __forceinline__ unsigned max_with(unsigned x) {
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false));
}
template <int LPR>
__device__ __forceinline__ unsigned row_max(unsigned x) {
  x = max_with<0x141>(max_with<0x4E>(max_with<0xB1>(x)));  // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror
  return LPR == 16 ? max_with<0x140>(x) : x;               // row_mirror
}
template <int LPR>
__device__ __forceinline__ unsigned rows_max(unsigned x) {
  if (LPR == 8) x = max_with<0x128>(x);  // row_ror 8
  u32x2 sw = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(sw[0], sw[1]);
  sw = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(sw[0], sw[1]);
}

__device__ __forceinline__ void store8(float *p, const float *v) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__hip_bfloat16 *p, const float *v) {  // (exact but for values below 2^-126)
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

template <typename T, int FORMAT, int D, int BLK>
__global__ __launch_bounds__(256) void k_kv_quantize(QuantArgs a, const T *__restrict__ k, const T *__restrict__ v,
                                                     const int *__restrict__ start_at, const int *__restrict__ count_at,
                                                     uint8_t *kcache, uint8_t *vcache, uint8_t *kscale, uint8_t *vscale) {
  using C = Code<FORMAT>;
  constexpr int LPR = D / 8;                                // lanes per row
  constexpr int THREADS = BLK * LPR < 256 ? BLK * LPR : 256;
  constexpr int ROWS = THREADS / LPR, PASSES = BLK / ROWS;  // rows at a time
  __shared__ unsigned s_top[THREADS / 64 + 1];
  const int lane8 = threadIdx.x % LPR * 8, row0 = threadIdx.x / LPR;
  for (int64_t unit = blockIdx.x; unit < a.n_units; unit += gridDim.x) {
    const int nth = (int)(unit % a.n_blocks);
    const int64_t rest = unit / a.n_blocks;
    const int h = (int)(rest % a.Hkv), is_v = (int)(rest / a.Hkv % 2), b = (int)(rest / a.Hkv / 2);
    const Span span = span_of(a, b, start_at, count_at);
    const int block = nth_block(span, BLK, nth);
    if (block < 0) continue;        // (the whole workgroup)
    const int first = block * BLK;  // first row of the block
    const T *x = (is_v ? v : k) + b * a.x_sb[is_v] + h * a.x_sh[is_v] + lane8;
    uint8_t *codes = (is_v ? vcache : kcache) + b * a.c_sb + h * a.c_sh + first * a.c_ss + lane8;
    uint8_t *scale = (is_v ? vscale : kscale) + b * a.s_sb + h * a.s_sh + block;

    Part<T> x_new[PASSES];
    unsigned row_top[PASSES], top = 0;  // bits of the largest magnitude: of the row, of this lane's finite rows
    if (threadIdx.x == 0) s_top[THREADS / 64] = first < span.start ? *scale : 0u;  // (no rows in front: a new block)
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int rel = first + p * ROWS + row0 - span.start;  // row among the new ones
      if (rel >= 0 && rel < span.count) x_new[p].load(x + rel * a.x_ss[is_v]);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      row_top[p] = row_max<LPR>(x_new[p].top());
      if (row_top[p] < 0x7F800000u) top = max(top, row_top[p]);
    }
    top = rows_max<LPR>(top);
    if (threadIdx.x % 64 == 0) s_top[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, s_top[w]);
    const unsigned old = s_top[THREADS / 64], s = max(C::need(top), old);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int rel = first + p * ROWS + row0 - span.start;
      uint2 *at = reinterpret_cast<uint2 *>(codes + (int64_t)(p * ROWS + row0) * a.c_ss);
      if (rel >= 0 && rel < span.count) {
        const unsigned nan = C::kNan * 0x01010101u;
        uint2 c = encode<FORMAT>(x_new[p], max(s, 1u));  // (s = 0: zeros, of either sign)
        if (row_top[p] >= 0x7F800000u) c = make_uint2(nan, nan);
        *at = c;
      } else if (rel < 0 && s > old) {  // a row in front, to the larger scale
        const uint2 was = *at;
        if (!C::is_nan(was.x)) {
          float c[8];
          C::unpack4(was.x, c);
          C::unpack4(was.y, c + 4);
          const float shift = old ? ldexpf(1.0f, (int)old - (int)s) : 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] *= shift;
          *at = pack8<FORMAT>(c, s);
        }
      }
    }
    if (threadIdx.x == 0) *scale = (uint8_t)s;
    __syncthreads();  // s_top is taken again
  }
}

template <typename T, int FORMAT, int D>
__global__ __launch_bounds__(256) void k_kv_dequantize(QuantArgs a, int shift, const uint8_t *__restrict__ kcache,
                                                       const uint8_t *__restrict__ vcache, const uint8_t *__restrict__ kscale,
                                                       const uint8_t *__restrict__ vscale, const int *__restrict__ start_at,
                                                       const int *__restrict__ count_at, T *__restrict__ k, T *__restrict__ v) {
  using C = Code<FORMAT>;
  constexpr int LPR = D / 8, ROWS = 256 / LPR, PASSES = 4;
  const int lane8 = threadIdx.x % LPR * 8, row0 = threadIdx.x / LPR;
  for (int64_t unit = blockIdx.x; unit < a.n_units; unit += gridDim.x) {
    const int nth = (int)(unit % a.n_blocks);
    const int64_t rest = unit / a.n_blocks;
    const int h = (int)(rest % a.Hkv), is_v = (int)(rest / a.Hkv % 2), b = (int)(rest / a.Hkv / 2);
    const Span span = span_of(a, b, start_at, count_at);
    const uint8_t *codes = (is_v ? vcache : kcache) + b * a.c_sb + h * a.c_sh + lane8;
    const uint8_t *scale = (is_v ? vscale : kscale) + b * a.s_sb + h * a.s_sh;
    T *x = (is_v ? v : k) + b * a.x_sb[is_v] + h * a.x_sh[is_v] + lane8;
    uint2 c[PASSES];
    unsigned s[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int rel = (nth * PASSES + p) * ROWS + row0;
      if (rel < span.count) {
        c[p] = *reinterpret_cast<const uint2 *>(codes + (int64_t)(span.start + rel) * a.c_ss);
        s[p] = scale[(span.start + rel) >> shift];
      }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int rel = (nth * PASSES + p) * ROWS + row0;
      if (rel >= span.count) continue;
      float val[8];
      C::unpack4(c[p].x, val);
      C::unpack4(c[p].y, val + 4);
      const float f = C::is_nan(c[p].x) ? NAN : scale_value(s[p]);
#pragma unroll
      for (int e = 0; e < 8; ++e) val[e] *= f;
      store8(x + rel * a.x_ss[is_v], val);
    }
  }
}

constexpr int kMostRows = INT32_MAX - 1024;  // row numbers within a block that holds a row stay within 32 bits

// `write`: the caches and scales are written, else k and v are.
int validate(const dam_quant_params *p, const dam_quant_cache *c, const void *k, const void *v, bool write) {
  if (!p || !c || (p->n_rows != 0 && (!k || !v)) || !c->kcache || !c->vcache || !c->kscale || !c->vscale) return DAM_ERR_INVALID_ARG;
  if (p->batch < 1 || p->hkv < 1 || p->kv_capacity < 1 || p->n_rows < 0 || p->pos < 0 || p->pos > p->kv_capacity)
    return DAM_ERR_INVALID_ARG;
  if (p->kv_capacity > kMostRows || p->n_rows > kMostRows) return DAM_ERR_UNSUPPORTED;
  if (p->dtype != DAM_F32 && p->dtype != DAM_BF16) return DAM_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return DAM_ERR_UNSUPPORTED;
  if (!quant_format_ok(c->format, c->block)) return DAM_ERR_UNSUPPORTED;
  const int per16 = p->dtype == DAM_BF16 ? 8 : 4;
  for (int i = 0; i < 3; ++i)
    if (p->k_stride[i] < 0 || p->k_stride[i] % per16 || p->v_stride[i] < 0 || p->v_stride[i] % per16 || p->kv_stride[i] < 0 ||
        p->kv_stride[i] % 16)
      return DAM_ERR_INVALID_ARG;
  if (c->scale_stride[0] < 0 || c->scale_stride[1] < 0) return DAM_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(c->kcache) || !aligned16(c->vcache)) return DAM_ERR_INVALID_ARG;
  // what is written must not lie on top of itself
  const int n[3] = {p->batch, p->hkv, write ? p->kv_capacity : p->n_rows};
  for (int i = 0; i < 3; ++i) {
    if (n[i] < 2) continue;
    const int64_t least = i == 2 ? p->head_dim : 1;
    if (write ? p->kv_stride[i] < least || (i < 2 && c->scale_stride[i] < 1) : p->k_stride[i] < least || p->v_stride[i] < least)
      return DAM_ERR_INVALID_ARG;
  }
  return DAM_OK;
}

QuantArgs make_args(const dam_quant_params *p, const dam_quant_cache *c, int64_t n_blocks) {
  QuantArgs a;
  a.B = p->batch; a.Hkv = p->hkv; a.cap = p->kv_capacity; a.n_rows = p->n_rows; a.pos = p->pos;
  a.n_blocks = (int)n_blocks;
  a.n_units = n_blocks * p->hkv * 2 * p->batch;
  a.x_sb[0] = p->k_stride[0]; a.x_sh[0] = p->k_stride[1]; a.x_ss[0] = p->k_stride[2];
  a.x_sb[1] = p->v_stride[0]; a.x_sh[1] = p->v_stride[1]; a.x_ss[1] = p->v_stride[2];
  a.c_sb = p->kv_stride[0]; a.c_sh = p->kv_stride[1]; a.c_ss = p->kv_stride[2];
  a.s_sb = c->scale_stride[0]; a.s_sh = c->scale_stride[1];
  return a;
}

// (a launch holds fewer than 2^32 threads)
int grid_of(const QuantArgs &a) { return (int)std::min<int64_t>(a.n_units, 1 << 22); }

template <typename T, int FORMAT, int D, int BLK>
void quantize(const QuantArgs &a, const dam_quant_cache *c, const void *k, const void *v, const int32_t *start,
              const int32_t *count, hipStream_t st) {
  constexpr int THREADS = BLK * (D / 8) < 256 ? BLK * (D / 8) : 256;
  k_kv_quantize<T, FORMAT, D, BLK><<<grid_of(a), THREADS, 0, st>>>(
      a, static_cast<const T *>(k), static_cast<const T *>(v), start, count, static_cast<uint8_t *>(c->kcache),
      static_cast<uint8_t *>(c->vcache), c->kscale, c->vscale);
}

template <typename T, int FORMAT, int D>
void quantize_by_block(const QuantArgs &a, const dam_quant_cache *c, const void *k, const void *v, const int32_t *start,
                       const int32_t *count, hipStream_t st) {
  if (c->block == 16) quantize<T, FORMAT, D, 16>(a, c, k, v, start, count, st);
  else if (c->block == 32) quantize<T, FORMAT, D, 32>(a, c, k, v, start, count, st);
  else if (c->block == 64) quantize<T, FORMAT, D, 64>(a, c, k, v, start, count, st);
  else quantize<T, FORMAT, D, 128>(a, c, k, v, start, count, st);
}

template <typename T, int FORMAT, int D>
void dequantize(const QuantArgs &a, const dam_quant_cache *c, const int32_t *start, const int32_t *count, void *k, void *v,
                hipStream_t st) {
  const int shift = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
  k_kv_dequantize<T, FORMAT, D><<<grid_of(a), 256, 0, st>>>(
      a, shift, static_cast<const uint8_t *>(c->kcache), static_cast<const uint8_t *>(c->vcache), c->kscale, c->vscale, start,
      count, static_cast<T *>(k), static_cast<T *>(v));
}

}  // namespace

extern "C" int dam_kv_quantize(const dam_quant_params *p, const dam_quant_cache *cache, const void *k, const void *v,
                               const int32_t *start, const int32_t *count, void *stream_v) {
  const int bad = validate(p, cache, k, v, true);
  if (bad != DAM_OK) return bad;
  if (!start && !count && p->n_rows > p->kv_capacity - p->pos) return DAM_ERR_INVALID_ARG;
  if (p->n_rows == 0) return DAM_OK;
  const QuantArgs a = make_args(p, cache, most_blocks(p->n_rows, p->kv_capacity, cache->block));
  hipStream_t st = static_cast<hipStream_t>(stream_v);
  const bool e4m3 = cache->format == DAM_KV_E4M3, wide = p->head_dim == 128;
  if (p->dtype == DAM_BF16) {
    if (e4m3 && wide) quantize_by_block<__hip_bfloat16, DAM_KV_E4M3, 128>(a, cache, k, v, start, count, st);
    else if (e4m3) quantize_by_block<__hip_bfloat16, DAM_KV_E4M3, 64>(a, cache, k, v, start, count, st);
    else if (wide) quantize_by_block<__hip_bfloat16, DAM_KV_INT8, 128>(a, cache, k, v, start, count, st);
    else quantize_by_block<__hip_bfloat16, DAM_KV_INT8, 64>(a, cache, k, v, start, count, st);
  } else {
    if (e4m3 && wide) quantize_by_block<float, DAM_KV_E4M3, 128>(a, cache, k, v, start, count, st);
    else if (e4m3) quantize_by_block<float, DAM_KV_E4M3, 64>(a, cache, k, v, start, count, st);
    else if (wide) quantize_by_block<float, DAM_KV_INT8, 128>(a, cache, k, v, start, count, st);
    else quantize_by_block<float, DAM_KV_INT8, 64>(a, cache, k, v, start, count, st);
  }
  return launch_status();
}

extern "C" int dam_kv_dequantize(const dam_quant_params *p, const dam_quant_cache *cache, const int32_t *start,
                                 const int32_t *count, void *k, void *v, void *stream_v) {
  const int bad = validate(p, cache, k, v, false);
  if (bad != DAM_OK) return bad;
  if (!start && !count && p->n_rows > p->kv_capacity - p->pos) return DAM_ERR_INVALID_ARG;
  if (p->n_rows == 0) return DAM_OK;
  const int rows = 4 * 256 / (p->head_dim / 8);  // of a workgroup
  const QuantArgs a = make_args(p, cache, ((int64_t)p->n_rows + rows - 1) / rows);
  hipStream_t st = static_cast<hipStream_t>(stream_v);
  const bool e4m3 = cache->format == DAM_KV_E4M3, wide = p->head_dim == 128;
  if (p->dtype == DAM_BF16) {
    if (e4m3 && wide) dequantize<__hip_bfloat16, DAM_KV_E4M3, 128>(a, cache, start, count, k, v, st);
    else if (e4m3) dequantize<__hip_bfloat16, DAM_KV_E4M3, 64>(a, cache, start, count, k, v, st);
    else if (wide) dequantize<__hip_bfloat16, DAM_KV_INT8, 128>(a, cache, start, count, k, v, st);
    else dequantize<__hip_bfloat16, DAM_KV_INT8, 64>(a, cache, start, count, k, v, st);
  } else {
    if (e4m3 && wide) dequantize<float, DAM_KV_E4M3, 128>(a, cache, start, count, k, v, st);
    else if (e4m3) dequantize<float, DAM_KV_E4M3, 64>(a, cache, start, count, k, v, st);
    else if (wide) dequantize<float, DAM_KV_INT8, 128>(a, cache, start, count, k, v, st);
    else dequantize<float, DAM_KV_INT8, 64>(a, cache, start, count, k, v, st);
  }
  return launch_status();
}
