// The decodes over a KV cache of 8-bit codes (dam_quant.h): one query row per (sequence, query head) over a list of kept
// keys of its own, over the merged list of its KV head's query heads, or over a plan of the matched patterns.
//
// Paper (arXiv 2506.11104): Sec. 3 (scaled dot-product attention) with the mask of Sec. 4.3 applied as -inf before the
// softmax. With the scales f_j, g_j of key j's rows:
//   z_j = (sum_d q_d kcode_jd) f_j scale log2 e,   w_j = 2^(z_j - m),   O = sum_j (w_j g_j) vcode_j / sum_j w_j.
//
// HBM bound: 2 d bytes per kept key. A row is read by LPR adjacent lanes (16 codes each, 8 in the grouped forms), a lane
// keeps four keys in flight, and the arithmetic is that of the codes: a row's scale enters once per row, not per element.
// A list is split over workgroups where the lists alone do not fill the chip, and the last workgroup of a list to finish
// merges its splits.
#include <hip/hip_bf16.h>
#include <math.h>

#include <algorithm>

#include "dam_internal.h"
#include "dam_quant.h"
#include "dam_splits.h"

namespace {
using namespace dam;

constexpr int kUnroll = 4;  // keys in flight per lane

struct QDecodeArgs {
  int B, Hq, Hkv, cap, shared_lists;
  int rows_of_kv;   // lists per KV head: query heads with a list each, or 1 merged list
  int G;            // query heads per list
  int splits;
  int block_shift;  // log2 of the rows that share a scale
  int pos, n_flags; // plans
  uint64_t flag;    // of this call (arrive_last)
  float scale;
  int64_t q_sb, q_sh, kv_sb, kv_sh, kv_ss, s_sb, s_sh, o_sb, o_sh;
};

template <int N>
__device__ __forceinline__ void load_q(const float *p, float *v) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 a = *reinterpret_cast<const float4 *>(p + i);
    v[i] = a.x, v[i + 1] = a.y, v[i + 2] = a.z, v[i + 3] = a.w;
  }
}
template <int N>
__device__ __forceinline__ void load_q(const __hip_bfloat16 *p, float *v) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p + i);
    const unsigned u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[i + 2 * k] = __uint_as_float(u[k] << 16), v[i + 2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ void store_out(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_out(__hip_bfloat16 *p, float v) { *p = __float2bfloat16(v); }

// N codes of a row as loaded.
template <int N>
struct Codes {
  unsigned w[N / 4];
  __device__ void load(const uint8_t *p) {
    if constexpr (N == 16) {
      const uint4 a = *reinterpret_cast<const uint4 *>(p);
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
      const uint2 a = *reinterpret_cast<const uint2 *>(p);
      w[0] = a.x, w[1] = a.y;
    }
  }
};

// The result of a list's G heads: O [head][D] unnormalised, reference (log2 units) and sum of weights. L = 0: nothing kept.
template <typename T>
__device__ __forceinline__ void finish(const QDecodeArgs &a, int b, int hq, int dim, float o, float M, float L, T *out,
                                       float *lse) {
  store_out(out + b * a.o_sb + hq * a.o_sh + dim, L == 0.0f ? 0.0f : o / L);
  if (lse && dim == 0) lse[(int64_t)b * a.Hq + hq] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// GM: most query heads of a list the registers are laid out for (1: a list per query head, no member bits).
template <typename T, int FORMAT, int D, int GM, bool PLAN>
__global__ __launch_bounds__(256) void k_decode_quant(
    QDecodeArgs a, const T *__restrict__ q, const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
    const uint8_t *__restrict__ ks, const uint8_t *__restrict__ vs, const int *__restrict__ kept_ptr,
    const int *__restrict__ kept_idx, const uint8_t *__restrict__ kept_member, const uint8_t *__restrict__ plan_table,
    float *__restrict__ part_o, float *__restrict__ part_ml, uint64_t *__restrict__ flags, T *__restrict__ out,
    float *__restrict__ lse) {
  using C = Code<FORMAT>;
  constexpr int N = GM == 1 ? 16 : 8;  // codes of a row per lane
  constexpr int LPR = D / N, GROUPS = 256 / LPR;
  __shared__ float s_o[GROUPS][D];
  __shared__ float s_m[GROUPS], s_l[GROUPS];
  __shared__ int s_last;

  // XCD-aware numbering: block n runs on XCD n % 8; all lists and splits of one (sequence, KV head) pair have ids with
  // the same n % 8, so that heads with lists of their own find the rows they share in one L2.
  const int per_pair = a.rows_of_kv * a.splits;
  const int slot = (int)blockIdx.x / kXcd, pair = slot / per_pair * kXcd + (int)blockIdx.x % kXcd;
  if (pair >= a.B * a.Hkv) return;
  const int within = slot % per_pair, nth = within / a.splits, split = within % a.splits;
  const int b = pair / a.Hkv, hkv = pair % a.Hkv;
  const int row = hkv * a.rows_of_kv + nth;            // list of the sequence
  const int n_rows = a.Hkv * a.rows_of_kv;
  const int item = b * n_rows + row;
  const int list = a.shared_lists ? row : item;
  const int hq0 = row * a.G;                           // first query head
  const int group = threadIdx.x / LPR, sub = threadIdx.x % LPR;
  const int64_t end = kept_ptr[list + 1];
  const int64_t stride = (int64_t)a.splits * GROUPS * kUnroll;

  float qf[GM][N];
#pragma unroll
  for (int x = 0; x < GM; ++x) {
#pragma unroll
    for (int e = 0; e < N; ++e) qf[x][e] = 0.0f;
    if (x < a.G) load_q<N>(q + b * a.q_sb + (hq0 + x) * a.q_sh + sub * N, qf[x]);
  }
  const uint8_t *kb = kc + b * a.kv_sb + hkv * a.kv_sh + sub * N, *vb = vc + b * a.kv_sb + hkv * a.kv_sh + sub * N;
  const uint8_t *ksb = ks + b * a.s_sb + hkv * a.s_sh, *vsb = vs + b * a.s_sb + hkv * a.s_sh;
  const uint8_t *table = PLAN ? plan_table + (int64_t)hkv * a.n_flags : nullptr;
  const float sl2 = a.scale * 1.4426950408889634f;  // logits in log2 units

  float m[GM], l[GM], o[GM][N];
#pragma unroll
  for (int x = 0; x < GM; ++x) {
    m[x] = -INFINITY;
    l[x] = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) o[x][e] = 0.0f;
  }

  int rows[kUnroll];
  unsigned who[kUnroll];  // member bits; 0 past the end of the list
  int64_t p0 = kept_ptr[list] + ((int64_t)split * GROUPS + group) * kUnroll;
  auto fetch = [&](int64_t at) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool ok = at + u < end;
      rows[u] = at < end ? kept_idx[ok ? at + u : at] : 0;
      who[u] = ok ? (GM == 1 && !PLAN && !kept_member ? 1u : kept_member[at + u]) : 0u;
    }
  };
  fetch(p0);
  for (; p0 < end; p0 += stride) {
    Codes<N> kf[kUnroll], vf[kUnroll];
    float kscale[kUnroll], vscale[kUnroll];
    unsigned cur[kUnroll], anyone = 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      int r = rows[u];
      cur[u] = who[u];
      if (PLAN) {
        // entry -1 - r: key pos - r; entry c >= 0: key c, for the heads that do not reach it through a diagonal. A key
        // that does not exist yet serves no head, and its row is taken from those that do.
        const int t = a.pos - r;
        if (r >= 0 && t >= 0 && t < a.n_flags) cur[u] &= ~(unsigned)table[t];
        if (r < 0) r += a.pos + 1;
        if (r < 0 || r > a.pos) cur[u] = 0;
        r = min(max(r, 0), a.pos);
      }
      r = in_cache(r, a.cap);
      kf[u].load(kb + r * a.kv_ss);
      vf[u].load(vb + r * a.kv_ss);
      kscale[u] = scale_value(ksb[r >> a.block_shift]);
      vscale[u] = scale_value(vsb[r >> a.block_shift]);
      anyone |= cur[u];
    }
    if (p0 + stride < end) fetch(p0 + stride);
    // NaN rows: the scale carries the NaN, so that it reaches the heads that keep the row alone
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (C::is_nan(kf[u].w[0])) kscale[u] = NAN;
      if (C::is_nan(vf[u].w[0])) {
        vscale[u] = NAN;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) vf[u].w[i] = 0u;
      }
    }
#pragma unroll
    for (int x = 0; x < GM; ++x) {
      if (x < a.G && __ballot((anyone >> x) & 1)) {  // some entry of this wave's pass is kept by head x
        float s[kUnroll];
        float mx = m[x];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          float d = 0.0f, c[4];
#pragma unroll
          for (int i = 0; i < N / 4; ++i) {
            C::unpack4(kf[u].w[i], c);
#pragma unroll
            for (int e = 0; e < 4; ++e) d = fmaf(qf[x][4 * i + e], c[e], d);
          }
          s[u] = (cur[u] >> x) & 1 ? row_sum<LPR>(d) * kscale[u] * sl2 : -INFINITY;
          mx = fmaxf(mx, s[u]);
        }
        const float ref = mx == -INFINITY ? 0.0f : mx;  // (none of the lane's keys so far is this head's)
        const float corr = __builtin_amdgcn_exp2f(m[x] - ref);
        l[x] *= corr;
#pragma unroll
        for (int e = 0; e < N; ++e) o[x][e] *= corr;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const float w = __builtin_amdgcn_exp2f(s[u] - ref);
          l[x] += w;
          const float wv = (cur[u] >> x) & 1 ? w * vscale[u] : 0.0f;
          float c[4];
#pragma unroll
          for (int i = 0; i < N / 4; ++i) {
            C::unpack4(vf[u].w[i], c);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][4 * i + e] = fmaf(wv, c[e], o[x][4 * i + e]);
          }
        }
        m[x] = mx;
      }
    }
  }

  // the row groups of this workgroup, one head after the other through the same staging area
  float *po = part_o + ((int64_t)item * a.splits + split) * a.G * D, *ml = part_ml + ((int64_t)item * a.splits + split) * a.G * 2;
#pragma unroll
  for (int x = 0; x < GM; ++x) {
    if (x < a.G) {
      __syncthreads();
      if (sub == 0) s_m[group] = m[x], s_l[group] = l[x];
#pragma unroll
      for (int e = 0; e < N; ++e) s_o[group][sub * N + e] = o[x][e];
      __syncthreads();
      if (threadIdx.x < D) {
        float M = -INFINITY;
        for (int g = 0; g < GROUPS; ++g) M = fmaxf(M, s_m[g]);
        const float ref = M == -INFINITY ? 0.0f : M;
        float L = 0.0f, acc = 0.0f;
        for (int g = 0; g < GROUPS; ++g) {
          const float w = __builtin_amdgcn_exp2f(s_m[g] - ref);
          L += w * s_l[g];
          acc += w * s_o[g][threadIdx.x];
        }
        if (a.splits == 1) {
          finish(a, b, hq0 + x, threadIdx.x, acc, M, L, out, lse);
        } else {
          store_through(po + x * D + threadIdx.x, acc);
          if (threadIdx.x == 0) store_through(ml + 2 * x, M), store_through(ml + 2 * x + 1, L);
        }
      }
    }
  }
  if (a.splits == 1) return;
  stores_done();
  __syncthreads();
  if (threadIdx.x < 64) {
    const bool last = arrive_last(flags + (int64_t)item * a.splits, a.splits, split, a.flag);
    if (threadIdx.x == 0) s_last = last;
  }
  __syncthreads();
  if (!s_last) return;
  // The last workgroup: a thread per pair of dims, the heads and dims in turn.
  for (int at = threadIdx.x; at < a.G * D / 2; at += 256) {
    const int x = at / (D / 2), c = at % (D / 2);
    const float2 *lo = reinterpret_cast<const float2 *>(part_o + (int64_t)item * a.splits * a.G * D) + at;
    const float2 *lm = reinterpret_cast<const float2 *>(part_ml + (int64_t)item * a.splits * a.G * 2) + x;
    float M = -INFINITY, L = 0.0f;
    float2 acc = make_float2(0.0f, 0.0f);
    for (int g0 = 0; g0 < a.splits; g0 += 8) {
      float2 e[8], v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int g = min(g0 + u, a.splits - 1);
        e[u] = load_through(lm + g * a.G);
        v[u] = load_through(lo + (int64_t)g * a.G * (D / 2));
      }
      float top = M;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (g0 + u >= a.splits) e[u] = make_float2(-INFINITY, 0.0f), v[u] = make_float2(0.0f, 0.0f);
        top = fmaxf(top, e[u].x);
      }
      const float ref = top == -INFINITY ? 0.0f : top, corr = __builtin_amdgcn_exp2f(M - ref);
      L *= corr, acc.x *= corr, acc.y *= corr;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __builtin_amdgcn_exp2f(e[u].x - ref);
        L += w * e[u].y, acc.x += w * v[u].x, acc.y += w * v[u].y;
      }
      M = top;
    }
    finish(a, b, hq0 + x, 2 * c, acc.x, M, L, out, lse);
    finish(a, b, hq0 + x, 2 * c + 1, acc.y, M, L, out, lse);
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int validate(const dam_decode_params *p, const void *q, const dam_quant_cache *c, const int32_t *kept_ptr,
             const int32_t *kept_idx, int64_t max_kept, const void *out) {
  if (!p || !q || !c || !c->kcache || !c->vcache || !c->kscale || !c->vscale || !kept_ptr || !out) return DAM_ERR_INVALID_ARG;
  if (p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->kv_capacity < 1) return DAM_ERR_INVALID_ARG;
  if (max_kept < 0 || (max_kept > 0 && !kept_idx)) return DAM_ERR_INVALID_ARG;
  if (p->dtype != DAM_F32 && p->dtype != DAM_BF16) return DAM_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return DAM_ERR_UNSUPPORTED;
  if (!quant_format_ok(c->format, c->block)) return DAM_ERR_UNSUPPORTED;
  const int per16 = p->dtype == DAM_BF16 ? 8 : 4;
  for (int i = 0; i < 2; ++i)
    if (p->q_stride[i] < 0 || p->q_stride[i] % per16 || p->o_stride[i] < 0 || c->scale_stride[i] < 0) return DAM_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (p->kv_stride[i] < 0 || p->kv_stride[i] % 16) return DAM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(c->kcache) || !aligned16(c->vcache)) return DAM_ERR_INVALID_ARG;
  if (!(p->scale >= 0.0f)) return DAM_ERR_INVALID_ARG;
  return DAM_OK;
}

int validate_grouped(const dam_decode_params *p, const void *q, const dam_quant_cache *c, const int32_t *kept_ptr,
                     const int32_t *kept_idx, const uint8_t *kept_member, int64_t max_kept, const void *out) {
  const int bad = validate(p, q, c, kept_ptr, kept_idx, max_kept, out);
  if (bad != DAM_OK) return bad;
  if (max_kept > 0 && !kept_member) return DAM_ERR_INVALID_ARG;
  if (p->hq / p->hkv > 8) return DAM_ERR_UNSUPPORTED;  // member bits are a byte
  return DAM_OK;
}

// Workgroups of a list, and the waves of each where the call takes the matrix-core kernel (`mfma`): eight waves per CU in
// workgroups of four, each wave with at least one block of 32 entries. Up to four waves are one workgroup.
GroupSplit splits_of(const dam_decode_params *p, int64_t max_kept, bool grouped, bool *mfma) {
  const int64_t lists = (int64_t)p->batch * (grouped ? p->hkv : p->hq);
  *mfma = grouped && decode_quant_mfma_fits(p);
  if (!*mfma) return {4, pick_splits(lists, max_kept)};
  const int64_t s = std::min<int64_t>((2048 + lists - 1) / lists, std::max<int64_t>(1, max_kept / 32));
  if (s <= 4) return {(int)s, 1};
  const int64_t groups = std::min<int64_t>(512 / lists, max_kept / 128);
  return {4, (int)std::min<int64_t>(std::max<int64_t>(groups, 1), 32)};
}

// What a call writes to its workspace; lists of query heads, or of KV heads.
Partials partials(void *ws, const dam_decode_params *p, int64_t max_kept, bool grouped) {
  bool mfma;
  return Partials(ws, p, splits_of(p, max_kept, grouped, &mfma).groups, (int64_t)p->batch * (grouped ? p->hkv : p->hq));
}

struct Plan {
  const uint8_t *table = nullptr;
  int n_flags = 0, pos = 0;
};

struct Call {
  const dam_decode_params *p;
  const void *q;
  const dam_quant_cache *c;
  const int32_t *kept_ptr, *kept_idx;
  const uint8_t *kept_member;
  Plan plan;
  void *out;
  float *lse;
  hipStream_t st;
};

template <typename T, int FORMAT, int D, int GM, bool PLAN>
void launch(const Call &x, const QDecodeArgs &a, const Partials &part) {
  const int pairs = a.B * a.Hkv, rounds = (pairs + kXcd - 1) / kXcd;
  k_decode_quant<T, FORMAT, D, GM, PLAN><<<rounds * kXcd * a.rows_of_kv * a.splits, 256, 0, x.st>>>(
      a, static_cast<const T *>(x.q), static_cast<const uint8_t *>(x.c->kcache), static_cast<const uint8_t *>(x.c->vcache),
      x.c->kscale, x.c->vscale, x.kept_ptr, x.kept_idx, x.kept_member, x.plan.table, part.o, part.ml, part.flags,
      static_cast<T *>(x.out), x.lse);
}

template <typename T, int FORMAT, int D>
void launch_form(const Call &x, const QDecodeArgs &a, const Partials &part) {
  if (x.plan.table) {
    if (a.G <= 4) launch<T, FORMAT, D, 4, true>(x, a, part);
    else launch<T, FORMAT, D, 8, true>(x, a, part);
  } else if (a.G == 1) {
    launch<T, FORMAT, D, 1, false>(x, a, part);
  } else if (a.G <= 4) {
    launch<T, FORMAT, D, 4, false>(x, a, part);
  } else {
    launch<T, FORMAT, D, 8, false>(x, a, part);
  }
}

// Arguments already validated, ws large enough.
int run(const Call &x, int64_t max_kept, bool grouped, void *ws) {
  const dam_decode_params *p = x.p;
  QDecodeArgs a;
  a.B = p->batch; a.Hq = p->hq; a.Hkv = p->hkv; a.cap = p->kv_capacity;
  a.shared_lists = p->shared_lists != 0;
  a.rows_of_kv = grouped ? 1 : p->hq / p->hkv;
  a.G = grouped ? p->hq / p->hkv : 1;
  bool mfma;
  const GroupSplit split = splits_of(p, max_kept, grouped, &mfma);
  a.splits = split.groups;
  a.block_shift = x.c->block == 16 ? 4 : x.c->block == 32 ? 5 : x.c->block == 64 ? 6 : 7;
  a.pos = x.plan.pos; a.n_flags = x.plan.n_flags;
  a.scale = p->scale > 0.0f ? p->scale : 1.0f / sqrtf((float)p->head_dim);
  a.q_sb = p->q_stride[0]; a.q_sh = p->q_stride[1];
  a.kv_sb = p->kv_stride[0]; a.kv_sh = p->kv_stride[1]; a.kv_ss = p->kv_stride[2];
  a.s_sb = x.c->scale_stride[0]; a.s_sh = x.c->scale_stride[1];
  a.o_sb = p->o_stride[0]; a.o_sh = p->o_stride[1];
  const Partials part = partials(ws, p, max_kept, grouped);
  if (mfma)
    return launch_decode_quant_mfma(p, split, a.scale, x.q, x.c, a.block_shift, x.kept_ptr, x.kept_idx, x.kept_member, part.o,
                                    part.ml, part.flags, x.out, x.lse, x.st, x.plan.table, x.plan.n_flags, x.plan.pos);
  a.flag = a.splits > 1 ? fresh_flag() : 0;
  const bool e4m3 = x.c->format == DAM_KV_E4M3, wide = p->head_dim == 128;
  if (p->dtype == DAM_BF16) {
    if (e4m3 && wide) launch_form<__hip_bfloat16, DAM_KV_E4M3, 128>(x, a, part);
    else if (e4m3) launch_form<__hip_bfloat16, DAM_KV_E4M3, 64>(x, a, part);
    else if (wide) launch_form<__hip_bfloat16, DAM_KV_INT8, 128>(x, a, part);
    else launch_form<__hip_bfloat16, DAM_KV_INT8, 64>(x, a, part);
  } else {
    if (e4m3 && wide) launch_form<float, DAM_KV_E4M3, 128>(x, a, part);
    else if (e4m3) launch_form<float, DAM_KV_E4M3, 64>(x, a, part);
    else if (wide) launch_form<float, DAM_KV_INT8, 128>(x, a, part);
    else launch_form<float, DAM_KV_INT8, 64>(x, a, part);
  }
  return launch_status();
}

}  // namespace

extern "C" size_t dam_sparse_attn_decode_quantized_workspace(const dam_decode_params *p, int64_t max_kept) {
  if (!p || p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->head_dim < 1 || max_kept < 0) return 0;
  return bytes_up_to_batch(p, [&](const dam_decode_params *x) { return partials(nullptr, x, max_kept, false); });
}

extern "C" size_t dam_sparse_attn_decode_grouped_quantized_workspace(const dam_decode_params *p, int64_t max_kept) {
  if (!p || p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->head_dim < 1 || max_kept < 0) return 0;
  return bytes_up_to_batch(p, [&](const dam_decode_params *x) { return partials(nullptr, x, max_kept, true); });
}

extern "C" int dam_sparse_attn_decode_quantized(const dam_decode_params *p, const void *q, const dam_quant_cache *cache,
                                                const int32_t *kept_ptr, const int32_t *kept_idx, int64_t max_kept, void *out,
                                                float *lse, void *ws, size_t ws_bytes, void *stream_v) {
  const int bad = validate(p, q, cache, kept_ptr, kept_idx, max_kept, out);
  if (bad != DAM_OK) return bad;
  if (!ws || ws_bytes < partials(nullptr, p, max_kept, false).bytes) return DAM_ERR_WORKSPACE;
  return run({p, q, cache, kept_ptr, kept_idx, nullptr, {}, out, lse, static_cast<hipStream_t>(stream_v)}, max_kept, false, ws);
}

extern "C" int dam_sparse_attn_decode_grouped_quantized(const dam_decode_params *p, const void *q, const dam_quant_cache *cache,
                                                        const int32_t *kept_ptr, const int32_t *kept_idx,
                                                        const uint8_t *kept_member, int64_t max_kept, void *out, float *lse,
                                                        void *ws, size_t ws_bytes, void *stream_v) {
  const int bad = validate_grouped(p, q, cache, kept_ptr, kept_idx, kept_member, max_kept, out);
  if (bad != DAM_OK) return bad;
  if (!ws || ws_bytes < partials(nullptr, p, max_kept, true).bytes) return DAM_ERR_WORKSPACE;
  return run({p, q, cache, kept_ptr, kept_idx, kept_member, {}, out, lse, static_cast<hipStream_t>(stream_v)}, max_kept, true, ws);
}

extern "C" int dam_sparse_attn_decode_patterns_quantized(const dam_decode_params *p, const void *q,
                                                         const dam_quant_cache *cache, const int32_t *plan_ptr,
                                                         const int32_t *plan_val, const uint8_t *plan_member,
                                                         const uint8_t *plan_table, int32_t n_flags, int32_t pos,
                                                         int64_t max_entries, void *out, float *lse, void *ws, size_t ws_bytes,
                                                         void *stream_v) {
  const int bad = validate_grouped(p, q, cache, plan_ptr, plan_val, plan_member, max_entries, out);
  if (bad != DAM_OK) return bad;
  if (!plan_table || n_flags < 1 || pos < 0 || pos >= p->kv_capacity) return DAM_ERR_INVALID_ARG;
  dam_decode_params shared = *p;
  shared.shared_lists = 1;  // a plan belongs to the heads, not to a sequence
  if (!ws || ws_bytes < partials(nullptr, &shared, max_entries, true).bytes) return DAM_ERR_WORKSPACE;
  return run({&shared, q, cache, plan_ptr, plan_val, plan_member, {plan_table, n_flags, pos}, out, lse,
              static_cast<hipStream_t>(stream_v)}, max_entries, true, ws);
}
