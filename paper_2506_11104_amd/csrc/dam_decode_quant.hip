// The decodes over a KV cache of 8-bit codes (dam_quant.h): one query row per (sequence, query head) over a list of kept
// keys of its own, over the merged list of its KV head's query heads, or over a plan of the matched patterns.
//
// Paper (arXiv 2506.11104): Sec. 3 (scaled dot-product attention) with the mask of Sec. 4.3 applied as -inf before the
// softmax; a list is row p of the masks of its heads. With the scales f_j, g_j of key j's rows, for each of a list's G heads
//   z_j = (sum_d q_d kcode_jd) f_j scale log2 e,   w_j = 2^(z_j - m),   O = sum_j (w_j g_j) vcode_j / sum_j w_j.
//
// HBM bound: 2 d bytes per listed key, half of a bf16 cache's.
//
// Merged lists and plans run on the matrix cores (k_decode_quant_group): the G query vectors are columns of the B operand of
// S^T = K Q^T and, as softmax weights, of O^T += V^T P^T, in blocks of 32 keys. What counts is that a block's arithmetic stays
// under its share of the memory's time (8 KB per wave at d = 128, eight waves per CU: some 4000 cycles): the codes become bf16
// between LDS and the products, which is exact, and the scales enter per key: K's on the logits, V's on the weights.
// A bf16 operand has 8 significant bits, and of a tile's 16 columns at most 8 hold heads. The others hold the same heads once
// more: columns 8 t + x what the terms before t leave of head x's weights. With bf16 queries (exact as they are) there are two
// terms, each rounded to nearest: a weight is off by at most 2^-17 of itself and to neither side, far below half a step of
// the output, 2^-8. (Cut off instead of rounded, the terms were low by up to 2^-15 while the sum l took whole weights, so that
// outputs came out low by 7e-6 in the mean.) With fp32 queries three terms, the upper 8 bits of what is left each, are
// all 24 bits, in two tiles of columns, and the queries themselves are split the same way, their partial logits added across the
// columns. (In products of 32 x 32, half of whose columns were idle, a lane had twice the logits to take through the softmax:
// plan step at batch 16 / 64k 39.7 us, now 38.8; fp32, two sequences at 32k 16.4, now 14.5; a block alone some 0.9 us, now 0.8.)
//
// A list per query head has one column (k_decode_quant_heads): plain ALUs, a row by 4 or 8 adjacent lanes with 16 codes each.
//
// Lists are split over waves, their workgroup merges them through LDS; where the lists alone do not fill the chip, over
// several workgroups, the last of which to finish merges those.
#include <hip/hip_bf16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dam_internal.h"
#include "dam_mfma.h"
#include "dam_quant.h"
#include "dam_splits.h"

namespace {
using namespace dam;

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kBlk = 32;                    // keys per block
constexpr int kMostWaves = 8;               // of a workgroup: the LDS of a CU at d = 128
constexpr int kMostGroups = 32;             // workgroups of a list

// A wave's LDS: two slots of K rows, two of V rows, then what goes with the rows.
template <int D>
struct Lds {
  static constexpr int kSlot = kBlk * D;           // bytes of the K (or V) rows of a block
  static constexpr int kV = 2 * kSlot;
  static constexpr int kEntries = 4 * kSlot;       // four slots of 32 list entries and their member bytes
  static constexpr int kScales = kEntries + 1024;  // four slots of 32 words with a K scale, 32 with a V scale
  static constexpr int kFix = kScales + 1024;      // plans: four slots of table words
  static constexpr int kFloat = kFix + 1024;       // the block's 32 V scales (and K scales) as fp32
  static constexpr int kMember = kFloat + 256;     // member bytes of the next block's keys, by key
  static constexpr int kBytes = kMember + 64;
  // at the end, in the slots: the results of the columns' terms, [term][dims / 4][head] of 16 bytes, then (reference, sum)
  static constexpr int kPart = 8 * D * 4;
  static constexpr int kMl = 3 * kPart;
};

struct QDecodeArgs {
  int B, Hq, Hkv, cap, shared_lists;
  int G;               // query heads per KV head
  int waves, groups;   // a list is shared by `waves` waves of each of `groups` workgroups
  int block_shift;     // log2 of the rows that share a scale
  int by_xcd;          // lists per head: a (sequence, KV head) pair has an XCD of its own
  uint64_t flag;       // of this call (Arrivals)
  float scale;
  int64_t q_sb, q_sh, kv_sb, kv_sh, kv_ss, s_sb, s_sh, o_sb, o_sh;
  int pos, n_flags;    // plans: position of the query row, length P of the pattern flags
};

// Sixteen bytes per lane from a 64-bit address of the lane's own to LDS address lds_at + IMM + 16 * lane.
template <int IMM>
__device__ __forceinline__ void lds_copy16_at(unsigned lds_at, uint64_t addr) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off"
               :
               : "s"(lds_at), "n"(IMM), "v"(addr)
               : "memory", "scc", "m0");
}

// Where the 16-byte chunk c of row r of a block lies in its LDS row: at position c ^ spread(r). Sixteen rows 16 t .. read at one
// chunk, as K's operand does, and the sixteen rows {0..7, 16..23} or {8..15, 24..31}, as V's does, then touch every bank once.
template <int D>
__device__ __forceinline__ int spread(int r) {
  const int top = ((r >> 3) ^ (r >> 4)) & 1;
  return D == 128 ? top << 2 | ((r >> 1) & 3) : top << 1 | ((r >> 2) & 1);
}

constexpr int spread_of_16(int d) { return d == 128 ? 4 : 2; }

// All ones where bit `pos` of a word is clear.
__device__ __forceinline__ unsigned unset(unsigned w, int pos) { return ~(unsigned)__builtin_amdgcn_sbfe((int)w, pos, 1); }

__device__ __forceinline__ float upper16(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

__device__ __forceinline__ u32x2 lds_read_tr8(const unsigned char *lds, int byte) {
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                       (__attribute__((address_space(3))) i32x2 *)(const_cast<unsigned char *>(lds + byte))));
}

// Codes 2 i and 2 i + 1 of a word, as two bf16 numbers (exact).
template <int FORMAT>
__device__ __forceinline__ unsigned to_bf16(unsigned w, int i) {
  if constexpr (FORMAT == DAM_KV_E4M3) {
    const auto r = i ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    return __builtin_bit_cast(unsigned, r);
  } else {
    return pack_bf16((float)(int8_t)(w >> (16 * i)), (float)(int8_t)(w >> (16 * i + 8)));
  }
}

// Eight elements of a query as an operand: term `term` of them (bf16 queries are their first term; terms from 3 on are 0).
__device__ __forceinline__ u32x4 query_term(const __hip_bfloat16 *p, int) { return *reinterpret_cast<const u32x4 *>(p); }
__device__ __forceinline__ u32x4 query_term(const float *p, int term) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = reinterpret_cast<const float2 *>(p)[i];
    float a = x.x, b = x.y;
    for (int t = 0; t < term; ++t) a -= upper16(a), b -= upper16(b);
    r[i] = term < 3 ? __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u) : 0u;
  }
  return r;
}

// Weights are at most 2^8 against their reference, but V's scales reach from 2^-126 to 2^122: products and sums of the two would
// leave fp32's range at either end. Those of a head with a kept row of a scale of 2^64 or more are therefore held 2^44 times
// smaller (range 44), those of a head that keeps no rows but ones of scales below 2^-64 2^36 times larger (range -36); the
// largest scale of the rows kept so far decides, and what the accumulators hold moves with it. Behind the loop the range is
// added to the reference, in log2 units, and the sum of weights takes the factor instead: merges need not know of it, and
// the 80 between the ends leave them 46 bits before a weight of theirs falls below 2^-126. Up to 2^31 keys the accumulators stay
// below 2^126. Weight times scale is lost below 2^-126, in range 44 below 2^-82.
// (The common case, no scale outside and range 0 all over the wave, is one comparison per block.)
__device__ __forceinline__ bool in_range_0(unsigned s) { return s - 63u < 128u; }
__device__ __forceinline__ int range_of(float scale) { return scale >= 0x1p64f ? 44 : scale < 0x1p-64f ? -36 : 0; }  // (NaN: 0)
// Hands (m, l) on, m in log2 units, and returns the factor that O takes: a whole number in the place of m stays exact.
__device__ __forceinline__ float hand_on_range(int range, float &m, float &l) {
  if (range == 0 || m == -INFINITY) return 1.0f;
  const float whole = rintf(m), f = __builtin_amdgcn_exp2f(m - whole);
  m = whole + (float)range;
  l = ldexpf(l * f, -range);
  return f;
}
// log(2^m L)
__device__ __forceinline__ float lse_of(float m, float L) {
  int e;
  const float f = frexpf(L, &e);
  return ((m + (float)e) + log2f(f)) * 0.6931471805599453f;
}

// The largest over the four lanes that hold a column's keys.
__device__ __forceinline__ float column_max(float x) {
  u32x2 sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

__device__ __forceinline__ void store4(float *p, const float4 &v) {
  if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) *reinterpret_cast<float4 *>(p) = v;
  else p[0] = v.x, p[1] = v.y, p[2] = v.z, p[3] = v.w;
}
__device__ __forceinline__ void store4(__hip_bfloat16 *p, const float4 &v) {
  const unsigned lo = pack_bf16(v.x, v.y), hi = pack_bf16(v.z, v.w);
  if ((reinterpret_cast<uintptr_t>(p) & 7) == 0) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(lo, hi);
  } else {
    unsigned short *u = reinterpret_cast<unsigned short *>(p);
    u[0] = (unsigned short)lo, u[1] = (unsigned short)(lo >> 16), u[2] = (unsigned short)hi, u[3] = (unsigned short)(hi >> 16);
  }
}

// Results of one column put together: four dims of a head, unnormalised, their reference (log2 units) and sum of weights.
struct Merged {
  float4 o;
  float M, L;
  __device__ float weight(float m) const { return __builtin_amdgcn_exp2f(m - (M == -INFINITY ? 0.0f : M)); }
  __device__ void rescale(float top) {
    const float was = M;
    M = top;
    const float c = weight(was);
    L *= c, o.x *= c, o.y *= c, o.z *= c, o.w *= c;
  }
  __device__ void add(float m, float l, const float4 &p) {
    const float w = weight(m);
    L += w * l, o.x += w * p.x, o.y += w * p.y, o.z += w * p.z, o.w += w * p.w;
  }
};

// As load_through, 16 bytes at byte `at` behind a base that is the same for the whole wave.
__device__ __forceinline__ float4 load_through16(const void *base, unsigned at) {
  constexpr int kSc1 = 16;             // past this XCD's L2
  constexpr int kWords = 0x00020000;   // a resource of plain 32-bit words
  const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, -1, kWords);
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(all, at, 0, kSc1);
  return make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
}

// Groups share, share + shares, ... of column `col` (of head x) of a list, N fetched at a time.
template <int N>
__device__ __forceinline__ void merge_groups(Merged &r, const float *ml, const float4 *po, int share, int shares, int groups,
                                             int col, int cols, int x, int heads) {
  for (int g0 = share; g0 < groups; g0 += N * shares) {
    float2 e[N];
    float4 v[N];
    float top = r.M;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int g = min(g0 + u * shares, groups - 1);
      e[u] = load_through(reinterpret_cast<const float2 *>(ml) + g * heads + x);
      v[u] = load_through16(po, (unsigned)(g * cols + col) * 16u);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (g0 + u * shares >= groups) e[u] = make_float2(-INFINITY, 0.0f), v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      top = fmaxf(top, e[u].x);
    }
    r.rescale(top);
#pragma unroll
    for (int u = 0; u < N; ++u) r.add(e[u].x, e[u].y, v[u]);
  }
}

// The workgroups of a list count themselves in a word of the workspace, whose content before the call is unknown: it belongs to
// a call once its upper bits hold the call's number, and the number of workgroups that have arrived is below. The word is looked
// at when a workgroup starts, made the call's own (where no other workgroup has) beside the partial results' stores, counted up
// when both are done, and left as 0. (What another call left there, or anything else, has the call's 58 upper bits with a
// probability of 2^-58 per list.) So the way from a workgroup's results to the one that merges them is three trips to
// memory (stores, count, loads), where a flag per workgroup, read back by all, takes four: one sequence at 128k, 27 workgroups a
// list, 13.3 us instead of 14.2; at 32k 9.15 / 10.0, from a plan at 8k 8.35 / 8.9; plan step at batch 16 / 64k, two workgroups a
// list, the same.
constexpr uint64_t kArrived = 63;  // (more than kMostGroups)
struct Arrivals {
  uint64_t *word;
  uint64_t call, seen = 0;
  __device__ Arrivals(uint64_t *at, uint64_t flag) : word(at), call(flag & ~kArrived) {}
  __device__ void look() { seen = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
  __device__ void claim() {
    uint64_t was = seen;
    if ((was & ~kArrived) != call)
      __hip_atomic_compare_exchange_strong(word, &was, call, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  // After the workgroup's stores and its claim are done: whether it is the last of n.
  __device__ bool last_of(int n) {
    const uint64_t before = __hip_atomic_fetch_add(word, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((int)(before & kArrived) != n - 1) return false;
    __hip_atomic_store(word, (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
  }
};

// A wave owns every splits-th block of 32 list entries and two LDS slots of K and V rows, filled by load-to-LDS
// copies whose addresses come from the list; the entries are staged three blocks ahead and the scale bytes with the rows, by
// the same kind of copy, so that every vector-memory operation of the loop is one of these copies and the waits are counted
// by hand. WIDE: a head's rows span 4 GiB or more, and their addresses are formed in 64 bits.
template <typename T, int FORMAT, int D, bool PLAN, bool WIDE>
__global__ __launch_bounds__(64 * kMostWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_decode_quant_group(
    QDecodeArgs a, const T *__restrict__ q, const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
    const uint8_t *__restrict__ ks, const uint8_t *__restrict__ vs, const int *__restrict__ kept_ptr,
    const int *__restrict__ kept_idx, const uint8_t *__restrict__ kept_member, const uint8_t *__restrict__ plan_table,
    float *__restrict__ part_o, float *__restrict__ part_ml, uint64_t *__restrict__ flags, T *__restrict__ out, float *__restrict__ lse) {
  using C = Code<FORMAT>;
  using S = Lds<D>;
  constexpr int kTerms = sizeof(T) == 2 ? 2 : 3;  // of a weight
  constexpr int kTiles = (kTerms + 1) / 2;        // of 16 columns: two terms of eight heads
  constexpr int kFrags = D / 32;                  // of a key's dims, a quarter of them per lane
  constexpr int kDims = D / 16;                   // blocks of 16 dims
  constexpr int kCopies = D / 32;                 // of a block's K (or V) rows
  extern __shared__ __attribute__((aligned(256))) unsigned char lds_all[];
  __shared__ int s_last;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char *lds = lds_all + wave * S::kBytes;  // this wave's slots
  const int n = lane & 15, kg = lane >> 4;          // column of the products, quarter of the wave
  const int head = n & 7, term = n >> 3;            // query head of the list, term of its weights (in the first tile)
  const int key = lane & 31, hf = lane >> 5;        // where a lane stands for a key of the block
  const int sub = lane / (D / 16), pos = lane % (D / 16);  // copies: row within the instruction's, 16-byte position
  const int G = a.G;
  const int group = (int)blockIdx.x % a.groups, pair = (int)blockIdx.x / a.groups;
  const int splits = a.waves * a.groups, split = group * a.waves + wave;
  const int b = pair / a.Hkv, hkv = pair % a.Hkv;
  const int list = a.shared_lists ? hkv : pair, hq0 = hkv * G;
  const int lo = __builtin_amdgcn_readfirstlane(kept_ptr[list]), end = __builtin_amdgcn_readfirstlane(kept_ptr[list + 1]);
  Arrivals arrivals(flags + (int64_t)pair * a.groups, a.flag);
  if (a.groups > 1 && threadIdx.x == 0) arrivals.look();
  // (entries are counted without a sign: a list may end at 2^31 - 1, and its last block a little further)
  const int n_blocks = (int)(((unsigned)max(end - lo, 0) + kBlk - 1) / kBlk);
  // this wave's blocks are split, split + splits, ...: every wave gets its share of each run of the list
  const int nb = n_blocks > split ? (n_blocks - split + splits - 1) / splits : 0;
  const float c2 = a.scale * 1.4426950408889634f;
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;

  f32x4 oacc[kTiles][kDims];
#pragma unroll
  for (int j = 0; j < kTiles; ++j)
#pragma unroll
    for (int dt = 0; dt < kDims; ++dt) oacc[j][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m_run = -INFINITY, l_run = 0.0f;  // reference of the weights (raw logits), this lane's part of their sum
  int range = 0;                          // of this column's accumulators (range_of)
  bool plain = true;                      // (wave-uniform) all are 0

  if (nb > 0) {
    const unsigned char *k_rows = kc + b * a.kv_sb + hkv * a.kv_sh, *v_rows = vc + b * a.kv_sb + hkv * a.kv_sh;
    const uint64_t idx_at = reinterpret_cast<uint64_t>(kept_idx), member_at = reinterpret_cast<uint64_t>(kept_member);
    // scale bytes of K (lanes 0 .. 31) and V of this head
    const uint64_t ks_at = reinterpret_cast<uint64_t>(ks + b * a.s_sb + hkv * a.s_sh);
    const uint64_t vs_at = reinterpret_cast<uint64_t>(vs + b * a.s_sb + hkv * a.s_sh);
    const uint64_t table_at = reinterpret_cast<uint64_t>(plan_table) + (uint64_t)hkv * (unsigned)a.n_flags;
    const int last_row = PLAN ? min(a.pos, a.cap - 1) : a.cap - 1;
    auto entry0 = [&](int i) { return lo + (split + i * splits) * kBlk; };
    // The row of a list entry. (An index outside the cache is pulled to its nearest row; PLAN: an entry v < 0 is the diagonal
    // -1 - v and stands for key pos + 1 + v, an entry v >= 0 is column v, and a key that does not exist yet, masked below,
    // is taken from those that do, since rows beyond the position may hold anything.)
    auto row_of = [&](int v) {
      if (PLAN && v < 0) v += a.pos + 1;
      return min(max(v, 0), last_row);
    };
    // Entries of local block i -> entry slot i & 3: lanes 0..31 fetch the key indices, lanes 32..40 the nine
    // aligned words that hold the block's 32 member bytes (the other lanes repeat the ninth). Entries past the
    // end of the list repeat its last one; their keys are masked below. An aligned word that holds a byte of
    // an array lies inside that byte's page, so the words at the array's two ends are safe to read.
    auto copy_entries = [&](int i) {
      const int e0 = entry0(i);
      const uint64_t first = (member_at + (unsigned)e0) & ~(uint64_t)3, last = (member_at + (unsigned)(end - 1)) & ~(uint64_t)3;
      const uint64_t addr = lane < 32 ? idx_at + 4ull * min((unsigned)e0 + (unsigned)key, (unsigned)(end - 1))
                                      : min(first + 4u * (unsigned)min(lane - 32, 8), last);
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + S::kEntries + (i & 3) * 256), addr);
    };
    auto entry = [&](int i, int k) { return *reinterpret_cast<const int *>(lds + S::kEntries + (i & 3) * 256 + 4 * k); };
    // PLAN: the aligned word that holds table[pos - c] for every column entry c of local block i (its entries have
    // landed) -> fix slot i & 3, lane k < 32 for entry k; every other lane and entry fetches the table's first word.
    // (A block without a column entry issues no copy: the copy, when there is one, is older than the copies of the
    // block's scales and rows, which are all that the waits below leave outstanding.)
    auto table_index = [&](int v) { return (v >= 0 && v <= a.pos && a.pos - v < a.n_flags) ? a.pos - v : -1; };
    auto copy_fix = [&](int i) {
      const int t = lane < 32 ? table_index(entry(i, key)) : -1;
      if (__builtin_amdgcn_ballot_w64(t >= 0) == 0) return;
      const uint64_t addr = t >= 0 ? (table_at + (unsigned)t) & ~(uint64_t)3 : reinterpret_cast<uint64_t>(plan_table) & ~(uint64_t)3;
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + S::kFix + (i & 3) * 256), addr);
    };
    // Scales and rows of local block i: one copy of the words that hold the 32 keys' scale bytes, kCopies of K rows and as
    // many of V rows into slot i & 1, LDS row r for key r of the block. Returns where in those words the scale bytes of this
    // lane's key lie (bits of K's, and of V's from bit 8 on).
    auto copy_rows = [&](int i) {
      const unsigned k_at = __builtin_amdgcn_readfirstlane(lds_base + (i & 1) * S::kSlot);
      const unsigned v_at = k_at + S::kV;
      const unsigned s = (unsigned)row_of(entry(i, key)) >> a.block_shift;
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + S::kScales + (i & 3) * 256), ((hf ? vs_at : ks_at) + s) & ~(uint64_t)3);
      if constexpr (WIDE) {
        uint64_t off[kCopies];
#pragma unroll
        for (int it = 0; it < kCopies; ++it) {
          const int r = 64 / (D / 16) * it + sub;
          off[it] = (uint64_t)row_of(entry(i, r)) * (uint64_t)a.kv_ss + ((pos ^ spread<D>(r)) << 4);
        }
        const uint64_t k0 = reinterpret_cast<uint64_t>(k_rows), v0 = reinterpret_cast<uint64_t>(v_rows);
        lds_copy16_at<0 * 1024>(k_at, k0 + off[0]);
        lds_copy16_at<1 * 1024>(k_at, k0 + off[1]);
        if constexpr (kCopies == 4) lds_copy16_at<2 * 1024>(k_at, k0 + off[2]), lds_copy16_at<3 * 1024>(k_at, k0 + off[3]);
        lds_copy16_at<0 * 1024>(v_at, v0 + off[0]);
        lds_copy16_at<1 * 1024>(v_at, v0 + off[1]);
        if constexpr (kCopies == 4) lds_copy16_at<2 * 1024>(v_at, v0 + off[2]), lds_copy16_at<3 * 1024>(v_at, v0 + off[3]);
      } else {
        unsigned off[kCopies];
#pragma unroll
        for (int it = 0; it < kCopies; ++it) {
          const int r = 64 / (D / 16) * it + sub;
          // (row index and row stride are below 2^24: the 24-bit multiply runs at full rate, the 32-bit one does not)
          off[it] = __umul24((unsigned)row_of(entry(i, r)), (unsigned)a.kv_ss) + ((pos ^ spread<D>(r)) << 4);
        }
        lds_copy16_once<1024 * 0>(k_at, k_rows, off[0]);
        lds_copy16_once<1024 * 1>(k_at, k_rows, off[1]);
        if constexpr (kCopies == 4) lds_copy16_once<1024 * 2>(k_at, k_rows, off[2]), lds_copy16_once<1024 * 3>(k_at, k_rows, off[3]);
        lds_copy16_once<1024 * 0>(v_at, v_rows, off[0]);
        lds_copy16_once<1024 * 1>(v_at, v_rows, off[1]);
        if constexpr (kCopies == 4) lds_copy16_once<1024 * 2>(v_at, v_rows, off[2]), lds_copy16_once<1024 * 3>(v_at, v_rows, off[3]);
      }
      return (((unsigned)ks_at + s) & 3) * 8 | (((unsigned)vs_at + s) & 3) * 0x800;
    };
    // Which heads keep which key of local block i (its entries and table words have landed): a byte per key, dealt out so
    // that bit 8 r of word t says whether this lane's head keeps the key of accumulator r of tile t, 16 t + 4 kg + r.
    struct Kept {
      unsigned w[2];
    };
    const int member_shift = (int)((member_at + (unsigned)lo) & 3);  // (blocks start a multiple of 32 entries apart)
    auto keeps = [&](int i) {
      unsigned mem = lds[S::kEntries + (i & 3) * 256 + 128 + member_shift + key];
      if ((unsigned)entry0(i) + (unsigned)key >= (unsigned)end) mem = 0u;
      if (PLAN) {
        const int v = entry(i, key);
        const bool exists = v < 0 ? a.pos + 1 + v >= 0 : v <= a.pos;
        const int t = table_index(v);
        unsigned covered = 0;  // heads that reach this column's key through a matched diagonal
        if (t >= 0) {
          const unsigned word = *reinterpret_cast<const unsigned *>(lds + S::kFix + (i & 3) * 256 + 4 * key);
          covered = (word >> (8 * (int)((table_at + (unsigned)t) & 3))) & 0xFFu;
        }
        mem = exists ? mem & ~covered : 0u;
      }
      lds[S::kMember + key] = (unsigned char)mem;  // (both half-waves hold the same)
      Kept k;
#pragma unroll
      for (int t = 0; t < 2; ++t) k.w[t] = *reinterpret_cast<const unsigned *>(lds + S::kMember + 16 * t + 4 * kg) >> head;
      return k;
    };

    // Q fragments: B operand of S^T = K Q^T. Column n of tile j is term 2 j + n / 8 of query head n % 8 of the list (zero beyond
    // the list's); fragment c of this lane covers dims kg D / 4 + 8 c .. + 7 (the order of the dims in the contraction is K's).
    bf16x8 qf[kTiles][kFrags];
    {
      const T *qp = q + b * a.q_sb + (int64_t)(hq0 + min(head, G - 1)) * a.q_sh + kg * (D / 4);
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int c = 0; c < kFrags; ++c) {
          u32x4 raw = {0u, 0u, 0u, 0u};
          if (head < G) raw = query_term(qp + 8 * c, 2 * j + term);
          qf[j][c] = __builtin_bit_cast(bf16x8, raw);
        }
    }
    copy_entries(0);
    if (nb > 1) copy_entries(1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // (the Q fragments have arrived with that wait; the empty statement tells the compiler so)
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
      for (int c = 0; c < kFrags; ++c) asm volatile("" : "+v"(qf[j][c]));
    if (PLAN) {
      copy_fix(0);
      if (nb > 1) copy_fix(1);
    }
    if (nb > 2) copy_entries(2);
    unsigned bits_now = copy_rows(0), bits_next = 0;
    if (nb > 1) bits_next = copy_rows(1);

    const float less = term ? 1.0f : 0.0f;  // the second term of a weight: less its first
    float *vsf = reinterpret_cast<float *>(lds + S::kFloat), *ksf = vsf + 32;
    // LDS byte offsets of this lane's operand fragments in a slot; the others differ by an XOR (and tile 1 by 16 rows). K: rows n
    // and 16 + n, quarter kg of their chunks. V: a transposing read takes eight bytes of a row per lane (lanes 2 r and 2 r + 1 of
    // sixteen the 16 bytes of row r of eight) and leaves a lane the byte of its own column of all eight rows: dim 16 dt + n of
    // the keys 4 kg + {0..3, 16..19}, the order in which the lane holds weights.
    constexpr int kFlip = spread_of_16(D);  // spread(r + 16) is spread(r) ^ this
    const int kbase = n * D + (((D / 64 * kg) ^ spread<D>(n)) << 4);
    const int vrow = 16 * ((lane >> 3) & 1) + 4 * kg + ((lane >> 1) & 3);
    const int vbase = vrow * D + (spread<D>(vrow) << 4) + 8 * (lane & 1);
    Kept kept_now, kept_next;

    for (int i = 0; i < nb; ++i) {
      // The copies were issued in the order ... rows i, entries i + 2 (PLAN: table words i + 1), scales and rows i + 1: what
      // block i needs and the entries of block i + 2 have landed once nothing but the copies of block i + 1's scales and rows is
      // outstanding.
      if (i + 1 < nb) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * kCopies + 1) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const unsigned char *kslot = lds + (i & 1) * S::kSlot;
      const unsigned char *vslot = lds + S::kV + (i & 1) * S::kSlot;

      // Everything the block needs from LDS is asked for at once, for its latency to be paid once.
      const unsigned *words = reinterpret_cast<const unsigned *>(lds + S::kScales + (i & 3) * 256);
      const unsigned kword = words[key], vword = words[32 + key];
      const int some = key * D + 4 * key % D;  // a code of the key's row (NaN throughout or nowhere), in a bank of its own
      const unsigned kcode = kslot[some], vcode = vslot[some];
      u32x4 kw[2][D / 64];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
          kw[t][j] = *reinterpret_cast<const u32x4 *>(kslot + ((kbase ^ ((j ^ (t * kFlip)) << 4)) + 16 * D * t));
      if (i == 0) kept_now = keeps(0);
      u32x2 vw[kDims];
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt) vw[dt] = lds_read_tr8(vslot, vbase ^ (dt << 4));

      // Scales of this lane's key of the block. NaN rows: the scale carries the NaN, which reaches the heads that keep the row
      // through the logits (K's codes do so themselves in e4m3) or the weights; a V row's codes are cleared, since the product
      // would carry them to all heads.
      float kscale = scale_value((kword >> (bits_now & 31)) & 0xFFu);
      const unsigned vbyte = (vword >> (bits_now >> 8)) & 0xFFu;
      float vscale = scale_value(vbyte);
      const bool odd = __ballot(!in_range_0(vbyte)) != 0;
      const bool vbad = C::is_nan(vcode);
      if (vbad) vscale = NAN;
      if (FORMAT == DAM_KV_INT8 && C::is_nan(kcode)) kscale = NAN;
      const unsigned vbads = (unsigned)__ballot(vbad);
      if (hf == 0) vsf[key] = vscale, ksf[key] = kscale;

      // S^T = K Q^T; accumulator r of tile t is key 16 t + 4 kg + r
      f32x4 s[kTiles][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) s[j][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < kFrags; ++c) {
          const unsigned w0 = kw[t][c / 2][2 * (c % 2)], w1 = kw[t][c / 2][2 * (c % 2) + 1];
          const u32x4 f = {to_bf16<FORMAT>(w0, 0), to_bf16<FORMAT>(w0, 1), to_bf16<FORMAT>(w1, 0), to_bf16<FORMAT>(w1, 1)};
#pragma unroll
          for (int j = 0; j < kTiles; ++j)
            s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), qf[j][c], s[j][t], 0, 0, 0);
        }
      }
      if (i + 1 < nb) kept_next = keeps(i + 1);
      // logits: the sum over a query's terms, which are columns n, n ^ 8 and tiles; K's scales; masked keys to -inf (after the
      // products, so that a NaN row does not get past it)
      float w[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f32x4 f = *reinterpret_cast<const f32x4 *>(ksf + 16 * t + 4 * kg);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = s[0][t][r];
          if (kTiles == 2) {
            x += s[kTiles - 1][t][r];
            x += dpp_move<0x128>(x);  // row_ror 8
          }
          const unsigned off = unset(kept_now.w[t], 8 * r);
          w[4 * t + r] = __uint_as_float((off & 0xFF800000u) | (~off & __float_as_uint(x * f[r])));
        }
      }

      // (wave-uniform) the range that the accumulators need with this block's kept rows
      if (__builtin_expect(odd || !plain, 0)) {
        float l_all = l_run + __shfl_xor(l_run, 16);
        l_all += __shfl_xor(l_all, 32);
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!unset(kept_now.w[e / 4], 8 * (e % 4))) top = fmaxf(top, (float)range_of(vsf[16 * (e / 4) + 4 * kg + e % 4]));
        top = column_max(top);
        // (a head that has kept a row has a sum that is not 0: at least 2^-8 from that of the largest logit)
        const int to = top == -INFINITY ? range : l_all == 0.0f ? (int)top : max(range, (int)top);
        if (__ballot(to != range)) {
#pragma unroll
          for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int dt = 0; dt < kDims; ++dt)
#pragma unroll
              for (int r = 0; r < 4; ++r) oacc[j][dt][r] = ldexpf(oacc[j][dt][r], range - to);
        }
        range = to;
        plain = __ballot(range != 0) == 0;
      }

      // online softmax, a head in the four lanes that hold its column; the reference the weights are taken against only moves
      // when the maximum has grown past it by more than 8 in log2 units
      float mx = w[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, w[e]);
      const float m_top = fmaxf(m_run, column_max(mx));
      const bool move = (m_top - m_run) * c2 > 8.0f;  // (-inf) - (-inf) is NaN: no move
      const float m_new = move ? m_top : m_run;
      const float m_ref = m_new == -INFINITY ? 0.0f : m_new;
      const float off = m_ref * c2;
      if (__ballot(move)) {
        const float corr = move ? __builtin_amdgcn_exp2f((m_run - m_ref) * c2) : 1.0f;  // old reference -inf: 0
        l_run *= corr;
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
          for (int dt = 0; dt < kDims; ++dt) {
            f32x4 &o = oacc[j][dt];
            o = f32x4{o[0] * corr, o[1] * corr, o[2] * corr, o[3] * corr};
          }
      }
      m_run = m_new;
      // the weights, times the scales of V's rows; the sum is taken over the weights themselves
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(w[e], c2, -off));
      l_run += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x4 f = *reinterpret_cast<const f32x4 *>(vsf + 16 * t + 4 * kg);
        if (__builtin_expect(!plain, 0))
          f = f32x4{ldexpf(f[0], -range), ldexpf(f[1], -range), ldexpf(f[2], -range), ldexpf(f[3], -range)};
#pragma unroll
        for (int r = 0; r < 4; ++r) w[4 * t + r] *= f[r];
      }
      // (wave-uniform) a weight of 0 times a scale that is NaN or beyond the column's range; NaN rows' codes
      if (__builtin_expect(vbads || !plain, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __uint_as_float(~unset(kept_now.w[e / 4], 8 * (e % 4)) & __float_as_uint(w[e]));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // bits r of the keys in bytes r of the word
          const unsigned gone = (((vbads >> (16 * t + 4 * kg)) & 15u) * 0x204081u & 0x01010101u) * 0xFFu;
#pragma unroll
          for (int dt = 0; dt < kDims; ++dt) vw[dt][t] &= ~gone;
        }
      }
      // the terms of the weights: in the columns below 8 the weight as bf16, from 8 on what that leaves as bf16 (fp32 queries: the
      // upper 16 bits, those of what remains, and in the second tile of what remains then)
      u32x4 p[kTiles];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        if (kTiles == 1) {
          const unsigned first = pack_bf16(w[e], w[e + 1]);
          p[0][e / 2] = pack_bf16(__builtin_fmaf(-less, __uint_as_float(first << 16), w[e]),
                                  __builtin_fmaf(-less, __uint_as_float(first & 0xFFFF0000u), w[e + 1]));
        } else {
          float r0 = __builtin_fmaf(-less, upper16(w[e]), w[e]), r1 = __builtin_fmaf(-less, upper16(w[e + 1]), w[e + 1]);
          p[0][e / 2] = __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x07060302u);
          r0 = w[e] - upper16(w[e]), r1 = w[e + 1] - upper16(w[e + 1]);
          r0 -= upper16(r0), r1 -= upper16(r1);
          p[kTiles - 1][e / 2] = __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x07060302u);
        }
      }

      // O^T += V^T P^T: accumulator r of dim block dt is dim 16 dt + 4 kg + r
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt) {
        const unsigned x0 = vw[dt][0], x1 = vw[dt][1];
        const u32x4 f = {to_bf16<FORMAT>(x0, 0), to_bf16<FORMAT>(x0, 1), to_bf16<FORMAT>(x1, 0), to_bf16<FORMAT>(x1, 1)};
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
          oacc[j][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, p[j]),
                                                                oacc[j][dt], 0, 0, 0);
      }
      // every LDS read of block i has returned (the products consumed them): its slots are free for block i + 2
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      kept_now = kept_next;
      bits_now = bits_next;
      if (i + 3 < nb) copy_entries(i + 3);
      if (PLAN && i + 2 < nb) copy_fix(i + 2);
      if (i + 2 < nb) bits_next = copy_rows(i + 2);
    }
  }

  if (a.groups > 1 && threadIdx.x == 0) arrivals.claim();
  // The waves' results meet in LDS, dealt out in columns as everything from here on: column c G + x is dims 4 c .. + 3 of
  // head x, 16 bytes at 16 (c G + x) of the wave's own slots, term t's share of it t kPart further; behind them the
  // head's reference (log2 units) and sum.
  float l_tot = l_run + __shfl_xor(l_run, 16);
  l_tot += __shfl_xor(l_tot, 32);
  float m_log2 = m_run == -INFINITY ? -INFINITY : m_run * c2;
  if (__builtin_expect(!plain, 0)) {
    const float f = hand_on_range(range, m_log2, l_tot);
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) oacc[j][dt][r] *= f;
  }
  if (head < G) {
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      if (2 * j + term >= kTerms) continue;
      float4 *mine_o = reinterpret_cast<float4 *>(lds + (2 * j + term) * S::kPart) + head;
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt)
        mine_o[(4 * dt + kg) * G] = make_float4(oacc[j][dt][0], oacc[j][dt][1], oacc[j][dt][2], oacc[j][dt][3]);
    }
    if (lane < 8) reinterpret_cast<float2 *>(lds + S::kMl)[n] = make_float2(m_log2, l_tot);
  }
  __syncthreads();
  const int cols = G * (D / 4);
  auto finish = [&](int x, int c, const float4 &o, float M, float L) {
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;  // (L = 0: no key; NaN stays)
    store4(out + b * a.o_sb + (int64_t)(hq0 + x) * a.o_sh + 4 * c, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (lse && c == 0) lse[(int64_t)b * a.Hq + hq0 + x] = L == 0.0f ? -INFINITY : lse_of(M, L);
  };
  float4 *po = reinterpret_cast<float4 *>(part_o) + (int64_t)pair * a.groups * cols;  // [group][column]
  float *ml = part_ml + (int64_t)pair * a.groups * G * 2;                             // [group][head][2]
  for (int col = threadIdx.x; col < cols; col += blockDim.x) {
    const int x = col % G, c = col / G;
    Merged r = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.0f};
    for (int w = 0; w < a.waves; ++w) r.M = fmaxf(r.M, reinterpret_cast<const float2 *>(lds_all + w * S::kBytes + S::kMl)[x].x);
    for (int w = 0; w < a.waves; ++w) {
      const unsigned char *its = lds_all + w * S::kBytes;
      const float2 e = reinterpret_cast<const float2 *>(its + S::kMl)[x];
      r.add(e.x, e.y, reinterpret_cast<const float4 *>(its)[col]);
#pragma unroll
      for (int t = 1; t < kTerms; ++t) r.add(e.x, 0.0f, reinterpret_cast<const float4 *>(its + t * S::kPart)[col]);
    }
    if (a.groups == 1) {
      finish(x, c, r.o, r.M, r.L);
    } else {
      store_through(po + group * cols + col, r.o.x, r.o.y, r.o.z, r.o.w);
      if (c == 0) {
        store_through(ml + (group * G + x) * 2, r.M);
        store_through(ml + (group * G + x) * 2 + 1, r.L);
      }
    }
  }
  if (a.groups == 1) return;
  stores_done();
  __syncthreads();
  if (threadIdx.x == 0) s_last = arrivals.last_of(a.groups);
  __syncthreads();
  if (!s_last) return;
  // The last workgroup merges the groups. Threads that share a column take them in turn; where there are fewer threads than
  // columns, a thread takes several columns.
  const int shares = max((int)blockDim.x / cols, 1), share = threadIdx.x / cols;
  float4 *sum = reinterpret_cast<float4 *>(lds_all);  // [thread] O, then [thread] (M, L)
  float2 *sum_ml = reinterpret_cast<float2 *>(lds_all + blockDim.x * sizeof(float4));
  for (int col = threadIdx.x % cols; col < cols; col += blockDim.x) {
    const int x = col % G;
    Merged r = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.0f};
    if (share < shares) {
      // Bound by the latency of reading the groups back: as many as there are, up to eight, are fetched at a time (one sequence
      // at 128k, eight heads in 27 groups, four at a time 15.4 us, eight 14.6, when all else took longer by 1 us), but no more:
      // each costs a thread two loads (plan step at batch 16 / 64k, two groups for a thread, two at a time 40.4 us, eight
      // 41.1, sixteen 42.9).
      const int each = (a.groups + shares - 1) / shares;
      if (each <= 2) merge_groups<2>(r, ml, po, share, shares, a.groups, col, cols, x, G);
      else if (each <= 4) merge_groups<4>(r, ml, po, share, shares, a.groups, col, cols, x, G);
      else merge_groups<8>(r, ml, po, share, shares, a.groups, col, cols, x, G);
    }
    if (shares > 1) {  // (then every thread comes by here once)
      sum[threadIdx.x] = r.o;
      sum_ml[threadIdx.x] = make_float2(r.M, r.L);
      __syncthreads();
      if (share > 0) return;
      for (int y = 1; y < shares; ++y) {
        const float4 oy = sum[y * cols + col];
        const float2 e = sum_ml[y * cols + col];
        r.rescale(fmaxf(r.M, e.x));
        r.add(e.x, e.y, oy);
      }
    }
    if (share == 0) finish(x, col / G, r.o, r.M, r.L);
  }
}

// The largest value, and the sum, over the lanes of a wave that hold the same columns (lanes LPR apart).
template <int LPR>
__device__ __forceinline__ float wave_max(float x) {
  if (LPR <= 4) x = fmaxf(x, dpp_move<0x124>(x));  // row_ror 4
  x = fmaxf(x, dpp_move<0x128>(x));                // row_ror 8
  u32x2 sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
template <int LPR>
__device__ __forceinline__ float row16_sum(float x) {
  if (LPR <= 4) x += dpp_move<0x124>(x);
  return x + dpp_move<0x128>(x);
}

// A query's sixteen elements against sixteen codes of a row.
template <typename T, int FORMAT>
struct Query {  // as fp32
  float v[16];
  __device__ void load(const float *p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = reinterpret_cast<const float4 *>(p)[i];
      v[4 * i] = x.x, v[4 * i + 1] = x.y, v[4 * i + 2] = x.z, v[4 * i + 3] = x.w;
    }
  }
  __device__ void load(const __hip_bfloat16 *p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 x = reinterpret_cast<const u32x4 *>(p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[8 * i + 2 * e] = __uint_as_float(x[e] << 16), v[8 * i + 2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
    }
  }
  __device__ float dot(const u32x4 &codes) const {
    float d = 0.0f, c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Code<FORMAT>::unpack4(codes[i], c);
#pragma unroll
      for (int e = 0; e < 4; ++e) d = fmaf(v[4 * i + e], c[e], d);
    }
    return d;
  }
};
template <>
struct Query<__hip_bfloat16, DAM_KV_E4M3> {  // pairs of bf16 numbers: products of two codes with one instruction
  u32x4 v[2];
  __device__ void load(const __hip_bfloat16 *p) { v[0] = reinterpret_cast<const u32x4 *>(p)[0], v[1] = reinterpret_cast<const u32x4 *>(p)[1]; }
  __device__ float dot(const u32x4 &codes) const {
    float d = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned x = v[i / 4][i % 4], y = to_bf16<DAM_KV_E4M3>(codes[i / 2], i % 2);
      d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), d, false);
    }
    return d;
  }
};

// A list per query head. A row is read by LPR adjacent lanes, and a lane keeps kUnroll keys in flight (their row numbers are
// fetched a pass ahead); a row's scales enter once per row. Two keys a lane leave short lists more waves and workgroups to be
// split over than four do, and long ones are held up by their arithmetic either way: one sequence with 8 fp32 heads of 1640 keys
// 6.9 us (four: 7.9, eight: 9.4), with 32 heads of 1640 keys 7.4 (7.8, 9.6), of 6550 keys 13.0 (12.9, 13.6). Nor are there more
// than 16 workgroups to a list, which one of them has to merge: 8 fp32 heads of 1640 keys 7.2, with up to 32 workgroups 7.5, 8 heads
// of 6550 keys 9.6 either way; few lists that are longer still would gain (8 heads of one KV head, 13100 keys 13.1, 11.5).
constexpr int kUnroll = 2;
constexpr int kHeadWaves = 8;
constexpr int kMostHeadGroups = 16;
template <typename T, int FORMAT, int D, bool WIDE>
__global__ __launch_bounds__(64 * kHeadWaves) void k_decode_quant_heads(
    QDecodeArgs a, const T *__restrict__ q, const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
    const uint8_t *__restrict__ ks, const uint8_t *__restrict__ vs, const int *__restrict__ kept_ptr,
    const int *__restrict__ kept_idx, float *__restrict__ part_o, float *__restrict__ part_ml, uint64_t *__restrict__ flags,
    T *__restrict__ out, float *__restrict__ lse) {
  using C = Code<FORMAT>;
  constexpr int LPR = D / 16, GROUPS = 64 / LPR;  // lanes per row, rows of a wave
  __shared__ float s_o[kHeadWaves][D];
  __shared__ float2 s_ml[kHeadWaves];
  __shared__ int s_last;

  // block n runs on XCD n % 8. by_xcd: all workgroups of a (sequence, KV head) pair have ids with the same n % 8, so that its
  // heads find the rows they share in one L2; else they are dealt out over the XCDs in turn
  const int per_pair = a.G * a.groups, slot = (int)blockIdx.x / (a.by_xcd ? kXcd : 1);
  const int pair = a.by_xcd ? slot / per_pair * kXcd + (int)blockIdx.x % kXcd : slot / per_pair;
  if (pair >= a.B * a.Hkv) return;
  const int b = pair / a.Hkv, hkv = pair % a.Hkv;
  const int hq = hkv * a.G + slot % per_pair / a.groups, group = slot % a.groups, item = b * a.Hq + hq;
  const int list = a.shared_lists ? hq : item;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LPR;
  const int64_t end = kept_ptr[list + 1];
  const int64_t stride = (int64_t)a.groups * a.waves * GROUPS * kUnroll;

  Query<T, FORMAT> qf;
  qf.load(q + b * a.q_sb + hq * a.q_sh + sub * 16);
  const uint8_t *kb = kc + b * a.kv_sb + hkv * a.kv_sh, *vb = vc + b * a.kv_sb + hkv * a.kv_sh;
  const uint8_t *ksb = ks + b * a.s_sb + hkv * a.s_sh, *vsb = vs + b * a.s_sb + hkv * a.s_sh;
  const float sl2 = a.scale * 1.4426950408889634f;  // logits in log2 units

  Arrivals arrivals(flags + (int64_t)item * a.groups, a.flag);
  if (a.groups > 1 && threadIdx.x == 0) arrivals.look();

  float m = -INFINITY, l = 0.0f, o[16];
  int range = 0;  // of this lane's sums (range_of)
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = 0.0f;
  int rows[kUnroll];
  int64_t p0 = kept_ptr[list] + ((int64_t)(group * a.waves + wave) * GROUPS + lane / LPR) * kUnroll;
  auto fetch = [&](int64_t at) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) rows[u] = kept_idx[min(at + u, end - 1)];
  };
  if (p0 < end) fetch(p0);
  for (; p0 < end; p0 += stride) {
    u32x4 kf[kUnroll], vf[kUnroll];
    float kscale[kUnroll], vscale[kUnroll];
    bool odd = range != 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const unsigned r = (unsigned)in_cache(rows[u], a.cap);
      // (a row index and a row stride below 2^24 each: the 24-bit multiply runs at full rate)
      using Offset = std::conditional_t<WIDE, uint64_t, unsigned>;
      const Offset at = (WIDE ? (Offset)(r * (uint64_t)a.kv_ss) : (Offset)__umul24(r, (unsigned)a.kv_ss)) + (unsigned)(16 * sub);
      kf[u] = *reinterpret_cast<const u32x4 *>(kb + at);
      vf[u] = *reinterpret_cast<const u32x4 *>(vb + at);
      kscale[u] = scale_value(ksb[r >> a.block_shift]);
      const unsigned vbyte = vsb[r >> a.block_shift];
      vscale[u] = scale_value(vbyte);
      odd |= !in_range_0(vbyte);
    }
    fetch(p0 + stride);  // (always, so that the waits behind it need not expect that it was not)
    float s[kUnroll], mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (FORMAT == DAM_KV_INT8 && C::is_nan(kf[u][0])) kscale[u] = NAN;  // (e4m3: the codes do it)
      s[u] = row_sum<LPR>(qf.dot(kf[u])) * (kscale[u] * sl2);
      if (p0 + u >= end) s[u] = -INFINITY;
      mx = fmaxf(mx, s[u]);
    }
    // the reference of the weights moves only when the maximum has grown past it by more than 8
    const bool move = mx > m + 8.0f, none = l == 0.0f;  // (none: no row so far)
    if (__ballot(move)) {
      const float to = move ? mx : m, corr = move ? __builtin_amdgcn_exp2f(m - to) : 1.0f;
      m = to;
      l *= corr;
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] *= corr;
    }
    if (__builtin_expect(odd, 0)) {  // the range that the sums need with these rows
      int top = range_of(vscale[0]);
#pragma unroll
      for (int u = 1; u < kUnroll; ++u)
        if (p0 + u < end) top = max(top, range_of(vscale[u]));
      const int to = none ? top : max(range, top);
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = ldexpf(o[e], range - to);
      range = to;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) vscale[u] = ldexpf(vscale[u], -range);
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const float w = __builtin_amdgcn_exp2f(s[u] - ref);
      l += w;
      if (FORMAT == DAM_KV_INT8 && C::is_nan(vf[u][0])) vscale[u] = NAN;
      const float wv = w * vscale[u];  // (past the end: the last key once more, with a weight of 0)
      float c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        C::unpack4(vf[u][i], c);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[4 * i + e] = fmaf(wv, c[e], o[4 * i + e]);
      }
    }
  }

  if (a.groups > 1 && threadIdx.x == 0) arrivals.claim();
  const float part = hand_on_range(range, m, l);
  // the rows of a wave, to one reference; the sums over them leave four dims to every lane of sixteen
  const float M = wave_max<LPR>(m), ref = M == -INFINITY ? 0.0f : M;
  float f = __builtin_amdgcn_exp2f(m - ref);
  l = row16_sum<LPR>(l * f);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  float t[8], r[4];
  f *= part;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[e] * f), __float_as_uint(o[e + 8] * f), false, false);
    t[e] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);  // dim e, e + 8 in the upper half-wave
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const u32x2 sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(t[e]), __float_as_uint(t[e + 4]), false, false);
    r[e] = row16_sum<LPR>(__uint_as_float(sw[0]) + __uint_as_float(sw[1]));  // dim e + 4 (lane / 16)
  }
  if ((lane & 15) < LPR) *reinterpret_cast<float4 *>(&s_o[wave][16 * sub + 4 * (lane >> 4)]) = make_float4(r[0], r[1], r[2], r[3]);
  if (lane == 0) s_ml[wave] = make_float2(M, l);
  __syncthreads();
  auto finish = [&](int dim, float acc, float top, float L) {  // (L = 0: no key)
    store_out(out + b * a.o_sb + hq * a.o_sh + dim, L == 0.0f ? 0.0f : acc / L);
    if (lse && dim == 0) lse[item] = L == 0.0f ? -INFINITY : lse_of(top, L);
  };
  float *po = part_o + ((int64_t)item * a.groups + group) * D, *ml = part_ml + ((int64_t)item * a.groups + group) * 2;
  for (int dim = threadIdx.x; dim < D; dim += 64 * a.waves) {
    float top = -INFINITY, L = 0.0f, acc = 0.0f;
    for (int w = 0; w < a.waves; ++w) top = fmaxf(top, s_ml[w].x);
    const float to = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < a.waves; ++w) {
      const float x = __builtin_amdgcn_exp2f(s_ml[w].x - to);
      L += x * s_ml[w].y;
      acc += x * s_o[w][dim];
    }
    if (a.groups == 1) {
      finish(dim, acc, top, L);
    } else {
      store_through(po + dim, acc);
      if (dim == 0) store_through(ml, top), store_through(ml + 1, L);
    }
  }
  if (a.groups == 1) return;
  stores_done();
  __syncthreads();
  if (threadIdx.x == 0) s_last = arrivals.last_of(a.groups);
  __syncthreads();
  if (!s_last) return;
  // the last workgroup: a thread per pair of dims
  for (int at = threadIdx.x; at < D / 2; at += 64 * a.waves) {
    const float2 *lo = reinterpret_cast<const float2 *>(part_o + (int64_t)item * a.groups * D) + at;
    const float2 *lm = reinterpret_cast<const float2 *>(part_ml + (int64_t)item * a.groups * 2);
    float top = -INFINITY, L = 0.0f;
    float2 acc = make_float2(0.0f, 0.0f);
    for (int g0 = 0; g0 < a.groups; g0 += 8) {
      float2 e[8], v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int g = min(g0 + u, a.groups - 1);
        e[u] = load_through(lm + g);
        v[u] = load_through(lo + g * (D / 2));
      }
      float now = top;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (g0 + u >= a.groups) e[u] = make_float2(-INFINITY, 0.0f), v[u] = make_float2(0.0f, 0.0f);
        now = fmaxf(now, e[u].x);
      }
      const float to = now == -INFINITY ? 0.0f : now, corr = __builtin_amdgcn_exp2f(top - to);
      L *= corr, acc.x *= corr, acc.y *= corr;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __builtin_amdgcn_exp2f(e[u].x - to);
        L += w * e[u].y, acc.x += w * v[u].x, acc.y += w * v[u].y;
      }
      top = now;
    }
    finish(2 * at, acc.x, top, L);
    finish(2 * at + 1, acc.y, top, L);
  }
}

int validate(const dam_decode_params *p, const void *q, const dam_quant_cache *c, const int32_t *kept_ptr,
             const int32_t *kept_idx, int64_t max_kept, const void *out) {
  if (!p || !q || !c || !c->kcache || !c->vcache || !c->kscale || !c->vscale || !kept_ptr || !out) return DAM_ERR_INVALID_ARG;
  if (p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->kv_capacity < 1) return DAM_ERR_INVALID_ARG;
  if (max_kept < 0 || (max_kept > 0 && !kept_idx)) return DAM_ERR_INVALID_ARG;
  if (p->dtype != DAM_F32 && p->dtype != DAM_BF16) return DAM_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return DAM_ERR_UNSUPPORTED;
  if (!quant_format_ok(c->format, c->block)) return DAM_ERR_UNSUPPORTED;
  // a launch holds fewer than 2^32 threads, 512 to a list here, pairs counted in eights
  if (((int64_t)p->batch * p->hkv + kXcd - 1) / kXcd * kXcd * (p->hq / p->hkv) >= 1 << 23) return DAM_ERR_UNSUPPORTED;
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

// Waves of a workgroup and workgroups of a list. Sharing a list among the waves of one workgroup is nearly free, among
// workgroups it costs 3 to 5 us behind the loop.
//
// Merged lists and plans, in blocks of 32 entries: a wave per SIMD (1024) in workgroups of four as long as a wave then has no
// more than eight blocks, which it takes at some 0.8 us each; beyond that the memory is what counts, and two waves per SIMD in
// workgroups of eight keep more in flight (plan step at batch 16 / 64k, 13 blocks a wave: 38.8 us, with one wave per SIMD 45.0
// before the last steps; 32 lists of 104 blocks: one wave per SIMD 12.2, two 13.9). No more workgroups than blocks need,
// nor than 32 a list.
// A list per head, in passes of 16 (d = 128) or 32 keys per wave: up to eight waves of a workgroup, and as many workgroups as
// CUs, each with a pass at least (one sequence, 32 heads, 1640 keys: 7.4 us; 15.8 in one workgroup of 16 waves per list).
GroupSplit splits_of(const dam_decode_params *p, int64_t max_kept, bool grouped) {
  const int64_t lists = (int64_t)p->batch * (grouped ? p->hkv : p->hq);
  if (!grouped) {
    const int per_wave = 64 / (p->head_dim / 16) * kUnroll;
    int waves = 1;
    while (waves < kHeadWaves && waves * per_wave < max_kept) waves *= 2;
    return {waves, (int)std::max<int64_t>(std::min<int64_t>({256 / lists, max_kept / (waves * per_wave), (int64_t)kMostHeadGroups}), 1)};
  }
  const int64_t blocks = std::max<int64_t>(1, (max_kept + kBlk - 1) / kBlk);
  const bool heavy = blocks * lists > 8 * 1024;
  int64_t w = std::min<int64_t>(std::max<int64_t>((heavy ? 2048 : 1024) / lists, 1), blocks);
  const int64_t rounds = (blocks + w - 1) / w;
  w = (blocks + rounds - 1) / rounds;
  if (w <= kMostWaves) {
    while (heavy && (w & (w - 1))) --w;  // (workgroups of 1, 2, 4 or 8 waves share a CU without a rest)
    return {(int)w, 1};
  }
  const int per = heavy ? 8 : 4;
  return {per, (int)std::min<int64_t>({(w + per - 1) / per, 256 / lists, (int64_t)kMostGroups})};
}

// Lists per head: whether a (sequence, KV head) pair has an XCD of its own, whose L2 its heads' common rows go to. Where the pairs
// leave an XCD a quarter more work than its share, or whole XCDs idle, the workgroups are dealt out over all of them instead.
// Own XCD / dealt out: 8 pairs of 4 heads 7.4 / 8.0 us, 14 pairs 8.2 / 8.4, 20 pairs of 8 heads 11.5 / 12.6; 12 pairs 8.9 / 8.3, 18 pairs
// 10.2 / 9.1, 9 pairs of 8 heads 10.6 / 8.7, 4 pairs 8.9 / 7.6, 2 pairs of 4 heads 8.1 / 7.2, one pair of 8 heads of 3000 keys 12.4 / 7.9.
bool pair_by_xcd(int64_t pairs) { return (pairs + kXcd - 1) / kXcd * kXcd * 4 <= pairs * 5; }

// What a call writes to its workspace; lists of query heads, or of KV heads.
Partials partials(void *ws, const dam_decode_params *p, int64_t max_kept, bool grouped) {
  return Partials(ws, p, splits_of(p, max_kept, grouped).groups, (int64_t)p->batch * (grouped ? p->hkv : p->hq));
}
// The workspace query's: enough for every smaller bound of the lists too, which may be split into more workgroups.
Partials most_partials(const dam_decode_params *p, int64_t max_kept, bool grouped) {
  const int64_t lists = (int64_t)p->batch * (grouped ? p->hkv : p->hq), blocks = (max_kept + kBlk - 1) / kBlk;
  const int64_t groups = std::min<int64_t>({(blocks + 3) / 4, 256 / lists, (int64_t)(grouped ? kMostGroups : kMostHeadGroups)});
  return Partials(nullptr, p, (int)std::max<int64_t>(groups, 1), lists);
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
  bool grouped;
  Plan plan;
  void *out;
  float *lse;
  hipStream_t st;
};

template <typename T, int FORMAT, int D, bool PLAN, bool WIDE>
int launch_group(const Call &x, const QDecodeArgs &a, const Partials &part) {
  const auto kernel = k_decode_quant_group<T, FORMAT, D, PLAN, WIDE>;
  // (more than the default limit of dynamic LDS from four waves on; idempotent, set on every call)
  if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                          kMostWaves * Lds<D>::kBytes) != hipSuccess)
    return DAM_ERR_DEVICE;
  kernel<<<a.B * a.Hkv * a.groups, 64 * a.waves, (size_t)Lds<D>::kBytes * a.waves, x.st>>>(
      a, static_cast<const T *>(x.q), static_cast<const uint8_t *>(x.c->kcache), static_cast<const uint8_t *>(x.c->vcache),
      x.c->kscale, x.c->vscale, x.kept_ptr, x.kept_idx, x.kept_member, x.plan.table, part.o, part.ml, part.flags,
      static_cast<T *>(x.out), x.lse);
  return launch_status();
}

template <typename T, int FORMAT, int D, bool WIDE>
int launch_heads(const Call &x, const QDecodeArgs &a, const Partials &part) {
  const int pairs = a.by_xcd ? (a.B * a.Hkv + kXcd - 1) / kXcd * kXcd : a.B * a.Hkv;
  k_decode_quant_heads<T, FORMAT, D, WIDE><<<pairs * a.G * a.groups, 64 * a.waves, 0, x.st>>>(
      a, static_cast<const T *>(x.q), static_cast<const uint8_t *>(x.c->kcache), static_cast<const uint8_t *>(x.c->vcache),
      x.c->kscale, x.c->vscale, x.kept_ptr, x.kept_idx, part.o, part.ml, part.flags, static_cast<T *>(x.out), x.lse);
  return launch_status();
}

template <typename T, int FORMAT, int D>
int launch_form(const Call &x, const QDecodeArgs &a, const Partials &part) {
  // 32-bit offsets of rows: products of a row index and a row stride of at most 24 bits each
  const bool wide = x.p->kv_capacity >= (1 << 24) || a.kv_ss >= (1 << 24) || (uint64_t)x.p->kv_capacity * (uint64_t)a.kv_ss >= (1ull << 32);
  if (!x.grouped) return wide ? launch_heads<T, FORMAT, D, true>(x, a, part) : launch_heads<T, FORMAT, D, false>(x, a, part);
  if (x.plan.table)
    return wide ? launch_group<T, FORMAT, D, true, true>(x, a, part) : launch_group<T, FORMAT, D, true, false>(x, a, part);
  return wide ? launch_group<T, FORMAT, D, false, true>(x, a, part) : launch_group<T, FORMAT, D, false, false>(x, a, part);
}

template <typename T>
int launch_type(const Call &x, const QDecodeArgs &a, const Partials &part) {
  if (x.c->format == DAM_KV_E4M3)
    return x.p->head_dim == 128 ? launch_form<T, DAM_KV_E4M3, 128>(x, a, part) : launch_form<T, DAM_KV_E4M3, 64>(x, a, part);
  return x.p->head_dim == 128 ? launch_form<T, DAM_KV_INT8, 128>(x, a, part) : launch_form<T, DAM_KV_INT8, 64>(x, a, part);
}

// Arguments already validated, ws large enough.
int run(const Call &x, int64_t max_kept, void *ws) {
  const dam_decode_params *p = x.p;
  QDecodeArgs a;
  a.B = p->batch; a.Hq = p->hq; a.Hkv = p->hkv; a.cap = p->kv_capacity;
  a.shared_lists = p->shared_lists != 0;
  a.G = p->hq / p->hkv;
  const GroupSplit split = splits_of(p, max_kept, x.grouped);
  a.waves = split.waves; a.groups = split.groups;
  a.block_shift = x.c->block == 16 ? 4 : x.c->block == 32 ? 5 : x.c->block == 64 ? 6 : 7;
  a.by_xcd = pair_by_xcd((int64_t)p->batch * p->hkv);
  a.flag = a.groups > 1 ? fresh_flag() : 0;
  a.scale = p->scale > 0.0f ? p->scale : 1.0f / sqrtf((float)p->head_dim);
  a.q_sb = p->q_stride[0]; a.q_sh = p->q_stride[1];
  a.kv_sb = p->kv_stride[0]; a.kv_sh = p->kv_stride[1]; a.kv_ss = p->kv_stride[2];
  a.s_sb = x.c->scale_stride[0]; a.s_sh = x.c->scale_stride[1];
  a.o_sb = p->o_stride[0]; a.o_sh = p->o_stride[1];
  a.pos = x.plan.pos; a.n_flags = x.plan.n_flags;
  const Partials part = partials(ws, p, max_kept, x.grouped);
  return p->dtype == DAM_BF16 ? launch_type<__hip_bfloat16>(x, a, part) : launch_type<float>(x, a, part);
}

}  // namespace

extern "C" size_t dam_sparse_attn_decode_quantized_workspace(const dam_decode_params *p, int64_t max_kept) {
  if (!p || p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->head_dim < 1 || max_kept < 0) return 0;
  return bytes_up_to_batch(p, [&](const dam_decode_params *x) { return most_partials(x, max_kept, false); });
}

extern "C" size_t dam_sparse_attn_decode_grouped_quantized_workspace(const dam_decode_params *p, int64_t max_kept) {
  if (!p || p->batch < 1 || p->hq < 1 || p->hkv < 1 || p->hq % p->hkv || p->head_dim < 1 || max_kept < 0) return 0;
  return bytes_up_to_batch(p, [&](const dam_decode_params *x) { return most_partials(x, max_kept, true); });
}

extern "C" int dam_sparse_attn_decode_quantized(const dam_decode_params *p, const void *q, const dam_quant_cache *cache,
                                                const int32_t *kept_ptr, const int32_t *kept_idx, int64_t max_kept, void *out,
                                                float *lse, void *ws, size_t ws_bytes, void *stream_v) {
  const int bad = validate(p, q, cache, kept_ptr, kept_idx, max_kept, out);
  if (bad != DAM_OK) return bad;
  if (!aligned16(ws)) return DAM_ERR_INVALID_ARG;
  if (!ws || ws_bytes < partials(nullptr, p, max_kept, false).bytes) return DAM_ERR_WORKSPACE;
  return run({p, q, cache, kept_ptr, kept_idx, nullptr, false, {}, out, lse, static_cast<hipStream_t>(stream_v)}, max_kept, ws);
}

extern "C" int dam_sparse_attn_decode_grouped_quantized(const dam_decode_params *p, const void *q, const dam_quant_cache *cache,
                                                        const int32_t *kept_ptr, const int32_t *kept_idx,
                                                        const uint8_t *kept_member, int64_t max_kept, void *out, float *lse,
                                                        void *ws, size_t ws_bytes, void *stream_v) {
  const int bad = validate_grouped(p, q, cache, kept_ptr, kept_idx, kept_member, max_kept, out);
  if (bad != DAM_OK) return bad;
  if (!aligned16(ws)) return DAM_ERR_INVALID_ARG;
  if (!ws || ws_bytes < partials(nullptr, p, max_kept, true).bytes) return DAM_ERR_WORKSPACE;
  return run({p, q, cache, kept_ptr, kept_idx, kept_member, true, {}, out, lse, static_cast<hipStream_t>(stream_v)}, max_kept, ws);
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
  if (!aligned16(ws)) return DAM_ERR_INVALID_ARG;
  if (!ws || ws_bytes < partials(nullptr, &shared, max_entries, true).bytes) return DAM_ERR_WORKSPACE;
  return run({&shared, q, cache, plan_ptr, plan_val, plan_member, true, {plan_table, n_flags, pos}, out, lse,
              static_cast<hipStream_t>(stream_v)}, max_entries, ws);
}
