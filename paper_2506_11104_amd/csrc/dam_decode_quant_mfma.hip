// The grouped decodes over a cache of 8-bit codes on the matrix cores: bf16 queries, head_dim 128, merged lists and plans.
//
// Paper (arXiv 2506.11104): Sec. 3 (scaled dot-product attention) with the mask of Sec. 4.3 applied as -inf before the
// softmax; the merged list is row p of the masks of a KV head's query heads. Codes and scales: dam_quant.h.
//
// The G query vectors of a (sequence, KV head) pair are columns of the B operand of S^T = K Q^T and, as softmax weights, of
// O^T += V^T P^T, in blocks of 32 keys. HBM bound (256 bytes per listed key, half of a bf16 cache's), so what counts is that
// the arithmetic of a block stays under the block's share of the memory's time (8 KB per wave, eight waves per CU: some 4000
// cycles): the codes become bf16 on the way from LDS to the products, which is exact, and the scales enter per key: K's in the
// conversion (e4m3) or on the logits (int8), V's on the weights.
// A weight has 8 significant bits as a bf16 number. Columns 16 .. 16 + G, which the products compute anyway, hold the same
// heads once more with what the weights of columns 0 .. G lose: 16 bits together, so the result is as exact as one of fp32
// weights, for no matrix instruction more.
//
// A wave owns every splits-th block of 32 list entries and two LDS slots of K and V rows (4 KiB each), filled by load-to-LDS
// copies whose addresses come from the list; the entries are staged three blocks ahead and the scale bytes with the rows, by
// the same kind of copy, so that every vector-memory operation of the loop is one of these copies and the waits are counted
// by hand. The waves of a workgroup merge their results through LDS, workgroups that share a list through memory, in the
// last one of them to finish.
#include <math.h>

#include "dam_internal.h"
#include "dam_mfma.h"
#include "dam_quant.h"

namespace {
using namespace dam;

constexpr int kBlk = 32;                    // keys per block
constexpr int kSlot = kBlk * 128;           // bytes of the K (or V) rows of a block
constexpr int kVSlots = 2 * kSlot;          // two K slots, then two V slots
constexpr int kEntries = 4 * kSlot;         // then four slots of 32 list entries and their member bytes
constexpr int kScales = kEntries + 4 * 256; // four slots of 32 words with a K scale, 32 with a V scale
constexpr int kFix = kScales + 4 * 256;     // PLAN: four slots of plan-table words
constexpr int kFloat = kFix + 4 * 256;      // the block's 32 V scales (and K scales) as fp32
constexpr int kMember = kFloat + 256;       // member bytes of the next block's keys, by key
constexpr int kLds = kMember + 64;
constexpr int kPart = 8 * 32 * 16;          // a wave's results: O of at most 8 heads at 0, what columns 16.. add to it here,
constexpr int kMl = 2 * kPart;              // (reference, sum) here

struct QMfmaArgs {
  int B, Hq, Hkv, cap, shared_lists;
  int waves, groups;  // a list is shared by `waves` waves of each of `groups` workgroups
  int block_shift;    // log2 of the rows that share a scale
  uint64_t flag;
  float scale;
  int64_t q_sb, q_sh, kv_sb, kv_sh, s_sb, s_sh, o_sb, o_sh;
  unsigned row_bytes;  // byte stride of a cache row
  int pos, n_flags;    // PLAN: position of the query row, length P of the pattern flags
};

// Four bytes per lane from a 64-bit address of the lane's own to LDS address lds_at + 4 * lane.
__device__ __forceinline__ void lds_copy4_at(unsigned lds_at, uint64_t addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_at), "v"(addr) : "memory", "m0");
}

// Where the 16-byte chunk c of row r of a block lies in its LDS row: at position c ^ spread(r). Sixteen rows read at one
// chunk, as K's operand does, and eight rows {0..3, 8..11} or {4..7, 12..15} read at two chunks 2 i and 2 i + 1, as V's does,
// then touch every bank once.
__device__ __forceinline__ int spread(int r) { return ((r >> 3) & 1) << 2 | ((r >> 1) & 1) << 1 | ((r >> 2) & 1); }

// All ones where bit POS of a word is clear.
__device__ __forceinline__ unsigned unset(unsigned w, int pos) { return ~(unsigned)__builtin_amdgcn_sbfe((int)w, pos, 1); }

__device__ __forceinline__ u32x2 lds_read_tr8(const unsigned char *lds, int byte) {
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                       (__attribute__((address_space(3))) i32x2 *)(const_cast<unsigned char *>(lds + byte))));
}

// Codes 2 i and 2 i + 1 of a word, as two bf16 numbers, times a scale (e4m3 only).
template <int FORMAT>
__device__ __forceinline__ unsigned to_bf16(unsigned w, int i, float scale) {
  if constexpr (FORMAT == DAM_KV_E4M3) {
    const auto r = i ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    return __builtin_bit_cast(unsigned, r);
  } else {
    return pack_bf16((float)(int8_t)(w >> (16 * i)), (float)(int8_t)(w >> (16 * i + 8)));  // (exact)
  }
}

template <int FORMAT, bool PLAN>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_decode_quant_mfma(
    QMfmaArgs a, const __hip_bfloat16 *__restrict__ q, const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
    const uint8_t *__restrict__ ks, const uint8_t *__restrict__ vs, const int *__restrict__ kept_ptr,
    const int *__restrict__ kept_idx, const uint8_t *__restrict__ kept_member, const uint8_t *__restrict__ plan_table,
    float *__restrict__ part_o, float *__restrict__ part_ml, uint64_t *__restrict__ flags, __hip_bfloat16 *__restrict__ out,
    float *__restrict__ lse) {
  using C = Code<FORMAT>;
  constexpr bool kScaleOnLogits = FORMAT == DAM_KV_INT8;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_all[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char *lds = lds_all + wave * kLds;  // this wave's slots
  const int n = lane & 31, hf = lane >> 5;     // column of the products, half-wave
  const int head = n & 15;                     // query head of the group; columns from 16 on hold what the weights lose
  const int sub = lane >> 3, pos = lane & 7;   // copies: row within the instruction's eight, 16-byte position
  const int G = a.Hq / a.Hkv;
  const int group = (int)blockIdx.x % a.groups, pair = (int)blockIdx.x / a.groups;
  const int splits = a.waves * a.groups, split = group * a.waves + wave;
  const int b = pair / a.Hkv, hkv = pair % a.Hkv;
  const int list = a.shared_lists ? hkv : pair;
  const int lo = __builtin_amdgcn_readfirstlane(kept_ptr[list]), end = __builtin_amdgcn_readfirstlane(kept_ptr[list + 1]);
  const int n_blocks = (end - lo + kBlk - 1) / kBlk;
  // this wave's blocks are split, split + splits, ...: every wave gets its share of each run of the list
  const int nb = n_blocks > split ? (n_blocks - split + splits - 1) / splits : 0;
  const float c2 = a.scale * 1.4426950408889634f;
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;

  f32x16 oacc[4];
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[db][e] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;  // reference of the weights (raw logits), this lane's part of their sum

  if (nb > 0) {
    const unsigned char *kg = kc + b * a.kv_sb + hkv * a.kv_sh, *vg = vc + b * a.kv_sb + hkv * a.kv_sh;
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
      const uint64_t addr = lane < 32 ? idx_at + 4ull * (unsigned)min(e0 + lane, end - 1)
                                      : min(first + 4u * (unsigned)min(lane - 32, 8), last);
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + kEntries + (i & 3) * 256), addr);
    };
    auto entry = [&](int i, int k) { return *reinterpret_cast<const int *>(lds + kEntries + (i & 3) * 256 + 4 * k); };
    // PLAN: the aligned word that holds table[pos - c] for every column entry c of local block i (its entries have
    // landed) -> fix slot i & 3, lane k < 32 for entry k; every other lane and entry fetches the table's first word.
    // (A block without a column entry issues no copy: the copy, when there is one, is older than the copies of the
    // block's scales and rows, which are all that the waits below leave outstanding.)
    auto table_index = [&](int v) { return (v >= 0 && v <= a.pos && a.pos - v < a.n_flags) ? a.pos - v : -1; };
    auto copy_fix = [&](int i) {
      const int t = lane < 32 ? table_index(entry(i, lane & 31)) : -1;
      if (__builtin_amdgcn_ballot_w64(t >= 0) == 0) return;
      const uint64_t addr = t >= 0 ? (table_at + (unsigned)t) & ~(uint64_t)3 : reinterpret_cast<uint64_t>(plan_table) & ~(uint64_t)3;
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + kFix + (i & 3) * 256), addr);
    };
    // Scales and rows of local block i: one copy of the words that hold the 32 keys' scale bytes, four of K rows and four of
    // V rows into slot i & 1, LDS row r for key r of the block. Returns where in those words the scale bytes of key lane & 31
    // lie (bits of K's, and of V's from bit 8 on).
    auto copy_rows = [&](int i) {
      const unsigned k_at = __builtin_amdgcn_readfirstlane(lds_base + (i & 1) * kSlot);
      const unsigned v_at = k_at + kVSlots;
      unsigned off[4];
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int r = 8 * it + sub;
        // (row index and row stride are below 2^24: the 24-bit multiply runs at full rate, the 32-bit one does not)
        off[it] = __umul24((unsigned)row_of(entry(i, r)), a.row_bytes) + ((pos ^ spread(r)) << 4);
      }
      const unsigned s = (unsigned)row_of(entry(i, n)) >> a.block_shift;
      lds_copy4_at(__builtin_amdgcn_readfirstlane(lds_base + kScales + (i & 3) * 256), ((hf ? vs_at : ks_at) + s) & ~(uint64_t)3);
      lds_copy16_once<0 * 1024>(k_at, kg, off[0]);
      lds_copy16_once<1 * 1024>(k_at, kg, off[1]);
      lds_copy16_once<2 * 1024>(k_at, kg, off[2]);
      lds_copy16_once<3 * 1024>(k_at, kg, off[3]);
      lds_copy16_once<0 * 1024>(v_at, vg, off[0]);
      lds_copy16_once<1 * 1024>(v_at, vg, off[1]);
      lds_copy16_once<2 * 1024>(v_at, vg, off[2]);
      lds_copy16_once<3 * 1024>(v_at, vg, off[3]);
      return (((unsigned)ks_at + s) & 3) * 8 | (((unsigned)vs_at + s) & 3) * 0x800;
    };
    // Which heads keep which key of local block i (its entries and table words have landed): a byte per key, dealt out so
    // that bit 8 (e % 4) of word e / 4 says whether this lane's head keeps the key of accumulator e, 8 (e / 4) + 4 hf + e % 4.
    struct Kept {
      unsigned w[4];
    };
    const int member_shift = (int)((member_at + (unsigned)lo) & 3);  // (blocks start a multiple of 32 entries apart)
    auto keeps = [&](int i) {
      unsigned mem = lds[kEntries + (i & 3) * 256 + 128 + member_shift + n];
      if (entry0(i) + n >= end) mem = 0u;
      if (PLAN) {
        const int v = entry(i, n);
        const bool exists = v < 0 ? a.pos + 1 + v >= 0 : v <= a.pos;
        const int t = table_index(v);
        unsigned covered = 0;  // heads that reach this column's key through a matched diagonal
        if (t >= 0) {
          const unsigned word = *reinterpret_cast<const unsigned *>(lds + kFix + (i & 3) * 256 + 4 * n);
          covered = (word >> (8 * (int)((table_at + (unsigned)t) & 3))) & 0xFFu;
        }
        mem = exists ? mem & ~covered : 0u;
      }
      lds[kMember + n] = (unsigned char)mem;  // (both half-waves hold the same)
      Kept k;
#pragma unroll
      for (int g = 0; g < 4; ++g) k.w[g] = *reinterpret_cast<const unsigned *>(lds + kMember + 8 * g + 4 * hf) >> head;
      return k;
    };

    // Q fragments: B operand of S^T = K Q^T. Column n is query head `head` of the group (zero beyond the group); fragment c
    // of this lane covers dims 64 hf + 8 c .. + 7 (the order of the dims in the contraction is K's).
    bf16x8 qf[8];
    {
      const __hip_bfloat16 *qp = q + b * a.q_sb + (int64_t)(hkv * G + min(head, G - 1)) * a.q_sh + 64 * hf;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (head < G) raw = *reinterpret_cast<const u32x4 *>(qp + 8 * c);
        qf[c] = __builtin_bit_cast(bf16x8, raw);
      }
    }
    copy_entries(0);
    if (nb > 1) copy_entries(1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // (the Q fragments have arrived with that wait; the empty statement tells the compiler so)
#pragma unroll
    for (int c = 0; c < 8; ++c) asm volatile("" : "+v"(qf[c]));
    if (PLAN) {
      copy_fix(0);
      if (nb > 1) copy_fix(1);
    }
    if (nb > 2) copy_entries(2);
    unsigned bits_now = copy_rows(0), bits_next = 0;
    if (nb > 1) bits_next = copy_rows(1);

    const float lost = n >= 16 ? 1.0f : 0.0f;           // this column's weights are what bf16 loses
    float *vsf = reinterpret_cast<float *>(lds + kFloat), *ksf = vsf + 32;
    // LDS byte offsets of this lane's operand fragments in a slot; the others differ by an XOR (and a2 by 2048 bytes). K: row n,
    // chunks 4 hf .. 4 hf + 3. V: a transposing read takes eight bytes of a row per lane (lanes 2 r and 2 r + 1 of sixteen the 16
    // bytes of row r of eight) and leaves a lane the byte of its own column of all eight rows: lane n dim 32 db + n of the
    // keys 16 a2 + 4 hf + {0..3, 8..11}, the order in which the lane holds weights.
    const int kbase = n * 128 + (((4 * hf) ^ spread(n)) << 4);
    const int vrow = 4 * hf + ((lane >> 1) & 3) + 8 * ((lane >> 3) & 1);
    const int vbase = vrow * 128 + ((((lane >> 4) & 1) ^ spread(vrow)) << 4) + 8 * (lane & 1);
    Kept kept_now, kept_next;

    for (int i = 0; i < nb; ++i) {
      // The copies were issued in the order ... rows i, entries i + 2 (PLAN: table words i + 1), scales and rows i + 1: what
      // block i needs and the entries of block i + 2 have landed once nothing but the nine copies of block i + 1's scales and
      // rows is outstanding.
      if (i + 1 < nb) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const unsigned char *kslot = lds + (i & 1) * kSlot;
      const unsigned char *vslot = lds + kVSlots + (i & 1) * kSlot;

      // Everything the block needs from LDS is asked for at once, for its latency to be paid once.
      const unsigned *words = reinterpret_cast<const unsigned *>(lds + kScales + (i & 3) * 256);
      const unsigned kword = words[n], vword = words[32 + n], vfirst = vslot[n * 128];
      u32x4 kw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kw[j] = *reinterpret_cast<const u32x4 *>(kslot + (kbase ^ (j << 4)));
      if (i == 0) kept_now = keeps(0);
      u32x2 vw[2][4];
#pragma unroll
      for (int a2 = 0; a2 < 2; ++a2)
#pragma unroll
        for (int db = 0; db < 4; ++db) vw[a2][db] = lds_read_tr8(vslot, (vbase ^ (db << 5)) + 2048 * a2);

      // Scales of key n of the block. NaN rows: the scale carries the NaN, which reaches the heads that keep the row through
      // the logits (K's codes do so themselves in e4m3) or the weights; a V row's codes are cleared, since the product would
      // carry them to all heads.
      float kscale = scale_value((kword >> (bits_now & 31)) & 0xFFu);
      float vscale = scale_value((vword >> (bits_now >> 8)) & 0xFFu);
      const bool vbad = C::is_nan(vfirst);
      if (vbad) vscale = NAN;
      const unsigned vbads = (unsigned)__ballot(vbad);
      if (kScaleOnLogits && C::is_nan(kw[0][0])) kscale = NAN;
      if (hf == 0) {
        vsf[n] = vscale;
        if (kScaleOnLogits) ksf[n] = kscale;
      }

      // S^T = K Q^T; accumulator e is key 8 (e / 4) + 4 hf + e % 4
      f32x16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const u32x4 f = {to_bf16<FORMAT>(kw[j][2 * z], 0, kscale), to_bf16<FORMAT>(kw[j][2 * z], 1, kscale),
                           to_bf16<FORMAT>(kw[j][2 * z + 1], 0, kscale), to_bf16<FORMAT>(kw[j][2 * z + 1], 1, kscale)};
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), qf[2 * j + z], s, 0, 0, 0);
        }
      if (i + 1 < nb) kept_next = keeps(i + 1);
      if (kScaleOnLogits) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 f = *reinterpret_cast<const float4 *>(ksf + 8 * g + 4 * hf);
          s[4 * g] *= f.x, s[4 * g + 1] *= f.y, s[4 * g + 2] *= f.z, s[4 * g + 3] *= f.w;
        }
      }
      // masked keys to -inf (after the products, so that a NaN row does not get past it)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const unsigned off = unset(kept_now.w[e / 4], 8 * (e % 4));
        s[e] = __uint_as_float((off & 0xFF800000u) | (~off & __float_as_uint(s[e])));
      }

      // online softmax, one head per lane pair (lane, lane ^ 32); the reference the weights are taken against
      // only moves when the maximum has grown past it by more than 8 in log2 units
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      {
        const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
      }
      const float m_top = fmaxf(m_run, mx);
      const bool move = (m_top - m_run) * c2 > 8.0f;  // (-inf) - (-inf) is NaN: no move
      const float m_new = move ? m_top : m_run;
      const float m_ref = m_new == -INFINITY ? 0.0f : m_new;
      const float off = m_ref * c2;
      if (__ballot(move)) {
        const float corr = move ? __builtin_amdgcn_exp2f((m_run - m_ref) * c2) : 1.0f;  // old reference -inf: 0
        l_run *= corr;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] *= corr;
      }
      m_run = m_new;
      // the weights, times the scales of V's rows; the sum is taken over the weights themselves
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -off));
#pragma unroll
      for (int g = 0; g < 4; ++g) l_run += (w[4 * g] + w[4 * g + 1]) + (w[4 * g + 2] + w[4 * g + 3]);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 f = *reinterpret_cast<const float4 *>(vsf + 8 * g + 4 * hf);
        w[4 * g] *= f.x, w[4 * g + 1] *= f.y, w[4 * g + 2] *= f.z, w[4 * g + 3] *= f.w;
      }
      if (vbads) {  // (wave-uniform) a weight of 0 times a NaN scale; the rows' codes
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = __uint_as_float(~unset(kept_now.w[e / 4], 8 * (e % 4)) & __float_as_uint(w[e]));
#pragma unroll
        for (int a2 = 0; a2 < 2; ++a2)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            // bits k of the keys in bytes k of the word
            const unsigned gone = (((vbads >> (16 * a2 + 8 * z + 4 * hf)) & 15u) * 0x204081u & 0x01010101u) * 0xFFu;
#pragma unroll
            for (int db = 0; db < 4; ++db) vw[a2][db][z] &= ~gone;
          }
      }
      // the upper 16 bits of a weight, or, in the columns from 16 on, those of what remains
      unsigned p[8];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float r0 = __builtin_fmaf(-lost, __uint_as_float(__float_as_uint(w[e]) & 0xFFFF0000u), w[e]);
        const float r1 = __builtin_fmaf(-lost, __uint_as_float(__float_as_uint(w[e + 1]) & 0xFFFF0000u), w[e + 1]);
        p[e / 2] = __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x07060302u);
      }

      // O^T += V^T P^T: accumulator e of dim block db is dim 32 db + 8 (e / 4) + 4 hf + e % 4
#pragma unroll
      for (int a2 = 0; a2 < 2; ++a2) {
        const u32x4 praw = {p[4 * a2], p[4 * a2 + 1], p[4 * a2 + 2], p[4 * a2 + 3]};
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const u32x2 x = vw[a2][db];
          const u32x4 f = {to_bf16<FORMAT>(x[0], 0, 1.0f), to_bf16<FORMAT>(x[0], 1, 1.0f), to_bf16<FORMAT>(x[1], 0, 1.0f),
                           to_bf16<FORMAT>(x[1], 1, 1.0f)};
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, praw), oacc[db],
                                                             0, 0, 0);
        }
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

  // The waves' results meet in LDS, dealt out in columns as everything from here on: column c G + x is dims 4 c .. + 3 of
  // head x, 16 bytes at 16 (c G + x) of the wave's own slots, what columns 16 .. add to it kPart further; behind them the
  // head's reference (log2 units) and sum.
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  if (head < G) {
    float4 *mine_o = reinterpret_cast<float4 *>(lds + (n >= 16 ? kPart : 0)) + head;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        mine_o[(8 * db + 2 * g + hf) * G] =
            make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2], oacc[db][4 * g + 3]);
    if (lane < 16) reinterpret_cast<float2 *>(lds + kMl)[n] = make_float2(m_run == -INFINITY ? -INFINITY : m_run * c2, l_tot);
  }
  __syncthreads();
  const int cols = G * 32;
  auto finish = [&](int x, int c, const float4 &o, float M, float L) {
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;  // (L = 0: no key; NaN stays)
    const int hq = hkv * G + x;
    __hip_bfloat16 *op = out + b * a.o_sb + hq * a.o_sh + 4 * c;
    const unsigned p0 = pack_bf16(o.x * inv, o.y * inv), p1 = pack_bf16(o.z * inv, o.w * inv);
    if ((reinterpret_cast<uintptr_t>(op) & 7) == 0) {
      *reinterpret_cast<uint2 *>(op) = make_uint2(p0, p1);
    } else {
      unsigned short *us = reinterpret_cast<unsigned short *>(op);
      us[0] = (unsigned short)p0, us[1] = (unsigned short)(p0 >> 16), us[2] = (unsigned short)p1, us[3] = (unsigned short)(p1 >> 16);
    }
    if (lse && c == 0) lse[(int64_t)b * a.Hq + hq] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  };
  float4 *po = reinterpret_cast<float4 *>(part_o) + (int64_t)pair * a.groups * cols;  // [group][column]
  float *ml = part_ml + (int64_t)pair * a.groups * G * 2;                             // [group][head][2]
  for (int col = threadIdx.x; col < cols; col += blockDim.x) {
    const int x = col % G, c = col / G;
    float M = -INFINITY, L = 0.0f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < a.waves; ++w) M = fmaxf(M, reinterpret_cast<const float2 *>(lds_all + w * kLds + kMl)[x].x);
    const float ref = M == -INFINITY ? 0.0f : M;
    for (int w = 0; w < a.waves; ++w) {  // weights 2^(reference - largest reference)
      const float4 ow = reinterpret_cast<const float4 *>(lds_all + w * kLds)[col];
      const float4 ol = reinterpret_cast<const float4 *>(lds_all + w * kLds + kPart)[col];
      const float2 e = reinterpret_cast<const float2 *>(lds_all + w * kLds + kMl)[x];
      const float wt = __builtin_amdgcn_exp2f(e.x - ref);
      L += wt * e.y;
      o.x += wt * (ow.x + ol.x);
      o.y += wt * (ow.y + ol.y);
      o.z += wt * (ow.z + ol.z);
      o.w += wt * (ow.w + ol.w);
    }
    if (a.groups == 1) {
      finish(x, c, o, M, L);
    } else {
      store_through(po + group * cols + col, o.x, o.y, o.z, o.w);
      if (c == 0) {
        store_through(ml + (group * G + x) * 2, M);
        store_through(ml + (group * G + x) * 2 + 1, L);
      }
    }
  }
  if (a.groups == 1) return;
  stores_done();
  __syncthreads();
  int *last = reinterpret_cast<int *>(lds_all + kEntries);  // (the results above lie below)
  if (wave == 0) {
    const bool is_last = arrive_last(flags + (int64_t)pair * a.groups, a.groups, group, a.flag);
    if (lane == 0) *last = is_last;
  }
  __syncthreads();
  if (!*last) return;
  // The last workgroup merges the groups. Threads that share a column take them in turn, four fetched at a time.
  const int shares = blockDim.x / cols, col = threadIdx.x % cols, share = threadIdx.x / cols;
  const int x = col % G;
  float M = -INFINITY, L = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (share < shares)
    for (int g0 = share; g0 < a.groups; g0 += 4 * shares) {
      float gm[4], gl[4], top = M;
      float2 go[4][2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int gr = min(g0 + u * shares, a.groups - 1);
        const float2 e = load_through(reinterpret_cast<const float2 *>(ml) + gr * G + x);
        const bool here = g0 + u * shares < a.groups;
        gm[u] = here ? e.x : -INFINITY;
        gl[u] = here ? e.y : 0.0f;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          go[u][z] = load_through(reinterpret_cast<const float2 *>(po + gr * cols + col) + z);
          if (!here) go[u][z] = make_float2(0.0f, 0.0f);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) top = fmaxf(top, gm[u]);
      const float ref = top == -INFINITY ? 0.0f : top;
      const float corr = __builtin_amdgcn_exp2f(M - ref);
      L *= corr;
      o.x *= corr, o.y *= corr, o.z *= corr, o.w *= corr;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float wt = __builtin_amdgcn_exp2f(gm[u] - ref);
        L += wt * gl[u];
        o.x += wt * go[u][0].x;
        o.y += wt * go[u][0].y;
        o.z += wt * go[u][1].x;
        o.w += wt * go[u][1].y;
      }
      M = top;
    }
  float4 *sum = reinterpret_cast<float4 *>(lds_all);  // [thread] O, then [thread] (M, L)
  float2 *sum_ml = reinterpret_cast<float2 *>(lds_all + 256 * sizeof(float4));
  if (shares > 1) {
    sum[threadIdx.x] = o;
    sum_ml[threadIdx.x] = make_float2(M, L);
    __syncthreads();
    if (share > 0) return;
    for (int y = 1; y < shares; ++y) {
      const float4 oy = sum[y * cols + col];
      const float2 e = sum_ml[y * cols + col];
      const float top = fmaxf(M, e.x), ref = top == -INFINITY ? 0.0f : top;
      const float w0 = __builtin_amdgcn_exp2f(M - ref), w1 = __builtin_amdgcn_exp2f(e.x - ref);
      L = w0 * L + w1 * e.y;
      o.x = w0 * o.x + w1 * oy.x;
      o.y = w0 * o.y + w1 * oy.y;
      o.z = w0 * o.z + w1 * oy.z;
      o.w = w0 * o.w + w1 * oy.w;
      M = top;
    }
  }
  if (share == 0) finish(x, col / G, o, M, L);
}

template <int FORMAT, bool PLAN>
int launch(const QMfmaArgs &a, const void *q, const dam_quant_cache *c, const int32_t *kept_ptr, const int32_t *kept_idx,
           const uint8_t *kept_member, const uint8_t *plan_table, float *part_o, float *part_ml, uint64_t *flags, void *out,
           float *lse, hipStream_t st) {
  const auto kernel = k_decode_quant_mfma<FORMAT, PLAN>;
  // (more than the default limit of dynamic LDS with four waves; idempotent, set on every call)
  if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * kLds) != hipSuccess)
    return DAM_ERR_DEVICE;
  kernel<<<a.B * a.Hkv * a.groups, 64 * a.waves, (size_t)kLds * a.waves, st>>>(
      a, static_cast<const __hip_bfloat16 *>(q), static_cast<const uint8_t *>(c->kcache), static_cast<const uint8_t *>(c->vcache),
      c->kscale, c->vscale, kept_ptr, kept_idx, kept_member, plan_table, part_o, part_ml, flags,
      static_cast<__hip_bfloat16 *>(out), lse);
  return launch_status();
}

}  // namespace

namespace dam {

bool decode_quant_mfma_fits(const dam_decode_params *p) {
  if (p->dtype != DAM_BF16 || p->head_dim != 128 || p->hq / p->hkv > 8) return false;
  // row addresses are a base per (sequence, KV head) plus a 32-bit byte offset, the product of a row index and a
  // row stride of at most 24 bits each
  if (p->kv_capacity >= (1 << 24) || p->kv_stride[2] >= (1 << 24)) return false;
  return (uint64_t)p->kv_capacity * (uint64_t)p->kv_stride[2] < (1ull << 32);
}

int launch_decode_quant_mfma(const dam_decode_params *p, GroupSplit split, float scale, const void *q, const dam_quant_cache *c,
                             int block_shift, const int32_t *kept_ptr, const int32_t *kept_idx, const uint8_t *kept_member,
                             float *part_o, float *part_ml, uint64_t *flags, void *out, float *lse, hipStream_t st,
                             const uint8_t *plan_table, int n_flags, int pos) {
  QMfmaArgs a;
  a.B = p->batch; a.Hq = p->hq; a.Hkv = p->hkv; a.cap = p->kv_capacity;
  a.shared_lists = p->shared_lists != 0;
  a.waves = split.waves; a.groups = split.groups;
  a.block_shift = block_shift;
  a.flag = split.groups > 1 ? fresh_flag() : 0;
  a.scale = scale;
  a.q_sb = p->q_stride[0]; a.q_sh = p->q_stride[1];
  a.kv_sb = p->kv_stride[0]; a.kv_sh = p->kv_stride[1];
  a.s_sb = c->scale_stride[0]; a.s_sh = c->scale_stride[1];
  a.o_sb = p->o_stride[0]; a.o_sh = p->o_stride[1];
  a.row_bytes = (unsigned)p->kv_stride[2];
  a.pos = pos; a.n_flags = n_flags;
  const bool e4m3 = c->format == DAM_KV_E4M3;
  if (plan_table)
    return e4m3 ? launch<DAM_KV_E4M3, true>(a, q, c, kept_ptr, kept_idx, kept_member, plan_table, part_o, part_ml, flags, out, lse, st)
                : launch<DAM_KV_INT8, true>(a, q, c, kept_ptr, kept_idx, kept_member, plan_table, part_o, part_ml, flags, out, lse, st);
  return e4m3 ? launch<DAM_KV_E4M3, false>(a, q, c, kept_ptr, kept_idx, kept_member, nullptr, part_o, part_ml, flags, out, lse, st)
              : launch<DAM_KV_INT8, false>(a, q, c, kept_ptr, kept_idx, kept_member, nullptr, part_o, part_ml, flags, out, lse, st);
}

}  // namespace dam
