// Attention of many query rows over a paged cache: what prompts and trees of drafted tokens share.
//
// A KV head's rows are its sequence's new tokens times the query heads of its group, token by token: row r is
// head r % G of token r / G, so that whatever the group the keys are read once for all of them.
// Rows are cut into tiles of kRows.  A tile walks the tokens it attends to 64 at a time with an online softmax.
//
// Work-groups have to know their sequence without the host knowing any length: sequence b's tiles start at slot
// floor(cu[b] G / kRows) + b, which leaves room for ceil(n_b G / kRows) of them; slots without rows end at once.
//
// On the matrix cores, v_mfma_f32_32x32x16_f16 throughout (lane l: c = l % 32, h = l / 32):
//   logits   S^T = K Q^T: first operand 32 tokens, second operand 32 query rows; a lane gets of its row c the
//            tokens 8 (r / 4) + 4 h + r % 4, r = 0..15.  A row's maximum and sum are over registers and one
//            exchange between the halves of the wave.
//   outputs  O^T = V^T P^T: the weights that a lane has are what it needs as second operand if the 16 tokens of a
//            product are taken in the order 4 h + j, 8 + 4 h + j (j = 0..3): nothing moves between lanes.  The
//            first operand is V with rows and columns exchanged, read that way from LDS (ds_read_b64_tr_b16).
// Tokens lie in LDS as rows of 256 bytes.  The 16-byte chunks of a key are exclusive-ored with its token, those of a
// value with 4 (token % 4): the lanes of a read spread over all banks.
//
// Weights go to the product in fp16.  For fp16 outputs one rounding of each weight, 2^-11 of it, which is what the
// output's own rounding costs; the reference exponent is put 7 below the largest logit (log2) seen when it last
// moved and moves when a weight would pass 2^15, so weights keep all bits down to 2^-21 of the largest and are not
// lost down to 2^-32.  For fp32 outputs a weight is two fp16 numbers, 2^14 times its value rounded and what that leaves: 22
// bits of it.  Sums, maxima and accumulators are fp32.
#pragma once

#include <type_traits>

#include "quest_common.h"
#include "quest_decode_core.h"

namespace quest {

struct RowsArgs {
  const char* q;
  const char* k_pool;
  const char* v_pool;
  const int32_t* cu;
  const int32_t* seq_lens;
  void* out;
  float* lse;
  float* part_acc;          // [splits][slots][kv heads][kRows][D]
  float* part_ml;           // [splits][slots][kv heads][kRows][2]: reference exponent, sum
  const char* k_new;        // trees: keys and values of the drafted nodes
  const char* v_new;
  const int64_t* mask;      // trees: [rows of cu][mask_words]
  int64_t q_stride, new_stride;   // bytes between tokens
  int batch, max_pages, page_shift, kv_heads, group;
  int slots, splits, mask_words, k_pages;
  int out_is_fp16;
  uint32_t q_sign;          // exclusive-ored onto q: sign bits where the scale is negative
  float scale_log2;         // |sm_scale| log2(e), not 0
};

constexpr int kTileTokens = 64;

#if defined(__HIPCC__)

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// The sequence and tile of a slot (see above); false: the slot has no rows.
struct RowTile {
  int b, first;        // sequence, first packed token of it
  int tokens;          // its new tokens
  int row0, rows;      // the tile's first row, rows of the sequence
};
template <int kRows>
__device__ __forceinline__ bool find_tile(RowTile& t, const int32_t* __restrict__ cu, int batch, int group, int slot,
                                          int lane) {
  int b = -1;
  for (int base = 0; base < batch; base += kWave) {  // the last sequence that starts at or before the slot
    const int i = base + lane;
    const bool before = i < batch && (int64_t)cu[i < batch ? i : 0] * group / kRows + i <= slot;
    const int n = __popcll(__ballot(before));
    b += n;
    if (n < kWave) break;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  t.b = b;
  t.first = cu[b];
  t.tokens = cu[b + 1] - t.first;
  t.rows = t.tokens * group;
  const int tile = slot - (int)((int64_t)t.first * group / kRows) - b;
  t.row0 = tile * kRows;
  return t.row0 < t.rows;
}

// Attention state of a wave's 32 rows; lane l: row l % 32.
template <bool kExact>
struct RowState {
  static constexpr float kBelow = kExact ? 0.f : 7.f;    // the reference lies this far below the largest logit
  static constexpr float kMove = kExact ? 1.f : 15.f;    // and moves when a logit is this far above it (log2)
  half8_t q[8];        // channels 16 i + 8 h ..+7
  f32x16_t acc[4];     // [d / 32]: channels 8 (r / 4) + 4 h + r % 4
  float ref, l;        // reference exponent; this lane's share of the row's sum

  __device__ __forceinline__ void init(const char* row, bool there, uint32_t sign, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint4 v = there ? ld16(row + i * 32 + (lane >> 5) * 16) : make_uint4(0, 0, 0, 0);
      v.x ^= sign, v.y ^= sign, v.z ^= sign, v.w ^= sign;
      q[i] = __builtin_bit_cast(half8_t, v);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    ref = kNegBig;
    l = 0.f;
  }

  // Fold a tile of 32 kBlocks tokens that lies in LDS.  masked: only the tokens of `allow` (bit t: token t of
  // the tile; a lane's own) count.
  template <int kBlocks>
  __device__ __forceinline__ void fold(const char* k, const char* v, float scale, bool masked, uint64_t allow, int lane) {
    f32x16_t s[kBlocks];
    const char* k_lane = k + (lane & 31) * kRowBytes;
    const int k_chunk = ((lane >> 5) ^ (lane & 15)) << 4;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 key = ld16(k_lane + t * (32 * kRowBytes) + (k_chunk ^ (i << 5)));
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, key), q[i], s[t], 0, 0, 0);
      }
    }
    if (masked) {
#pragma unroll
      for (int t = 0; t < kBlocks; ++t) {
        const uint32_t bits = (uint32_t)(allow >> (32 * t)) >> ((lane >> 5) * 4);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!(bits >> (8 * (r / 4) + r % 4) & 1)) s[t][r] = -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
    const LanePair p2 = pair_across32(as_u(top));
    top = fmaxf(as_f(p2.first), as_f(p2.second)) * scale;
    const bool move = top > ref + kMove;
    if (__ballot(move)) {
      const float to = move ? top - kBelow : ref;
      const float alpha = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
    }
    float sum[2] = {0.f, 0.f};
    half8_t w[kBlocks * 2], rest[kExact ? kBlocks * 2 : 1];
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], scale, -ref));
        sum[r & 1] += p;
        if constexpr (kExact) {
          const float scaled = p * kWeightScale;
          const _Float16 part = (_Float16)scaled;
          w[2 * t + r / 8][r % 8] = part;
          rest[2 * t + r / 8][r % 8] = (_Float16)(scaled - (float)part);
        } else {
          w[2 * t + r / 8][r % 8] = (_Float16)p;
        }
      }
    l += sum[0] + sum[1];
    // lane: token 4 h + (l % 16) / 4, channels 16 (l / 16 % 2) + 4 (l % 4) ..+3 of a block of 32
    const int quad = (lane >> 2) & 3;
    const char* v_lane = v + ((lane >> 5) * 4 + quad) * kRowBytes + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < kBlocks * 2; ++i)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const char* at = v_lane + i * (16 * kRowBytes) + ((d ^ quad) << 6);
        const short4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)at);
        const short4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(at + 8 * kRowBytes));
        const half8_t value =
            __builtin_bit_cast(half8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, w[i], acc[d], 0, 0, 0);
        if constexpr (kExact) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, rest[i], acc[d], 0, 0, 0);
      }
  }

  // The row's whole sum and what the accumulators have to be multiplied by.
  __device__ __forceinline__ float total() const {
    const LanePair s = pair_across32(as_u(l));
    return as_f(s.first) + as_f(s.second);
  }
  static constexpr float kUnscale = kExact ? 1.f / kWeightScale : 1.f;

  // Channels of the lane's accumulators, four at a time: f(channel, four values).
  template <class F>
  __device__ __forceinline__ void each4(float factor, int lane, F f) const {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        f(d * 32 + 2 * r + (lane >> 5) * 4,
          make_float4(acc[d][r] * factor, acc[d][r + 1] * factor, acc[d][r + 2] * factor, acc[d][r + 3] * factor));
  }
};

__device__ __forceinline__ void store4(void* out, int out_is_fp16, size_t idx, float4 v) {
  if (out_is_fp16) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    const h4 h = {(_Float16)v.x, (_Float16)v.y, (_Float16)v.z, (_Float16)v.w};
    *reinterpret_cast<h4*>(reinterpret_cast<_Float16*>(out) + idx) = h;
  } else {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + idx) = v;
  }
}

// Where the 16-byte chunk `slot` of a token's key (value) lies in its LDS tile.
__device__ __forceinline__ int k_place(int token, int slot) { return token * kRowBytes + ((slot ^ (token & 15)) << 4); }
__device__ __forceinline__ int v_place(int token, int slot) {
  return token * kRowBytes + ((slot ^ ((token & 3) << 2)) << 4);
}

#endif  // __HIPCC__

}  // namespace quest
