// Attention of many query rows over a paged cache: what prompts and trees of drafted tokens share.
//
// A KV head's rows are its sequence's new tokens times the query heads of its group, token by token: row r is
// head r % G of token r / G, so that whatever the group the keys are read once for all of them.
// Rows are cut into tiles of kRows.  A tile walks the tokens it attends to 64 at a time with an online softmax.
//
// The host knows no lengths, so every work-group works out the plan for itself: one sequence a lane, the row
// tiles times token tiles of all of them give the length of a split (`chunk` token tiles) with which about
// 2^target_log2 work-groups come out, however ragged the batch; a prefix sum finds the work-group's own sequence.
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
  float* part_acc;          // [units][kv heads][kRows][D]
  float* part_ml;           // [units][kv heads][kRows][2]: reference exponent, sum
  const char* k_new;        // trees: keys and values of the drafted nodes
  const char* v_new;
  const int64_t* mask;      // trees: [rows of cu][mask_words]
  int64_t q_stride, new_stride;   // bytes between tokens
  int batch, max_pages, page_shift, kv_heads, group;
  int mask_words, k_pages;
  int target_log2;          // work-groups to come out, about; below 0: no splits
  int least_chunk;          // token tiles of a split, at least
  int out_is_fp16;
  uint32_t q_sign;          // exclusive-ored onto q: sign bits where the scale is negative
  float scale_log2;         // |sm_scale| log2(e), not 0
};

constexpr int kTileTokens = 64;

#if defined(__HIPCC__)

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// The plan of one sequence, and where its units start.  A unit is a split of a row tile; sequence b's are in the order
// split * row_tiles + row tile.
struct Sequence {
  int b, first, tokens, seq_len;   // first: its first packed row
  int row_tiles, splits, chunk;
  int before;                      // units (row tiles) of the sequences before
  int units_before;
};
// Finds the sequence of unit `want` (kByTile: of row tile `want`, counted over all sequences); false: there is none.
template <bool kTree, int kRows, bool kByTile>
__device__ __forceinline__ bool find_sequence(Sequence& s, const RowsArgs& a, const int32_t* __restrict__ cu,
                                              const int32_t* __restrict__ seq_lens, bool list, int want, int lane) {
  int first = 0, tokens = 0, seq_len = 0, row_tiles = 0, tiles = 0;
  auto read = [&](int base) {
    const int i = min(base + lane, a.batch - 1);
    first = cu[i];
    tokens = cu[i + 1] - first;
    seq_len = seq_lens[i];
    row_tiles = base + lane < a.batch ? (tokens * a.group + kRows - 1) / kRows : 0;
    const int context = list ? min(a.k_pages, a.max_pages) << a.page_shift : seq_len;
    tiles = (context + kTileTokens - 1) / kTileTokens + (kTree ? (tokens + kTileTokens - 1) / kTileTokens : 0);
  };
  const int lanes = min(a.batch, kWave);  // sums over as many
  int64_t all = 0;
  for (int base = 0; base < a.batch; base += kWave) {
    read(base);
    all += (int64_t)row_tiles * tiles;
  }
  for (int d = 1; d < lanes; d <<= 1) all += __shfl_xor(all, d);
  all = ((int64_t)__builtin_amdgcn_readfirstlane((int)(all >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)all)) *
        a.kv_heads;
  const int64_t even = (all + (1ll << max(a.target_log2, 0)) - 1) >> max(a.target_log2, 0);
  s.chunk = a.target_log2 < 0 || even > INT32_MAX ? INT32_MAX : max(a.least_chunk, (int)even);
  int units_before = 0, tiles_before = 0;
  for (int base = 0; base < a.batch; base += kWave) {
    if (a.batch > kWave) read(base);
    const int splits = tiles / s.chunk + (tiles % s.chunk != 0);
    const int units = row_tiles * splits;
    int u = units, t = row_tiles;   // inclusive sums
    for (int d = 1; d < lanes; d <<= 1) {
      const int uu = __shfl_up(u, d), tt = __shfl_up(t, d);
      if (lane >= d) u += uu, t += tt;
    }
    u += units_before;
    t += tiles_before;
    const unsigned long long behind = __ballot((kByTile ? t : u) > want);  // (lanes without a sequence repeat the sum)
    if (behind != 0) {
      const int at = __builtin_ctzll(behind);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
      s.b = base + at;
      s.first = of(first);
      s.tokens = of(tokens);
      s.seq_len = of(seq_len);
      s.row_tiles = of(row_tiles);
      s.splits = of(splits);
      s.units_before = of(u - units);
      s.before = kByTile ? of(t - row_tiles) : s.units_before;
      return true;
    }
    units_before = __builtin_amdgcn_readlane(u, lanes - 1);
    tiles_before = __builtin_amdgcn_readlane(t, lanes - 1);
  }
  return false;
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

  // Logits of 32 kBlocks tokens that lie in LDS.
  template <int kBlocks>
  __device__ __forceinline__ void logits(f32x16_t (&s)[kBlocks], const char* k, int lane) const {
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
  }
  // Only the tokens of `allow` (bit t: token t; a lane's own) count.
  template <int kBlocks>
  __device__ __forceinline__ static void hide(f32x16_t (&s)[kBlocks], uint64_t allow, int lane) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      const uint32_t bits = (uint32_t)(allow >> (32 * t)) >> ((lane >> 5) * 4);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(bits >> (8 * (r / 4) + r % 4) & 1)) s[t][r] = -INFINITY;
    }
  }
  // The weights of 32 kBlocks tokens, as second operands of the products with their values.
  template <int kBlocks>
  struct Weights {
    half8_t w[kBlocks * 2], rest[kExact ? kBlocks * 2 : 1];
  };
  template <int kBlocks>
  __device__ __forceinline__ void weigh(Weights<kBlocks>& p, const f32x16_t (&s)[kBlocks], float scale) {
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
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], scale, -ref));
        sum[r & 1] += x;
        if constexpr (kExact) {
          const float scaled = x * kWeightScale;
          const _Float16 part = (_Float16)scaled;
          p.w[2 * t + r / 8][r % 8] = part;
          p.rest[2 * t + r / 8][r % 8] = (_Float16)(scaled - (float)part);
        } else {
          p.w[2 * t + r / 8][r % 8] = (_Float16)x;
        }
      }
    l += sum[0] + sum[1];
  }
  // Add the weighted values, which lie in LDS.
  template <int kBlocks>
  __device__ __forceinline__ void add(const Weights<kBlocks>& p, const char* v, int lane) {
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
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, p.w[i], acc[d], 0, 0, 0);
        if constexpr (kExact) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, p.rest[i], acc[d], 0, 0, 0);
      }
  }
  // All of it for a tile.
  template <int kBlocks>
  __device__ __forceinline__ void fold(const char* k, const char* v, float scale, bool masked, uint64_t allow, int lane) {
    f32x16_t s[kBlocks];
    logits(s, k, lane);
    if (masked) hide(s, allow, lane);
    Weights<kBlocks> p;
    weigh(p, s, scale);
    add(p, v, lane);
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

// The first n of 64 bits.
__device__ __forceinline__ uint64_t first_bits(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

// The stream of tokens that a row tile of sequence b and KV head hk attends to.  Stream places 0, 1, .. are the
// cached tokens in order, or those of the listed pages; (trees) from the next multiple of 64 on come the drafted nodes.
// Four places from a multiple of 4 on lie in one page.
template <bool kTree>
struct Stream {
  const int32_t* table;   // the sequence's page-table row
  const int32_t* pages;   // its list, or null
  int seq_len, seq_pages, listed, page_shift;
  int limit;              // cached tokens (without a list): nothing behind them is looked at
  int context;            // places before the drafted nodes
  int first, nodes;       // the drafted nodes' first packed row, and how many
  int tiles;              // of 64 places

  // `last`: the last position that a row of the tile attends to (prompts).
  __device__ __forceinline__ void init(const RowsArgs& a, const Sequence& s, int hk, int last,
                                       const int32_t* __restrict__ page_table, const int32_t* __restrict__ topk) {
    table = page_table + (size_t)s.b * a.max_pages;
    pages = kTree && topk != nullptr ? topk + ((size_t)s.b * a.kv_heads + hk) * a.k_pages : nullptr;
    listed = min(a.k_pages, a.max_pages);
    page_shift = a.page_shift;
    seq_len = s.seq_len;
    seq_pages = (seq_len + (1 << page_shift) - 1) >> page_shift;
    limit = kTree ? seq_len : last + 1;
    const int places = pages != nullptr ? listed << page_shift : max(limit, 0);
    context = (places + kTileTokens - 1) & ~(kTileTokens - 1);
    first = s.first;
    nodes = kTree ? s.tokens : 0;
    tiles = (context + nodes + kTileTokens - 1) / kTileTokens;
  }
  // What a lane knows of the four places from its `at` on: their physical page, and how many of them hold a token
  // (any number).
  struct Four {
    int phys, count;
  };
  __device__ __forceinline__ Four find(int at) const {
    if (kTree && at >= context) return {0, nodes - (at - context)};
    if (pages != nullptr) {
      const int entry = at >> page_shift;
      const int page = entry < listed ? pages[entry] : -1;
      if (page < 0 || page >= seq_pages) return {0, 0};
      return {table[page], seq_len - (page << page_shift) - (at & ((1 << page_shift) - 1))};
    }
    return {table[min(at, limit - 1) >> page_shift], limit - at};
  }
  // 16 bytes of the key and of the value of place at + lane / 16, of the four that lane `from` has looked up.  Returns
  // whether there is a token; if not, the value has to be zeroed when it has arrived: stale slots may hold anything, and
  // zero weights times that need not be zero.
  __device__ __forceinline__ bool load(const RowsArgs& a, int hk, int at, Four f, int from, int lane, uint4& key,
                                       uint4& value) const {
    const int sub = lane >> 4;
    if (kTree && at >= context) {
      const int64_t off = (int64_t)(first + min(at - context + sub, nodes - 1)) * a.new_stride + (int64_t)hk * kRowBytes +
                          (lane & 15) * 16;
      key = ld16(a.k_new + off);
      value = ld16(a.v_new + off);
    } else {
      const int phys = __builtin_amdgcn_readlane(f.phys, from);
      const int64_t row = (((int64_t)phys * a.kv_heads + hk) << page_shift) + (at & ((1 << page_shift) - 1));
      key = ld16(a.k_pool + row * kRowBytes + lane * 16);   // four rows of 256 bytes
      value = ld16(a.v_pool + row * kRowBytes + lane * 16);
    }
    return sub < __builtin_amdgcn_readlane(f.count, from);
  }
  // Which of 64 places hold a token, lane g having looked up the g-th four of them.
  __device__ __forceinline__ uint64_t held(Four f, int lane) const {
    return __ballot((lane & 3) < __builtin_amdgcn_ds_bpermute(lane & ~3, f.count));
  }
  // Which of the 64 places from p0 (a multiple of 64) on a row attends to, of the `held` ones: those up to its
  // position (prompts), all cached ones or those of its mask (trees).
  __device__ __forceinline__ uint64_t allow(uint64_t held, int p0, int position, const int64_t* __restrict__ mask,
                                            int mask_words) const {
    if (!kTree) return first_bits(position + 1 - p0);
    if (p0 < context) return held;
    const int word = (p0 - context) / 64;
    return word < mask_words ? (uint64_t)mask[word] & held : 0;
  }
  // Whether all rows from `position` on attend to all of those places.
  __device__ __forceinline__ bool whole(uint64_t held, int p0, int position) const {
    return kTree ? p0 < context && held == ~0ull : p0 + kTileTokens - 1 <= position;
  }
};

#endif  // __HIPCC__

}  // namespace quest
