// Attention of many query rows over a paged cache: what prompts and trees of drafted tokens share.
//
// A KV head's rows are its sequence's new tokens times the query heads of its group, token by token: row r is
// head r % G of token r / G, so that whatever the group the keys are read once for all of them.
// Rows are cut into tiles of kRows.  A tile walks the tokens it attends to 64 at a time with an online softmax.
//
// The host knows no lengths, so every work-group works out the plan for itself, one sequence a lane: from the row tiles
// and the row tiles times token tiles of all of them comes the length of a split (`chunk` token tiles) with which
// the units are no more than the compute units take at once (or in the few rounds that the host chose), however ragged
// the batch; a prefix sum finds the work-group's own sequence.  That is if the host allows splits: it does not where as many sequences
// (times KV heads) as the compute units take work-groups at once may have one each, though a single one of them may be long (nodes in 63
// sequences of 2000 tokens and one of 100000, 8 heads: 1800 us, in two calls 97 + 85).
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
// Weights go to the product in fp16.  For fp32 outputs, and for all outputs of few rows, a weight is two fp16 numbers, 2^14 times its
// value rounded and what that leaves, 22 bits of it down to 2^-16 of the largest weight, below that to within 2^-39 of the largest (the
// smallest step of what is left; weights under 2^-39 are in the sum alone): error 4e-7, three times below fp32 products one after the other.
// For fp16 outputs of many rows one rounding of each weight, 2^-11 of it, which is what the
// output's own rounding costs (error against 64 bits, 2-norm: 2.6e-4, 1.3 times that of one rounding at the end, while 22 bits take
// 1.33 to 1.42 times as long, 32k tokens of 32 / 8 heads 12.0 ms and 8.6; of few rows they take 1.00 to 1.12 times); the base is
// put so that the largest logit's weight is 2^7 and moves when a weight would pass 2^15, so weights keep all bits down
// to 2^-21 of the largest and are not lost down to 2^-31.  Outputs are divided by the sum of the weights as rounded, so that a row that
// sees one value, or the same one everywhere, gets it back (32k tokens 8.35 -> 8.61 ms, error 2.75e-4 -> 2.64e-4); the log-sum-exp is of
// the weights before.
// Sums, maxima and accumulators are fp32.
#pragma once

#include <type_traits>

#include "quest_common.h"
#include "quest_decode_core.h"
#include "quest_e4m3.h"

namespace quest {

struct RowsArgs {
  const char* q;
  const char* k_pool;
  const char* v_pool;
  const float2* scales;     // pages of 8 bits
  const int32_t* cu;
  const int32_t* seq_lens;
  void* out;
  float* lse;
  float* part_acc;          // [units][kv heads][kRows][D]
  float* part_ml;           // [units][kv heads][kRows][2]: reference (logit before the scale), sum
  const char* k_new;        // trees: keys and values of the drafted nodes
  const char* v_new;
  const int64_t* mask;      // trees: [rows of cu][mask_words]
  int64_t q_stride, new_stride;   // bytes between tokens
  int batch, max_pages, page_shift, kv_heads, group;
  int mask_words, k_pages;
  int most_units;           // units of a KV head that the tokens are split into at most; 0: no splits
  int least_chunk;          // token tiles of a split, at least
  int out_is_fp16;
  uint32_t q_sign;          // exclusive-ored onto q: sign bits where the scale is negative
  float scale;              // |sm_scale| log2(e), not 0
  float below, limit;       // RowState's kBelow and kMove in logits before the scale
};

constexpr int kTileTokens = 64;
// Splits of the longest sequence, about (a chunk is a whole number of tiles: up to 95): joining more takes longer than they save (60k
// tokens of a head: 43 us, 30 with).
constexpr int kMostSplits = 64;

#if defined(__HIPCC__)

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// v of this lane and all before it.
template <int N, class T>
__device__ __forceinline__ T row_shr(T v) {  // of the lane N before, in the same row of 16; 0 where there is none
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x110 + N, 0xf, 0xf, false));
}
template <class T>
__device__ __forceinline__ T up_to_lane(T v, int lane) {
  v += row_shr<1>(v);
  v += row_shr<2>(v);
  v += row_shr<4>(v);
  v += row_shr<8>(v);
  T before = 0;
#pragma unroll
  for (int row = 1; row < 4; ++row) {
    const T end = __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), row * 16 - 1));
    if (lane >= row * 16) before += end;
  }
  return v + before;
}
// The largest v of the wave's lanes (none below 0).
__device__ __forceinline__ int largest_of_wave(int v) {
  v = max(v, row_shr<1>(v));
  v = max(v, row_shr<2>(v));
  v = max(v, row_shr<4>(v));
  v = max(v, row_shr<8>(v));
  int of_rows = 0;
#pragma unroll
  for (int row = 1; row <= 4; ++row) of_rows = max(of_rows, __builtin_amdgcn_readlane(v, row * 16 - 1));
  return of_rows;
}

// The plan of one sequence, and where its units start.  A unit is a split of a row tile.  Without splits and for trees
// sequence b's are in the order split * row_tiles + row tile, the last row tile first.  A prompt's row tiles have fewer splits
// the earlier they are: row tile j before the last and row tile j behind the first share `slots` places, about as
// many as they need together, in the order slot * pairs + j: by turns while both have splits, so that those of the same
// tokens run at the same time.  (With places for as many splits of each as the last one has, half of
// them had nothing to do; work-groups start in order, and those behind the idle ones started a round later.)
struct Sequence {
  int b, first, tokens, seq_len;   // first: its first packed row
  int length;                      // cached tokens that its page-table row has room for: nothing behind the row is read
  int row_tiles, slots, chunk;     // chunk: INT32_MAX without splits
  int before;                      // units (row tiles) of the sequences before
  int units_before;

  template <int kRows>
  __device__ __forceinline__ int splits_of(int row_tile, int group) const {   // of a prompt's row tile
    const int rows = tokens * group, limit = seq_len - tokens + (min((row_tile + 1) * kRows, rows) - 1) / group + 1;
    const int tiles = (max(min(limit, length), 0) + kTileTokens - 1) / kTileTokens;
    return (tiles + chunk - 1) / chunk;
  }
  template <bool kTree>
  __device__ __forceinline__ bool paired() const { return !kTree && chunk != INT32_MAX && row_tiles > 1; }
  template <bool kTree>
  __device__ __forceinline__ int places() const { return paired<kTree>() ? (row_tiles + 1) / 2 : row_tiles; }  // of a slot
};
// Finds the sequence of unit `want` (kByTile: of row tile `want`, counted over all sequences); false: there is none.
template <bool kTree, int kRows, bool kByTile>
__device__ __forceinline__ bool find_sequence(Sequence& s, const RowsArgs& a, const int32_t* __restrict__ cu,
                                              const int32_t* __restrict__ seq_lens, bool list, int want, int lane) {
  int first = 0, tokens = 0, seq_len = 0, length = 0, row_tiles = 0;
  int places = 0, tiles = 0, last = 0;   // token tiles, of a pair of row tiles at most and of the last one
  auto read = [&](int base) {
    const int i = min(base + lane, a.batch - 1);
    first = cu[i];
    tokens = cu[i + 1] - first;
    seq_len = seq_lens[i];
    length = min(max(seq_len, 0), a.max_pages << a.page_shift);
    row_tiles = places = base + lane < a.batch ? (tokens * a.group + kRows - 1) / kRows : 0;
    const int context = list ? min(a.k_pages, a.max_pages) << a.page_shift : length;
    last = tiles = (context + kTileTokens - 1) / kTileTokens + (kTree ? (tokens + kTileTokens - 1) / kTileTokens : 0);
    if (!kTree && row_tiles > 1 && a.most_units > 0) {   // the last tokens of row tiles j and row_tiles - 1 - j add up to this at most
      int64_t both = 2 * (int64_t)(seq_len - tokens) + (row_tiles + 1) * kRows / a.group + 2;
      if (length < seq_len || seq_len < tokens) both = 2 * (int64_t)length;   // (past the row, or before the first token)
      tiles = (int)((both + 2 * (kTileTokens - 1)) / kTileTokens);
      places = (row_tiles + 1) / 2;
    }
  };
  // Slots of a sequence that is cut every `chunk` tiles.
  auto slots_of = [&](int chunk) {
    const int most = (last + chunk - 1) / chunk;
    return !kTree && row_tiles > 1 ? min((tiles - 2) / chunk + 2, 2 * most) : most;
  };
  auto whole = [](auto v) { return __builtin_bit_cast(decltype(v), __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kWave - 1)); };
  s.chunk = INT32_MAX;
  if (a.most_units > 0) {
    float work = 0.f;
    int count = 0, longest = 0;   // longest: of those that have rows
    for (int base = 0; base < a.batch; base += kWave) {
      read(base);
      work += whole(up_to_lane((float)places * (float)tiles, lane));
      count += whole(up_to_lane(!kTree && row_tiles > 1 ? 2 * places : places, lane));
      longest = max(longest, largest_of_wave(row_tiles > 0 ? last : 0));
    }
    const int least = max(a.least_chunk, longest / kMostSplits);
    // The chunk: with this one the units are at most work / chunk + count, so no more than there is room for (a
    // hundred-thousandth covers the roundings) ..
    const float even = work / (float)max(a.most_units - count, 1) * 1.00001f;
    if (a.most_units > count && even < 4e7f) s.chunk = max(least, (int)even + 1);
    if (s.chunk != INT32_MAX && a.batch <= kWave) {
      // .. and that is more than needed, as a last split is half a chunk on average: the smallest with which they still
      // are, within 3 %.
      int low = max(least, (int)(work / (float)a.most_units)), high = s.chunk;   // high: few enough
      while (high - low > high >> 5) {
        const int chunk = (low + high) >> 1;
        if (whole(up_to_lane(places * slots_of(chunk), lane)) <= a.most_units)
          high = chunk;
        else
          low = chunk + 1;
      }
      s.chunk = high;
    }
  }
  int units_before = 0, tiles_before = 0;
  for (int base = 0; base < a.batch; base += kWave) {
    if (a.batch > kWave || a.most_units == 0) read(base);
    const int slots = s.chunk == INT32_MAX ? 1 : slots_of(s.chunk);
    const int units = s.chunk == INT32_MAX ? row_tiles : places * slots;
    const int u = up_to_lane(units, lane) + units_before;
    const int t = kByTile ? up_to_lane(row_tiles, lane) + tiles_before : 0;
    const unsigned long long behind = __ballot((kByTile ? t : u) > want);  // (lanes without a sequence repeat the sum)
    if (behind != 0) {
      const int at = __builtin_ctzll(behind);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
      s.b = base + at;
      s.first = of(first);
      s.tokens = of(tokens);
      s.seq_len = of(seq_len);
      s.length = of(length);
      s.row_tiles = of(row_tiles);
      s.slots = of(slots);
      s.units_before = of(u - units);
      s.before = kByTile ? of(t - row_tiles) : s.units_before;
      return true;
    }
    units_before = __builtin_amdgcn_readlane(u, kWave - 1);
    tiles_before = __builtin_amdgcn_readlane(t, kWave - 1);
  }
  return false;
}

// Where the 16-byte chunk `slot` of a token's 8-bit key or value lies in its LDS tile.
__device__ __forceinline__ int place8(int token, int slot) { return token * kRowBytes8 + ((slot ^ ((token >> 1) & 7)) << 4); }

// Attention state of a wave's 32 rows; lane l: row l % 32.  Weights are 2^(scale (s - base)), s the logit before the scale
// and base close below the largest one: the difference first, which is exact near it, so that logits of any size keep
// their order.  kShifted: the products that make the logits start at -base, which costs 16 registers and no instruction.
template <bool kExact, bool kShifted>
struct RowState {
  static constexpr float kBelow = kExact ? 0.f : 7.f;    // the base lies this far below the largest logit (log2)
  static constexpr float kMove = kExact ? 1.f : 15.f;    // and moves when a logit is this far above it
  half8_t q[8];        // channels 16 i + 8 h ..+7
  f32x16_t acc[4];     // [d / 32]: channels 8 (r / 4) + 4 h + r % 4
  f32x16_t start;      // kShifted: -base
  float base, limit;   // moves when s - base is above; -3e38 while no token has counted
  float l;             // this lane's share of the row's sum
  float met;           // the same of the weights as the values meet them (not kExact), which outputs are divided by

  // Asks for the row's query; what uses it comes after ready().
  __device__ __forceinline__ void init(const char* row, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(half8_t, ld16(row + i * 32 + (lane >> 5) * 16));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) start[r] = 0.f;
    base = 0.f;
    limit = -3e38f;
    l = 0.f;
    met = 0.f;
  }
  __device__ __forceinline__ void ready(uint32_t sign) {
    if (sign != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint4 v = __builtin_bit_cast(uint4, q[i]);
        v.x ^= sign, v.y ^= sign, v.z ^= sign, v.w ^= sign;
        q[i] = __builtin_bit_cast(half8_t, v);
      }
    }
  }

  // Logits (kShifted: minus the base) of 32 kBlocks tokens that lie in LDS.
  template <int kBlocks>
  __device__ __forceinline__ void logits(f32x16_t (&s)[kBlocks], const char* k, int lane) const {
    const char* k_lane = k + (lane & 31) * kRowBytes;
    const int k_chunk = ((lane >> 5) ^ (lane & 15)) << 4;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      if constexpr (kShifted) {
        s[t] = start;
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
      }
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
  __device__ __forceinline__ void weigh(Weights<kBlocks>& p, f32x16_t (&s)[kBlocks], const RowsArgs& a) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
    const LanePair p2 = pair_across32(as_u(top));
    top = fmaxf(as_f(p2.first), as_f(p2.second));
    if (!kShifted) top -= base;
    const bool move = top > limit;
    if (__ballot(move)) {
      const float by = move ? top - a.below : 0.f;
      const float alpha = limit < -1e38f ? 0.f : __builtin_amdgcn_exp2f(-by * a.scale);
      base += by;
      limit = move ? a.limit : limit;
      l *= alpha;
      met *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
      if constexpr (kShifted) {
#pragma unroll
        for (int t = 0; t < kBlocks; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] -= by;
#pragma unroll
        for (int r = 0; r < 16; ++r) start[r] = -base;
      }
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_amdgcn_exp2f((kShifted ? s[t][r] : s[t][r] - base) * a.scale);
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
    if constexpr (!kExact) {
#pragma unroll
      for (int i = 0; i < 2 * kBlocks; ++i)
#pragma unroll
        for (int r = 0; r < 8; r += 2)
          met = __builtin_amdgcn_fdot2(half2_t{p.w[i][r], p.w[i][r + 1]}, half2_t{(_Float16)1, (_Float16)1}, met, false);
    }
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
  __device__ __forceinline__ void fold(const char* k, const char* v, const RowsArgs& a, bool masked, uint64_t allow, int lane) {
    f32x16_t s[kBlocks];
    logits(s, k, lane);
    if (masked) hide(s, allow, lane);
    Weights<kBlocks> p;
    weigh(p, s, a);
    add(p, v, lane);
  }

  // The same for 32 tokens that lie in LDS as 8-bit numbers, rows of 128 bytes (place8).  Row m = 8 i + 4 h + j of the first product is
  // token 16 (i / 2) + 8 h + 4 (i % 2) + j, so that a lane's weights are of tokens 8 h ..+7 and 16 + 8 h ..+7: eight of one page each,
  // whose values (turned by the LDS read, eight tokens of a channel) have one scale.
  __device__ __forceinline__ static int token8(int row) { return (row & 16) | ((row & 4) << 1) | ((row & 8) >> 1) | (row & 3); }
  __device__ __forceinline__ void logits8(f32x16_t (&s)[1], const char* k, float scale, int lane) const {
    const int token = token8(lane & 31);
    const char* k_lane = k + (lane >> 5) * 8;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint2 codes = *reinterpret_cast<const uint2*>(k_lane + place8(token, i));
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, halves_of(codes, scale)), q[i], s[0], 0, 0, 0);
    }
  }
  __device__ __forceinline__ static void hide8(f32x16_t (&s)[1], uint32_t allow, int lane) {
    const uint32_t bits = allow >> ((lane >> 5) * 8);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!(bits >> (16 * (r / 8) + r % 8) & 1)) s[0][r] = -INFINITY;
  }
  __device__ __forceinline__ void add8(const Weights<1>& p, const char* v, const float (&scale)[2], int lane) {
    typedef int int2_t __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) int2_t lds_int2_t;
    const int token = (lane >> 5) * 8 + ((lane & 15) >> 1), slot = (lane >> 4) & 1;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int2_t codes =
            __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2_t*)(v + place8(16 * i + token, 2 * d + slot) + (lane & 1) * 8));
        const half8_t value =
            __builtin_bit_cast(half8_t, halves_of(make_uint2((uint32_t)codes.x, (uint32_t)codes.y), scale[i]));
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, p.w[i], acc[d], 0, 0, 0);
        if constexpr (kExact) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, p.rest[i], acc[d], 0, 0, 0);
      }
  }

  // The row's whole sum, and that of the weights that its values met.
  __device__ __forceinline__ float total() const { return both_halves(l); }
  __device__ __forceinline__ float total_met() const { return both_halves(kExact ? l : met); }
  __device__ __forceinline__ static float both_halves(float v) {
    const LanePair s = pair_across32(as_u(v));
    return as_f(s.first) + as_f(s.second);
  }
  // log sum exp of a row, of its base and sum.
  __device__ __forceinline__ static float lse(float base, float total, float scale) {
    return total == 0.f ? -INFINITY : __builtin_fmaf(base, scale, __builtin_amdgcn_logf(total)) * kLn2;  // (NaN stays)
  }
  static constexpr float kUnscale = kExact ? 1.f / kWeightScale : 1.f;

  // Channels 32 kFrom to 32 kTo of the lane's accumulators, four at a time: f(channel, four values).
  template <int kFrom = 0, int kTo = 4, class F>
  __device__ __forceinline__ void each4(float factor, int lane, F f) const {
#pragma unroll
    for (int d = kFrom; d < kTo; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        f(d * 32 + 2 * r + (lane >> 5) * 4,
          make_float4(acc[d][r] * factor, acc[d][r + 1] * factor, acc[d][r + 2] * factor, acc[d][r + 3] * factor));
  }
};

// An fp16 output.  It is a mean of fp16 values: what the roundings of sums over a long context (2^-11 at most) carry past
// the largest fp16 is put back.
__device__ __forceinline__ _Float16 half_of(float x) {
  return (_Float16)(fabsf(x) < 65552.f ? __builtin_amdgcn_fmed3f(x, -65504.f, 65504.f) : x);
}
__device__ __forceinline__ void store_halves(void* to, float4 v) {
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<h4*>(to) = h4{half_of(v.x), half_of(v.y), half_of(v.z), half_of(v.w)};
}

// Where the 16-byte chunk `slot` of a token's key (value) lies in its LDS tile.
__device__ __forceinline__ int k_place(int token, int slot) { return token * kRowBytes + ((slot ^ (token & 15)) << 4); }
__device__ __forceinline__ int v_place(int token, int slot) {
  return token * kRowBytes + ((slot ^ ((token & 3) << 2)) << 4);
}

// 16 bytes a lane from memory to LDS at `to` + 16 lane, without registers in between: from a wave's address and a
// lane's offset, or a lane's address.  The compiler does not count these: dma_arrived<n> waits until at
// most the last n (and what was loaded since) are under way.  M0 is the instruction's LDS base; it is an operand here, so that the
// compiler writes it and knows that what it held is gone.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}
__device__ __forceinline__ void dma16(uint32_t to, const char* base, uint32_t offset) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               ::"{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base)
               : "memory");
}
__device__ __forceinline__ void dma16(uint32_t to, const char* from) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               ::"{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
               : "memory");
}
template <int N>
__device__ __forceinline__ void dma_arrived() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
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
    seq_len = s.length;
    seq_pages = (seq_len + (1 << page_shift) - 1) >> page_shift;
    limit = kTree ? seq_len : min(last + 1, seq_len);
    const int places = pages != nullptr ? listed << page_shift : max(limit, 0);
    context = (places + kTileTokens - 1) & ~(kTileTokens - 1);
    first = s.first;
    nodes = kTree ? s.tokens : 0;
    tiles = (context + nodes + kTileTokens - 1) / kTileTokens;
  }
};

// A wave's walk over the stream in steps of kPlaces (32 or 64) places, step i at place start + i stride.  What page a place
// is in is looked up for many steps at a time, one page (or part of one, where a page is longer than a step) a lane:
// lane e of the first step's, then the next step's, ..  The lookups' latency, twice a memory access with a list, is
// then paid once in 16 to 64 steps, and nothing waits for a lookup behind the keys and values under way.
// k8: pages of 8 bits, whose numbers become fp16 numbers on the way from registers to LDS (many row tiles) or from LDS to the products (few);
// drafted nodes are fp16 as ever.
template <bool kTree, int kPlaces, bool k8 = false>
struct Walk {
  int start, stride;
  int shift;            // log2 of the places a lane looks up: a page, at most a step
  int per_step_log2;    // lanes of a step
  int first_step;       // step of lane 0
  int phys, left;       // this lane's page, and how many of its places (from its first on) hold a token
  float2 scale;         // k8: of its keys and values
  static constexpr int kLog2 = kPlaces == 64 ? 6 : 5;

  __device__ __forceinline__ void init(const Stream<kTree>& s, int start_, int stride_) {
    start = start_;
    stride = stride_;
    shift = min(s.page_shift, kLog2);
    per_step_log2 = kLog2 - shift;
    first_step = 0;
  }
  __device__ __forceinline__ bool knows(int step) const { return (step - first_step) << per_step_log2 < kWave; }
  __device__ __forceinline__ void find(const Stream<kTree>& s, int step, int lane) {
    first_step = step;
    const int at = start + (step + (lane >> per_step_log2)) * stride + ((lane & ((1 << per_step_log2) - 1)) << shift);
    phys = 0;
    left = 0;
    if (kTree && at >= s.context) {
      left = s.nodes - (at - s.context);
    } else if (s.pages != nullptr) {
      const int entry = at >> s.page_shift;
      const int page = entry < s.listed ? s.pages[entry] : -1;
      if (page >= 0 && page < s.seq_pages) {
        phys = s.table[page];
        left = s.seq_len - (page << s.page_shift) - (at & ((1 << s.page_shift) - 1));
      }
    } else if (at < s.limit) {
      phys = s.table[at >> s.page_shift];
      left = s.limit - at;
    }
  }
  __device__ __forceinline__ void find8(const RowsArgs& a, const Stream<kTree>& s, int hk, int step, int lane) {
    find(s, step, lane);
    const int at = start + (step + (lane >> per_step_log2)) * stride + ((lane & ((1 << per_step_log2) - 1)) << shift);
    scale = make_float2(1.f, 1.f);   // (a page without tokens may have any)
    if (left > 0 && (!kTree || at < s.context)) scale = a.scales[(size_t)phys * a.kv_heads + hk];
  }
  // Key and value of the step's place `eight` + lane / 8 (`eight`: a multiple of 8): channels 16 (lane % 8) ..+15; zeros where there
  // is no token.  kOnce: past the caches (the large kernel, whose row tiles read the same tokens at about the same time: 32k of 32 / 8
  // heads through them 8.8 ms, past them 9.0).
  template <bool kOnce>
  __device__ __forceinline__ void load8(const RowsArgs& a, const Stream<kTree>& s, int hk, int step, int eight, int lane,
                                        uint4& key, uint4& value) const {
    const int from = ((step - first_step) << per_step_log2) + (eight >> shift);
    const int page = __builtin_amdgcn_readlane(phys, from);
    const int at = (start + step * stride + eight) & ((1 << s.page_shift) - 1);
    const uint32_t block = ((uint32_t)(page * a.kv_heads + hk) << (s.page_shift - 3)) + (at >> 3);
    const int tokens = min(max(__builtin_amdgcn_readlane(left, from) - (eight & ((1 << shift) - 1)), 0), 8);
    // (the same in all lanes, which the compiler does not see)
    const uint32_t of_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)block);
    const int bytes = __builtin_amdgcn_readfirstlane(tokens * kRowBytes8);
    key = row16<kOnce>(rows_at(a.k_pool, of_wave, bytes), lane);
    value = row16<kOnce>(rows_at(a.v_pool, of_wave, bytes), lane);
  }
  // What load8 brought, into LDS (k, v: the tile), as it is or as fp16 numbers.  `of`: the scales as they were then.
  struct Scales8 {
    float2 scale;
    int first_step;
  };
  __device__ __forceinline__ Scales8 scales8() const { return {scale, first_step}; }
  __device__ __forceinline__ static void put_codes(int eight, int lane, uint4 key, uint4 value, char* k, char* v) {
    const int at = place8(eight + (lane >> 3), lane & 7);
    st16(k + at, key);
    st16(v + at, value);
  }
  // The scale (`of`: the keys' or the values') of the step's place `eight`, a lane's own.
  __device__ __forceinline__ float scale_of_lane(float of, int step, int eight) const {
    const int from = ((step - first_step) << per_step_log2) + (eight >> shift);
    return as_f((uint32_t)__builtin_amdgcn_ds_bpermute(from * 4, (int)as_u(of)));
  }
  __device__ __forceinline__ void put8(const Scales8& of, int step, int eight, int lane, uint4 key, uint4 value, char* k, char* v) const {
    const int from = ((step - of.first_step) << per_step_log2) + (eight >> shift);
    const float k_scale = from_lane(of.scale.x, from), v_scale = from_lane(of.scale.y, from);
    const int token = eight + (lane >> 3), slot = (lane & 7) * 2;
    // (Eight lanes write at a time, to 32 banks: chunks that differ modulo 8.  32k tokens of 32 / 8 heads 8.50 -> 8.43 ms.)
    const int odd = (lane >> 2) & 1;
    auto half = [odd](uint4 x, bool second) { return odd != second ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y); };
    st16(k + k_place(token, slot + odd), halves_of(half(key, false), k_scale));
    st16(k + k_place(token, slot + 1 - odd), halves_of(half(key, true), k_scale));
    st16(v + v_place(token, slot + odd), halves_of(half(value, false), v_scale));
    st16(v + v_place(token, slot + 1 - odd), halves_of(half(value, true), v_scale));
  }
  // 16 bytes of the key and of the value of the step's place `four` + lane / 16 (`four`: a multiple of 4).  Returns whether
  // there is a token; if not, the value has to be zeroed when it has arrived: stale slots may hold anything, and
  // zero weights times that need not be zero.
  __device__ __forceinline__ bool load(const RowsArgs& a, const Stream<kTree>& s, int hk, int step, int four, int lane,
                                       uint4& key, uint4& value) const {
    const int sub = lane >> 4, at = start + step * stride + four;
    const int from = ((step - first_step) << per_step_log2) + (four >> shift);
    if (kTree && at >= s.context) {
      const int64_t off = (int64_t)(s.first + min(at - s.context + sub, s.nodes - 1)) * a.new_stride +
                          (int64_t)hk * kRowBytes + (lane & 15) * 16;
      key = ld16(a.k_new + off);
      value = ld16(a.v_new + off);
    } else {
      const int page = __builtin_amdgcn_readlane(phys, from);
      const int64_t row = (((int64_t)page * a.kv_heads + hk) << s.page_shift) + (at & ((1 << s.page_shift) - 1));
      key = ld16(a.k_pool + row * kRowBytes + lane * 16);   // four rows of 256 bytes
      value = ld16(a.v_pool + row * kRowBytes + lane * 16);
    }
    return (four & ((1 << shift) - 1)) + sub < __builtin_amdgcn_readlane(left, from);
  }
  // The same straight into LDS, where k_place and v_place would put it (`k_lds`, `v_lds`: the tile's addresses): a lane
  // fetches the chunk that belongs at its own place.  Rows that are not there get a row that is (the first of the
  // sequence): any finite value will do under a weight of zero.  To be waited for with dma_arrived.
  __device__ __forceinline__ void fetch(const RowsArgs& a, const Stream<kTree>& s, int hk, int step, int four, int lane,
                                        uint32_t k_lds, uint32_t v_lds) const {
    const int sub = lane >> 4, at = start + step * stride + four;
    const int from = ((step - first_step) << per_step_log2) + (four >> shift);
    const int there = __builtin_amdgcn_readlane(left, from) - (four & ((1 << shift) - 1));
    const uint32_t k_chunk = ((lane & 15) ^ ((four + sub) & 15)) << 4, v_chunk = ((lane & 15) ^ (sub << 2)) << 4;
    k_lds += four * kRowBytes;
    v_lds += four * kRowBytes;
    const bool drafts = kTree && at >= s.context;
    const int page = __builtin_amdgcn_readlane(phys, from);
    const int64_t row = (((int64_t)page * a.kv_heads + hk) << s.page_shift) + (at & ((1 << s.page_shift) - 1));
    if (!drafts && there >= 4) {
      dma16(k_lds, a.k_pool + row * kRowBytes, sub * kRowBytes + k_chunk);
      dma16(v_lds, a.v_pool + row * kRowBytes, sub * kRowBytes + v_chunk);
      return;
    }
    const char *k = a.k_pool, *v = a.v_pool;
    int64_t off = (row + sub) * kRowBytes;
    if (drafts || (kTree && sub >= there)) {
      k = a.k_new;
      v = a.v_new;
      const int node = drafts ? min(at - s.context + sub, s.nodes - 1) : 0;
      off = (int64_t)(s.first + node) * a.new_stride + (int64_t)hk * kRowBytes;
    } else if (sub >= there) {
      off = (((int64_t)s.table[0] * a.kv_heads + hk) << s.page_shift) * kRowBytes;
    }
    dma16(k_lds, k + off + k_chunk);
    dma16(v_lds, v + off + v_chunk);
  }
  // Which of the step's places hold a token.
  __device__ __forceinline__ uint64_t held(int step, int lane) const {
    const int place = lane & (kPlaces - 1);
    const int from = ((step - first_step) << per_step_log2) + (place >> shift);
    const uint64_t all = __ballot((place & ((1 << shift) - 1)) < __builtin_amdgcn_ds_bpermute(from * 4, left));
    return kPlaces == 64 ? all : all & 0xffffffffull;
  }
  // Which of them a row attends to: those up to its position (prompts), all cached ones or those of its mask (trees).
  __device__ __forceinline__ uint64_t allow(const Stream<kTree>& s, uint64_t held, int step, int position,
                                            const int64_t* __restrict__ mask, int mask_words) const {
    const int at = start + step * stride;
    if (!kTree) return first_bits(min(position + 1, s.limit) - at);
    if (at < s.context) return held;
    const int node = at - s.context;
    return (node >> 6) < mask_words ? ((uint64_t)mask[node >> 6] >> (node & 63)) & held : 0;
  }
  // Whether all rows from `position` on attend to all of them.
  __device__ __forceinline__ bool whole(const Stream<kTree>& s, uint64_t held, int step, int position) const {
    const int at = start + step * stride;
    return kTree ? at < s.context && held == (kPlaces == 64 ? ~0ull : 0xffffffffull) : at + kPlaces <= min(position + 1, s.limit);
  }
};

#endif  // __HIPCC__

}  // namespace quest
