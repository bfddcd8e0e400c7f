// Attention of one query a sequence over pages of 8 bits: listed pages, or all.
//
// Bound by memory: a token's key and value of a head are 256 bytes, read once.  The tokens of a sequence are cut into tiles of
// 64 (128 where query heads share a KV head), a quarter for each of a work-group's four waves; a lane looks up the page of eight tokens,
// ahead of the keys and values, which are on their way to a wave 16 KiB at a time, and go on across the lookups.
//
// The host knows no lengths: the tiles of all sequences are one line that is cut into equal shares, a work-group each, however ragged
// the batch.  A share that ends inside a sequence leaves a partial result; the share of a (sequence, KV head) that arrives last joins
// them (quest_team.h).
//
// One query head per KV head: the vector unit.  A lane has 16 channels of every eighth token; products of pairs in fp16, which e4m3
// numbers times their scale are exactly, summed in fp32.  Weights are relative to a base that moves when a logit passes it by
// more than 8 (log2), so that sums are scaled again a few times and not at every token.
// Two to eight query heads per KV head: GroupState (quest_decode_core.h) on the matrix cores, its keys and values made fp16 numbers
// on the way.
#include <algorithm>

#include "quest_common.h"
#include "quest_decode_core.h"
#include "quest_e4m3.h"
#include "quest_rows_core.h"
#include "quest_team.h"

namespace quest {

namespace {

constexpr int kWaves = 4;
constexpr int kMostParts = 64;           // shares of a sequence, about

struct DecodeArgs : AttnArgs {
  const float2* scales;
  const int32_t* topk;
  int k_pages, listed;    // entries of a list, and how many of them count
  int shares;             // of the line of all sequences' tiles; 0: one work-group a sequence
  int loose;              // more than a share for each compute unit
  int count, per_die;     // shares or sequences, and (share, column) pairs of a die (0: every eighth sequence's)
};

// The tiles of all sequences, one after the other, are one line that is cut into shares of `length` tiles.  A sequence has a tile at
// least.  A list is taken to have as many entries as its sequence has pages at most (more only if it names a page twice: the last
// share sees to those).
// A share that ends one sequence and begins the next does two lookups and leaves two results, which takes longer than a few
// tiles: where shares up to kMore tiles longer (more than one share a compute unit: up to six tiles or a third) are enough for every
// sequence to begin a share of its own, the line has gaps and they do (up to 64 sequences; five of 831 to 1066 tokens by 8 KV heads 11.5
// -> 8.9 us, of 16 / 8 heads 13.3 -> 10.3, 12 of 525 to 2763 of 32 / 8 heads 19.2 -> 15.6, four of 16k 32.0 -> 28.8).
struct Line {
  static constexpr int kMore = 3;
  int length;
  int b, seq_len, first, tiles;   // the sequence that the share begins in: its first tile on the line, and how many it has
  int span;                       // its tiles with the gap behind them

  template <int kTile>
  __device__ __forceinline__ static int tiles_of(const DecodeArgs& a, int seq_len) {
    int tokens = min(max(seq_len, 0), a.max_pages << a.page_shift);
    if (a.topk != nullptr) tokens = min((tokens + (1 << a.page_shift) - 1) >> a.page_shift, a.listed) << a.page_shift;
    return max((tokens + kTile - 1) / kTile, 1);
  }
  template <int kTile>
  __device__ __forceinline__ void at(const DecodeArgs& a, int sequence) {
    b = sequence;
    seq_len = a.seq_lens[b];
    tiles = span = tiles_of<kTile>(a, seq_len);
  }
  // Where share `share` begins; false: behind the line's end.
  template <int kTile>
  __device__ __forceinline__ bool find(const DecodeArgs& a, int share, int lane) {
    if (a.shares == 0) {
      if (share >= a.batch) return false;
      length = INT32_MAX;
      first = 0;
      at<kTile>(a, share);
      return true;
    }
    if (a.batch == 1) {
      at<kTile>(a, 0);
      first = 0;
      length = share_length(a, tiles, tiles);
      return (int64_t)share * length < tiles;
    }
    int mine = 0, total = 0, longest = 0;
    auto read = [&](int base) {
      seq_len = a.seq_lens[min(base + lane, a.batch - 1)];
      mine = base + lane < a.batch ? tiles_of<kTile>(a, seq_len) : 0;
    };
    for (int base = 0; base < a.batch; base += kWave) {
      read(base);
      total += __builtin_amdgcn_readlane(up_to_lane(mine, lane), kWave - 1);
      longest = max(longest, largest_of_wave(mine));
    }
    length = share_length(a, total, longest);
    int spans = mine;
    if (a.batch <= kWave) {
      const int step = a.loose ? max(length / (3 * kMore), 2) : 1;
      int longer = 0;
      if (a.batch <= 16) {   // lane 16 j + b: shares that sequence b takes if they are j steps longer
        const int tiles_here = __builtin_amdgcn_ds_bpermute((lane & 15) * 4, mine), at = length + (lane >> 4) * step;
        const float needed = row16_sum((float)((tiles_here + at - 1) / at));
        const unsigned long long enough = __ballot(needed <= (float)a.shares && (lane >> 4) <= kMore);
        if (enough != 0) longer = length + (__builtin_ctzll(enough) >> 4) * step;
      } else {
        for (int j = 0; j <= kMore && longer == 0; ++j) {
          const int at = length + j * step;
          if (__builtin_amdgcn_readlane(up_to_lane((mine + at - 1) / at, lane), kWave - 1) <= a.shares) longer = at;
        }
      }
      if (longer != 0) {
        length = longer;
        spans = (mine + length - 1) / length * length;
        total = __builtin_amdgcn_readlane(up_to_lane(spans, lane), kWave - 1);
      }
    }
    const int64_t begin = (int64_t)share * length;
    if (begin >= total) return false;
    first = 0;
    for (int base = 0; base < a.batch; base += kWave) {
      if (a.batch > kWave) {
        read(base);
        spans = mine;
      }
      const int end = up_to_lane(spans, lane) + first;
      const unsigned long long behind = __ballot(end > begin);
      if (behind != 0) {
        const int l = __builtin_ctzll(behind);
        b = base + l;
        seq_len = __builtin_amdgcn_readlane(seq_len, l);
        tiles = __builtin_amdgcn_readlane(mine, l);
        span = __builtin_amdgcn_readlane(spans, l);
        first = __builtin_amdgcn_readlane(end, l) - span;
        return true;
      }
      first = __builtin_amdgcn_readlane(end, kWave - 1);
    }
    return false;
  }
  __device__ __forceinline__ static int share_length(const DecodeArgs& a, int total, int longest) {
    return max((int)(((int64_t)total + a.shares - 1) / a.shares), (longest + kMostParts - 1) / kMostParts);
  }
};

// Where the eights of tokens of a wave's steps lie, kEights lanes a step.
struct Places {
  int block, bytes;     // bytes: of the tokens that there are, 0 to 1024
  float2 scale;
};

// One query head: lane l has channels 16 (l % 8) ..+15 of tokens l / 8 of every eight.
struct OneHead {
  static constexpr int kSlots = 1, kStride = kHeadDim;
  static constexpr int kEights = 2, kRing = 4;   // of a step; steps under way
  static constexpr float kMove = 8.f;
  uint32_t q[8];
  float m, l, limit, acc[16];   // limit: m + kMove, -3e38 while no token has counted

  struct Regs {
    uint4 k[2], v[2];
  };
  __device__ __forceinline__ void init(char*, const char* query, int, int lane) {
    const uint4 a = ld16(query + (lane & 7) * 32), b = ld16(query + (lane & 7) * 32 + 16);
    q[0] = a.x, q[1] = a.y, q[2] = a.z, q[3] = a.w, q[4] = b.x, q[5] = b.y, q[6] = b.z, q[7] = b.w;
    m = 0.f;
    limit = -3e38f;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.f;
  }
  __device__ __forceinline__ float logit(uint4 k, float scale) const {
    const uint4 a = halves_of(make_uint2(k.x, k.y), scale), b = halves_of(make_uint2(k.z, k.w), scale);
    float z = dot2(q[0], a.x, 0.f), y = dot2(q[4], b.x, 0.f);
    z = dot2(q[1], a.y, z), y = dot2(q[5], b.y, y);
    z = dot2(q[2], a.z, z), y = dot2(q[6], b.z, y);
    z = dot2(q[3], a.w, z), y = dot2(q[7], b.w, y);
    z += y;
    z += as_f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u(z), 0xb1, 0xf, 0xf, false));    // lane ^ 1
    z += as_f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u(z), 0x4e, 0xf, 0xf, false));    // lane ^ 2
    z += as_f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u(z), 0x141, 0xf, 0xf, false));   // 7 - lane of eight
    return z;
  }
  __device__ __forceinline__ void add(uint4 v, float p, float scale) {
    const uint32_t codes[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes[i], scale, false);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes[i], scale, true);
      acc[4 * i] = __builtin_fmaf(p, a[0], acc[4 * i]);
      acc[4 * i + 1] = __builtin_fmaf(p, a[1], acc[4 * i + 1]);
      acc[4 * i + 2] = __builtin_fmaf(p, b[0], acc[4 * i + 2]);
      acc[4 * i + 3] = __builtin_fmaf(p, b[1], acc[4 * i + 3]);
    }
  }
  __device__ __forceinline__ void fold(const Regs& r, const Places& p, int step, float scale_log2, int lane) {
    float z[2], v_scale[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      z[i] = logit(r.k[i], from_lane(p.scale.x, 2 * step + i)) * scale_log2;
      v_scale[i] = from_lane(p.scale.y, 2 * step + i);
      const int bytes = __builtin_amdgcn_readlane(p.bytes, 2 * step + i);
      if (bytes < 1024 && lane * 16 >= bytes) z[i] = -INFINITY;   // stale slots contribute nothing
    }
    const float top = fmaxf(z[0], z[1]);
    const bool move = top > limit;
    if (__ballot(move)) {
      const float to = move ? top : m;
      const float alpha = limit < -1e38f ? 0.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      limit = move ? to + kMove : limit;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[j] *= alpha;
    }
    const float p0 = __builtin_amdgcn_exp2f(z[0] - m), p1 = __builtin_amdgcn_exp2f(z[1] - m);
    l += p0 + p1;
    add(r.v[0], p0, v_scale[0]);
    add(r.v[1], p1, v_scale[1]);
  }
  // The wave's result: acc[channel], m, l in LDS.  Eight lanes have each channel: of two that meet, each keeps half of the
  // channels (16, then 8, 4 and 2 a lane).
  struct Meeting {
    float mine, others;   // weights
  };
  __device__ __forceinline__ Meeting meet(float other_m, float other_l) {
    const float a = l != 0.f ? m : kNegBig, b = other_l != 0.f ? other_m : kNegBig;   // (NaN counts)
    m = fmaxf(a, b);
    const Meeting w = {__builtin_amdgcn_exp2f(a - m), __builtin_amdgcn_exp2f(b - m)};
    l = l * w.mine + other_l * w.others;
    return w;
  }
  __device__ __forceinline__ void finish(float* to, float* to_m, float* to_l, int lane) {
    auto across8 = [](float v) { return as_f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u(v), 0x128, 0xf, 0xf, false)); };
    Meeting w = meet(across8(m), across8(l));
    const bool high = lane & 8;
    float a8[8], a4[4], a2[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float keep = high ? acc[j + 8] : acc[j], give = high ? acc[j] : acc[j + 8];
      a8[j] = keep * w.mine + across8(give) * w.others;
    }
    // (the swaps bring the pair in the order first row, second row of the two, whichever of them a lane is in)
    auto rows = [&](auto swap, bool odd) {
      const auto pm = swap(as_u(m), as_u(m)), pl = swap(as_u(l), as_u(l));
      const Meeting x = meet(as_f(odd ? pm.first : pm.second), as_f(odd ? pl.first : pl.second));
      return odd ? Meeting{x.others, x.mine} : x;   // of the first, of the second
    };
    auto swap16 = [](uint32_t x, uint32_t y) {
      const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
      return LanePair{r[0], r[1]};
    };
    auto swap32 = [](uint32_t x, uint32_t y) {
      const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
      return LanePair{r[0], r[1]};
    };
    w = rows(swap16, lane & 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const LanePair p = swap16(as_u(a8[j]), as_u(a8[j + 4]));
      a4[j] = as_f(p.first) * w.mine + as_f(p.second) * w.others;
    }
    w = rows(swap32, lane & 32);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const LanePair p = swap32(as_u(a4[j]), as_u(a4[j + 2]));
      a2[j] = as_f(p.first) * w.mine + as_f(p.second) * w.others;
    }
    const int channel = (lane & 7) * 16 + (lane & 8) + ((lane >> 2) & 4) + ((lane >> 4) & 2);
    *reinterpret_cast<float2*>(to + channel) = make_float2(a2[0], a2[1]);
    if (lane == 0) *to_m = m, *to_l = l;
  }
};

// Up to eight query heads, 32 tokens a step, on the matrix cores (v_mfma_f32_16x16x32_f16; lane l: c = l % 16, g = l / 16).
// Keys and values lie in LDS as they came, rows of 128 bytes whose chunks of 16 are exclusive-ored with place().  Columns are those of
// GroupState: column n is head n % 8, columns 0-7 carry 2^14 times a weight rounded to fp16, columns 8-15 2^12 times what that leaves.
//   logits   first operand: row m of product t = 0, 1 is token 8 (m / 4) + 4 t + m % 4, so that a lane's results are the
//            tokens 8 g + 4 t + 0..3 of its column; a lane has the 32 channels from 32 g on, eight for each of four products.
//   values   first operand: channels 16 d + c of the tokens 8 g ..+7, turned by ds_read_b64_tr_b8; the weights that a lane has are the
//            second operand.  Nothing moves between lanes.
// A key's scale is multiplied onto its logit, a value's onto the value where it becomes an fp16 number.
struct ManyHeads {
  static constexpr int kSlots = kGroupHeads, kStride = kGroupStride;
  static constexpr int kEights = 4, kRing = 2;
  typedef int int2_t __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) int2_t lds_int2_t;
  char* stage;      // 2 * 32 rows of this wave
  uint4 q[4];       // of column c: channels 32 g + 8 j ..+7
  f32x4_t acc[8];   // [d]: channels 16 d + 4 g + i of column c
  float ref, l;     // exponent reference of the column (log2), this lane's share of its sum

  struct Regs {
    uint4 k[4], v[4];
  };
  __device__ __forceinline__ static int place(int token, int chunk) {
    return token * kRowBytes8 + ((chunk ^ ((token >> 1) & 7) ^ ((token >> 3) & 2)) << 4);
  }
  __device__ __forceinline__ void init(char* lds, const char* query, int heads, int lane) {
    stage = lds;
    const int head = lane & (kGroupHeads - 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 v = ld16(query + (head < heads ? head : 0) * kRowBytes + (lane >> 4) * 64 + j * 16);
      q[j] = head < heads ? v : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    ref = kNegBig;
    l = 0.f;
  }
  __device__ __forceinline__ static half8_t eight(uint32_t x, uint32_t y, float scale) {
    return __builtin_bit_cast(half8_t, halves_of(make_uint2(x, y), scale));
  }
  __device__ __forceinline__ void fold(const Regs& r, const Places& p, int step, float scale_log2, int lane) {
    const int c = lane & 15, g = lane >> 4;
    char* k = stage;
    char* v = stage + 32 * kRowBytes8;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = place(8 * e + (lane >> 3), lane & 7);
      st16(k + at, r.k[e]);
      st16(v + at, r.v[e]);
    }
    const int from = (step * 4 + g) * 4;
    const float k_scale = as_f((uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)as_u(p.scale.x))) * scale_log2;
    const float v_scale = as_f((uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)as_u(p.scale.y)));
    const int there = __builtin_amdgcn_ds_bpermute(from, p.bytes) >> 7;   // tokens of the lane's eight
    lds_in_order();
    float z[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int token = 8 * (c >> 2) + 4 * t + (c & 3);
      const uint4 a = ld16(k + place(token, 2 * g)), b = ld16(k + place(token, 2 * g + 1));
      f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
      auto product = [&](uint32_t x, uint32_t y, int j, f32x4_t s) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(eight(x, y, 1.f), __builtin_bit_cast(half8_t, q[j]), s, 0, 0, 0);
      };
      s0 = product(a.x, a.y, 0, s0);
      s1 = product(b.x, b.y, 2, s1);
      s0 = product(a.z, a.w, 1, s0);
      s1 = product(b.z, b.w, 3, s1);
#pragma unroll
      for (int i = 0; i < 4; ++i) z[4 * t + i] = (s0[i] + s1[i]) * k_scale;
    }
    if (__ballot(there < 8)) {   // stale slots contribute nothing
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= there) z[i] = -INFINITY;
    }
    float top = z[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
    LanePair p2 = pair_across16(as_u(top));
    p2 = pair_across32(as_u(fmaxf(as_f(p2.first), as_f(p2.second))));
    top = fmaxf(as_f(p2.first), as_f(p2.second));
    // weights stay at or below 2: the reference moves only when a logit passes that
    const bool move = top > ref + 1.f;
    if (__ballot(move)) {
      const float to = move ? top : ref;
      const float alpha = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < 8; ++d) acc[d] *= alpha;
    }
    half8_t w;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __builtin_amdgcn_exp2f(z[i] - ref);
      sum[i & 1] += x;
      const float scaled = x * kWeightScale;
      const _Float16 part = (_Float16)scaled;
      w[i] = (lane & 8) ? (_Float16)((scaled - (float)part) * kRestScale) : part;
    }
    l += sum[0] + sum[1];
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int2_t codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2_t*)(v + place(8 * g + (c >> 1), d) + (c & 1) * 8));
      acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight((uint32_t)codes.x, (uint32_t)codes.y, v_scale), w, acc[d], 0, 0, 0);
    }
    lds_in_order();
  }
  __device__ __forceinline__ void finish(float* to, float* to_m, float* to_l, int lane) {
    LanePair s = pair_across16(as_u(l));
    s = pair_across32(as_u(as_f(s.first) + as_f(s.second)));
    const int head = lane & 15, g = lane >> 4;
    const float unscale = (lane & 8) ? 1.f / (kWeightScale * kRestScale) : 1.f / kWeightScale;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = row_ror_add<8>(acc[d][i] * unscale);   // the two parts of the weights
      if (head < kGroupHeads)
        *reinterpret_cast<float4*>(to + head * kStride + 16 * d + 4 * g) = make_float4(o[0], o[1], o[2], o[3]);
    }
    if (lane < kGroupHeads) {
      to_m[lane] = ref;
      to_l[lane] = as_f(s.first) + as_f(s.second);
    }
  }
};

__device__ __forceinline__ float lse_of(float top, float sum) {
  return sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <class Head>
__global__ __launch_bounds__(kWaves* kWave, 2) void decode_e4m3_kernel(const DecodeArgs a) {
  constexpr int kSlots = Head::kSlots, kStride = Head::kStride, kEights = Head::kEights, kRing = Head::kRing;
  constexpr int kTile = kWaves * kEights * 8;
  constexpr int kStage = kSlots > 1 ? 2 * 32 * kRowBytes8 / 4 : 0, kResult = kSlots * kStride;
  __shared__ __align__(16) float acc_lds[kWaves][kStage > kResult ? kStage : kResult];
  __shared__ float m_lds[kWaves][kSlots], l_lds[kWaves][kSlots];
  __shared__ uint32_t arrived;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  const int columns = a.kv_heads * a.subs;   // KV heads, in parts of up to eight query heads
  // Work-groups go to the eight dies by turns: a share's columns are on one, where what they read at a time is adjacent (heads of
  // the same pages), and every die has the same number of work-groups (96 heads have two shares each: 296 us on two dies, 119 on eight).
  int column, index;
  if (a.per_die > 0) {
    const int at = blockIdx.x % 8 * a.per_die + blockIdx.x / 8;
    index = at / columns, column = at - index * columns;
    if (index >= a.count) return;
  } else {
    column = blockIdx.x / 8 % columns, index = blockIdx.x / 8 / columns * 8 + blockIdx.x % 8;
  }
  const int hk = column / a.subs, head0 = column % a.subs * kSlots;
  const int n_heads = min(kSlots, a.group - head0);
  Line line;
  if (!line.find<kTile>(a, index, lane)) return;
  const int64_t begin = a.shares > 0 ? (int64_t)index * line.length : 0;
  const int eights_shift = a.page_shift - 3;   // log2 of a page's eights of tokens
#pragma unroll 1
  for (;;) {
    // The share's part of sequence b: its tiles [first_tile, end_tile), the whole or one of `parts`.
    const int b = line.b, seq_len = min(max(line.seq_len, 0), a.max_pages << a.page_shift);
    const int first_tile = (int)max(begin - line.first, (int64_t)0);
    int end_tile = (int)min(begin + line.length - line.first, (int64_t)line.tiles);
    const int share0 = line.first / line.length, parts = (line.first + line.tiles - 1) / line.length - share0 + 1;
    const size_t out_row = (size_t)b * a.num_heads + (size_t)hk * a.group + head0;

    Head st;
    st.init(reinterpret_cast<char*>(acc_lds[wave]), a.q + out_row * kRowBytes, n_heads, lane);
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    const int32_t* list = a.topk != nullptr ? a.topk + ((size_t)b * a.kv_heads + hk) * a.k_pages : nullptr;
    const int seq_pages = (seq_len + (1 << a.page_shift) - 1) >> a.page_shift;
    if (list != nullptr && end_tile == line.tiles) {   // entries that are not counted in the sequence's tiles
      bool more = false;
      for (int base = (end_tile * kTile) >> a.page_shift; base < a.listed; base += 4 * kWave)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int page = list[min(base + i * kWave + lane, a.listed - 1)];
          more = more || (base + i * kWave + lane < a.listed && page >= 0 && page < seq_pages);
        }
      if (__ballot(more)) end_tile = ((a.listed << a.page_shift) + kTile - 1) / kTile;
    }
    // Places of kPlaceSteps steps at a time, those of the next in three parts while the wave is at these: the list's and the page
    // table's entries two ahead, the scales one.
    constexpr int kPlaceSteps = kWave / kEights, kTurns = kPlaceSteps / kRing;   // turns: of the ring
    const int steps = end_tile - first_tile, turns = (steps + kRing - 1) / kRing;
    struct Found {
      int at, eight, bytes;   // (page, head); eight tokens in it; 0 bytes: nothing
    };
    auto find = [&](int base) {
      const int step = base + lane / kEights;
      const int eight = ((first_tile + step) * kWaves + wave) * kEights + lane % kEights;
      const int entry = eight >> eights_shift, in_page = eight & ((1 << eights_shift) - 1);
      bool there = step < steps;
      int page = entry;
      if (list != nullptr) {
        there = there && entry < a.listed;
        page = list[there ? entry : 0];
      }
      there = there && page >= 0 && page < seq_pages;
      Found f;
      f.at = table[there ? page : 0] * a.kv_heads + hk;
      f.eight = in_page;
      f.bytes = there ? min(max(seq_len - (page << a.page_shift) - in_page * 8, 0), 8) * kRowBytes8 : 0;
      return f;
    };
    auto settle = [](Found& f) {
      f.at = settled(f.at);
      f.bytes = settled(f.bytes);
    };
    auto scale_at = [&](const Found& f) { return a.scales[f.bytes > 0 ? f.at : 0]; };
    auto places = [&](const Found& f, float2 scale) {
      Places p;
      p.block = (int)((uint32_t)f.at << eights_shift) + f.eight;
      p.bytes = f.bytes;
      scale.x = as_f((uint32_t)settled((int)as_u(scale.x)));
      scale.y = as_f((uint32_t)settled((int)as_u(scale.y)));
      p.scale = f.bytes > 0 ? scale : make_float2(1.f, 1.f);   // (a page without tokens may have any)
      return p;
    };
    typename Head::Regs r[kRing];
    auto load = [&](typename Head::Regs& to, int block, int bytes, int step) {
#pragma unroll
      for (int e = 0; e < kEights; ++e) {
        const int at = step * kEights + e;
        const uint32_t first = (uint32_t)__builtin_amdgcn_readlane(block, at);
        const int n = __builtin_amdgcn_readlane(bytes, at);
        to.k[e] = row16<true>(rows_at(a.k_pool, first, n), lane);
        to.v[e] = row16<true>(rows_at(a.v_pool, first, n), lane);
      }
    };
    Found next = find(0);
    settle(next);
    float2 scale = scale_at(next);
    Places now;
    now.block = (int)((uint32_t)next.at << eights_shift) + next.eight;
#pragma unroll
    for (int j = 0; j < kRing; ++j) load(r[j], now.block, next.bytes, j);
    now = places(next, scale);
    if (turns >= kTurns) next = find(kPlaceSteps);
#pragma unroll 1
    for (int turn0 = 0; turn0 < turns; turn0 += kTurns) {
      const int n = min(turns - turn0, kTurns);
      Found after = next;
      if (n == kTurns) {
        settle(next);
        scale = scale_at(next);
        after = find((turn0 + 2 * kTurns) * kRing);
      }
      auto ring = [&](int turn, const Places& from) {
#pragma unroll
        for (int j = 0; j < kRing; ++j) {
          if ((turn0 + turn) * kRing + j < steps) st.fold(r[j], now, turn * kRing + j, a.scale_log2, lane);
          load(r[j], from.block, from.bytes, (turn * kRing + j + kRing) & (kPlaceSteps - 1));
        }
      };
      int turn = 0;
#pragma unroll 1
      do {
        ring(turn, now);
      } while (++turn < min(n, kTurns - 1));
      if (n == kTurns) {
        const Places then = places(next, scale);
        ring(kTurns - 1, then);
        now = then;
        next = after;
      }
    }

    st.finish(acc_lds[wave], m_lds[wave], l_lds[wave], lane);
    __syncthreads();
    // Head `slot`, channels 2 lane and 2 lane + 1, over the four waves.
    auto joined = [&](int slot, float2& ml) {
      float w[kWaves], top = kNegBig, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, l_lds[i][slot] > 0.f ? m_lds[i][slot] : kNegBig);
      float2 o = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        w[i] = l_lds[i][slot] != 0.f ? __builtin_amdgcn_exp2f(m_lds[i][slot] - top) : 0.f;   // (NaN counts)
        sum += w[i] * l_lds[i][slot];
        const float2 x = *reinterpret_cast<const float2*>(&acc_lds[i][slot * kStride + lane * 2]);
        o.x += w[i] * x.x;
        o.y += w[i] * x.y;
      }
      ml = make_float2(top, sum);
      return o;
    };
    bool done = false;   // the outputs are somebody else's, or written
    if (parts > 1) {
      // A share has two places: for what began in a share before, and for what goes on in the next.
      auto place = [&](int part) { return (((size_t)(share0 + part) * 2 + (part == 0)) * columns + column) * kSlots; };
      const size_t mine = place(index - share0);
      for (int slot = wave; slot < n_heads; slot += kWaves) {
        float2 ml;
        const float2 o = joined(slot, ml);
        dev_st2(a.part_acc + (mine + slot) * kHeadDim + lane * 2, o);
        if (lane == 0) dev_st2(a.part_ml + (mine + slot) * 2, ml);
      }
      wait_stores();
      __syncthreads();
      uint32_t* counter = reinterpret_cast<uint32_t*>(a.counters + ((size_t)b * columns + column) * kTeamWordStride);
      if (threadIdx.x == 0) arrived = team_arrive(counter, a.device_fences);
      __syncthreads();
      done = arrived != (uint32_t)parts - 1;
      if (!done) {
        team_acquire(a.device_fences);
        if (threadIdx.x == 0) team_reset(counter);
        // Half a wave, four channels a lane, has a head's parts (one head: every eighth part).
        constexpr int kClasses = kSlots > 1 ? 1 : 2 * kWaves, kHalf = kWave / 2;
        const int half = lane >> 5, l = lane & (kHalf - 1), which = wave * 2 + half;
        const int slot = kSlots > 1 ? min(which, n_heads - 1) : 0, from = kSlots > 1 ? 0 : which;
        const int count = (parts - from + kClasses - 1) / kClasses, most = (parts + kClasses - 1) / kClasses;   // (most: whole wave)
        auto row = [&](int i) { return place(min(from + i * kClasses, parts - 1)) + slot; };
        float top = kNegBig, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int base = 0; base < most; base += kHalf) {
          float2 ml = dev_ld2(a.part_ml + row(base + l) * 2);
          constexpr int kAhead = 8;
          float2 x[kAhead][2];
          auto ask = [&](int i) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
              const float* at = a.part_acc + row(base + i + j) * kHeadDim + l * 4;
              x[j][0] = dev_ld2(at);
              x[j][1] = dev_ld2(at + 2);
            }
          };
          ask(0);
          if (base + l >= count) ml = make_float2(kNegBig, 0.f);
          float next = row16_max(ml.y != 0.f ? ml.x : kNegBig);   // (NaN counts)
          const LanePair m2 = pair_across16(as_u(next));
          next = fmaxf(fmaxf(as_f(m2.first), as_f(m2.second)), top);
          const float alpha = __builtin_amdgcn_exp2f(top - next);
          const float weight = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - next) : 0.f;
          const float add = row16_sum(weight * ml.y);
          const LanePair s2 = pair_across16(as_u(add));
          sum = sum * alpha + (as_f(s2.first) + as_f(s2.second));
          o.x *= alpha, o.y *= alpha, o.z *= alpha, o.w *= alpha;
          top = next;
          const int n = min(most - base, kHalf);
#pragma unroll 1
          for (int i = 0; i < n; i += kAhead) {
            if (i > 0) ask(i);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
              const float w = as_f((uint32_t)__builtin_amdgcn_ds_bpermute(((lane & kHalf) + min(i + j, kHalf - 1)) * 4, (int)as_u(weight)));
              const float by = i + j < n ? w : 0.f;
              o.x += by * x[j][0].x, o.y += by * x[j][0].y;
              o.z += by * x[j][1].x, o.w += by * x[j][1].y;
            }
          }
        }
        if constexpr (kSlots > 1) {
          if (which < n_heads) {
            const float factor = sum != 0.f ? 1.f / sum : 0.f;
            const size_t at = (out_row + slot) * kHeadDim + l * 4;
            o = make_float4(o.x * factor, o.y * factor, o.z * factor, o.w * factor);
            if (a.out_is_fp16)
              store_halves((_Float16*)a.out + at, o);
            else
              *reinterpret_cast<float4*>((float*)a.out + at) = o;
            if (a.lse != nullptr && l == 0) a.lse[out_row + slot] = lse_of(top, sum);
          }
          done = true;
        } else {
          const LanePair m2 = pair_across32(as_u(top)), s2 = pair_across32(as_u(sum));
          const float to = fmaxf(as_f(m2.first), as_f(m2.second));
          const float wa = __builtin_amdgcn_exp2f(as_f(m2.first) - to), wb = __builtin_amdgcn_exp2f(as_f(m2.second) - to);
          auto both = [&](float v) {
            const LanePair p = pair_across32(as_u(v));
            return as_f(p.first) * wa + as_f(p.second) * wb;
          };
          o = make_float4(both(o.x), both(o.y), both(o.z), both(o.w));
          if (lane < kHalf) *reinterpret_cast<float4*>(&acc_lds[wave][l * 4]) = o;
          if (lane == 0) m_lds[wave][0] = to, l_lds[wave][0] = as_f(s2.first) * wa + as_f(s2.second) * wb;
          __syncthreads();
        }
      }
    }
    if (!done) {
      for (int slot = wave; slot < n_heads; slot += kWaves) {
        float2 ml;
        const float2 o = joined(slot, ml);
        const float factor = ml.y != 0.f ? 1.f / ml.y : 0.f;
        const size_t at = (out_row + slot) * kHeadDim + lane * 2;
        if (a.out_is_fp16)
          *reinterpret_cast<half2_t*>((_Float16*)a.out + at) = half2_t{half_of(o.x * factor), half_of(o.y * factor)};
        else
          *reinterpret_cast<float2*>((float*)a.out + at) = make_float2(o.x * factor, o.y * factor);
        if (a.lse != nullptr && lane == 0) a.lse[out_row + slot] = lse_of(ml.x, ml.y);
      }
    }
    // The next sequence, if the share goes on in it.
    const int64_t end = (int64_t)line.first + line.span;
    if (a.shares == 0 || end >= begin + line.length || b + 1 >= a.batch) return;
    line.first = (int)end;
    line.at<kTile>(a, b + 1);
    __syncthreads();
  }
}

bool many_heads(const quest_cache& c) { return group_size(c) > 1; }
int tile_tokens(const quest_cache& c) { return kWaves * 8 * (many_heads(c) ? ManyHeads::kEights : OneHead::kEights); }
int columns_of(const quest_cache& c) { return kv_heads(c) * attention_subs(c); }
// Shares of a column: a work-group on every compute unit, or one a sequence.  (More of them for few sequences leave more to join and no
// more bytes under way: 128 pages of each of 32 heads 9.0 us, with twice as many 10.4; 590k tokens of 16 sequences and 8 KV heads
// 196 us and 201.)  Twice as many where there would be more than one on some units and one on others, or more than a fifth of the units
// had none: ten sequences of 3000 to 30000 tokens of 32 heads 265 -> 204 us, 40 of 900 to 8000 of 32 / 8 heads 84 -> 69, one of 30000 of
// 96 heads 119 -> 112. None where the (sequence, KV head) pairs are more than two for a compute unit: the units then even out what
// sequences differ by.  One each and in shares: 128 sequences of 10 to 2000 tokens and 8 KV heads 53 us and 73, 256 96 and 130, 65 of 500
// to 8000 101 and 123, 80 127 and 130, 100 of 4000 147 and 149, 17 of 2000 to 4000 and 32 heads 89 and 90; but 128 of 500 to 8000 and 8 KV
// heads 197 and 185, 24 of 300 to 6000 and 32 heads 119 and 98.  One long sequence is what this border is bad at: of 60000 tokens among 64 of 2000,
// 32 / 8 heads, 549 and 98 (among 63, in shares, 73; fp16 pages 121), among 16, 32 heads, 419 and 144 (fp16 224), among 39 465 and
// 179 (fp16 333).
int most_shares(const quest_cache& c) {
  const int columns = columns_of(c);
  const int64_t tiles = ((int64_t)c.max_pages_per_seq * c.page_size / tile_tokens(c) + 1) * c.batch;
  const int64_t pairs = (int64_t)c.batch * columns;
  if (pairs > 512 || tiles > INT32_MAX) return 0;
  return std::max((pairs > 256 || 256 / columns * columns < 208 ? 512 : 256) / columns, c.batch);
}
size_t share_bytes(const quest_cache& c) {
  return (size_t)2 * columns_of(c) * (many_heads(c) ? kGroupHeads : 1) * (kHeadDim + 2) * sizeof(float);
}
// (The counters' part is as long as that of an fp16 cache of the shape, also where these pages need none: one workspace serves
// both, so nothing else may lie there.)
size_t counter_bytes(const quest_cache& c) { return decode_counter_bytes(c); }

}  // namespace

size_t decode_e4m3_workspace_bytes(const quest_cache& c) {
  return counter_bytes(c) + most_shares(c) * share_bytes(c);
}

bool decode_e4m3_fits_a_launch(const quest_cache& c) {
  return ((int64_t)std::max(most_shares(c), c.batch) + 8) * columns_of(c) < 1 << 24;   // 2^32 threads
}

int launch_decode_e4m3(const quest_cache& c, const void* q, const int32_t* topk_idx, int k_pages, float sm_scale, void* out,
                       int out_is_fp16, float* lse, void* workspace, size_t workspace_bytes, const char* who, hipStream_t s) {
  DecodeArgs a = {};
  fill_attn_args(a, c, q, sm_scale, out, out_is_fp16, lse);
  a.scales = (const float2*)c.scales;
  a.topk = topk_idx;
  a.k_pages = k_pages;
  a.listed = topk_idx != nullptr ? std::min(k_pages, c.max_pages_per_seq) : 0;
  const size_t counters = counter_bytes(c);
  const size_t room = workspace != nullptr && workspace_bytes > counters ? (workspace_bytes - counters) / share_bytes(c) : 0;
  a.shares = most_shares(c);
  if (room < (size_t)a.shares) a.shares = room >= (size_t)c.batch ? (int)room : 0;   // as far as it goes
  a.counters = (uint64_t*)workspace;
  a.part_acc = (float*)((char*)workspace + counters);
  a.part_ml = a.part_acc + (size_t)a.shares * 2 * columns_of(c) * (many_heads(c) ? kGroupHeads : 1) * kHeadDim;
  a.count = a.shares > 0 ? a.shares : c.batch;
  const int64_t blocks = (int64_t)a.count * columns_of(c);
  a.loose = blocks > 256;
  // (a few sequences, too, but not many: if they are sorted by length, dies should have one of every eight)
  a.per_die = a.count % 8 != 0 && (a.shares > 0 || a.count < 24) ? (int)((blocks + 7) / 8) : 0;
  const dim3 grid((unsigned)(a.per_die > 0 ? a.per_die * 8 : (int64_t)(a.count + 7) / 8 * 8 * columns_of(c))), block(kWaves * kWave);
  if (many_heads(c))
    hipLaunchKernelGGL(decode_e4m3_kernel<ManyHeads>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(decode_e4m3_kernel<OneHead>, grid, block, 0, s, a);
  return check_launch(who);
}

}  // namespace quest
