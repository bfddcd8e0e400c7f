// Attention of one query a sequence over pages of 8 bits: listed pages, or all.
//
// Bound by memory: a token's key and value of a head are 256 bytes, read once.  The tokens of a sequence are cut into tiles of
// 64, of which each of a work-group's four waves has 16; a lane looks up the page of eight of them for 32 tiles ahead, so that nothing
// waits for a lookup behind keys and values under way.  Four steps of 4 KiB are on their way to a wave at a time.
//
// The host knows no lengths, so every work-group works out for itself how the tokens of all sequences are cut: the length of a
// split is what gives as many units (splits of a sequence) as the host asks for, however ragged the batch.  The split of a
// (sequence, KV head) that arrives last joins them (quest_team.h).
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
constexpr int kSteps = 4;                // steps under way
constexpr int kWalkSteps = 32;           // looked up at a time: two lanes a step
constexpr int kMostParts = 64;           // splits of a sequence, about
constexpr int kTileTokens8 = 64;

struct DecodeArgs : AttnArgs {
  const float2* scales;
  const int32_t* topk;
  int k_pages, listed;    // entries of a list, and how many of them count
  int most_units;         // over all sequences; 0: one a sequence
};

// A sequence's part: tiles [first_tile, end_tile).
struct Unit {
  int b, seq_len, first_tile, end_tile;
  int part, parts;        // which of the sequence's parts, of how many
};

__device__ __forceinline__ int tiles_of(const DecodeArgs& a, int seq_len) {
  const int tokens = a.topk != nullptr ? a.listed << a.page_shift : min(max(seq_len, 0), a.max_pages << a.page_shift);
  return (tokens + kTileTokens8 - 1) / kTileTokens8;
}
__device__ __forceinline__ float whole_sum(float v, int lane) {
  return as_f((uint32_t)__builtin_amdgcn_readlane((int)as_u(up_to_lane(v, lane)), kWave - 1));
}
__device__ __forceinline__ bool find_unit(Unit& u, const DecodeArgs& a, int unit, int lane) {
  int chunk = INT32_MAX;
  int tiles = 0, seq_len = 0;
  auto read = [&](int base) {
    seq_len = a.seq_lens[min(base + lane, a.batch - 1)];
    tiles = base + lane < a.batch ? tiles_of(a, seq_len) : 0;
  };
  if (a.most_units > 0) {
    float sum = 0.f;
    int longest = 0;
    for (int base = 0; base < a.batch; base += kWave) {
      read(base);
      sum += whole_sum((float)tiles, lane);
      longest = max(longest, largest_of_wave(tiles));
    }
    // With this chunk the units are at most sum / chunk + batch (a ten-thousandth covers the roundings).
    const float even = fminf(sum / (float)(a.most_units - a.batch) * 1.0001f, 1e9f);
    chunk = max((int)even + 1, (longest + kMostParts - 1) / kMostParts);
  }
  int before = 0;
  for (int base = 0; base < a.batch; base += kWave) {
    if (a.batch > kWave || a.most_units == 0) read(base);
    const int parts = base + lane < a.batch ? max(1, (int)(((int64_t)tiles + chunk - 1) / chunk)) : 0;
    const int end = up_to_lane(parts, lane) + before;
    const unsigned long long behind = __ballot(end > unit);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind);
      u.b = base + at;
      u.seq_len = min(max(__builtin_amdgcn_readlane(seq_len, at), 0), a.max_pages << a.page_shift);
      u.parts = __builtin_amdgcn_readlane(parts, at);
      u.part = unit - (__builtin_amdgcn_readlane(end, at) - u.parts);
      const int all = __builtin_amdgcn_readlane(tiles, at);
      u.first_tile = u.part * (u.parts > 1 ? chunk : 0);
      u.end_tile = u.part + 1 < u.parts ? u.first_tile + chunk : all;
      return true;
    }
    before = __builtin_amdgcn_readlane(end, kWave - 1);
  }
  return false;
}

// One query head: lane l has channels 16 (l % 8) ..+15 of tokens l / 8 of every eight.
struct OneHead {
  static constexpr int kSlots = 1, kStride = kHeadDim;
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
  __device__ __forceinline__ static void load(Regs& r, const char* k, const char* v, size_t first, size_t second, int lane) {
    r.k[0] = ld16_stream(k + first + lane * 16);
    r.k[1] = ld16_stream(k + second + lane * 16);
    r.v[0] = ld16_stream(v + first + lane * 16);
    r.v[1] = ld16_stream(v + second + lane * 16);
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
  // left: tokens of the two eights that there are (anything from below zero to above eight).
  __device__ __forceinline__ void fold(Regs& r, const int (&left)[2], const float2 (&scale)[2], float scale_log2, int lane) {
    float z[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      z[i] = logit(r.k[i], scale[i].x) * scale_log2;
      if (left[i] < 8 && (lane >> 3) >= left[i]) {   // stale slots contribute nothing, whatever they hold
        z[i] = -INFINITY;
        r.v[i] = make_uint4(0, 0, 0, 0);
      }
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
    add(r.v[0], p0, scale[0].y);
    add(r.v[1], p1, scale[1].y);
  }
  // The wave's result: acc[channel], m, l in LDS.
  template <class Pair>
  __device__ __forceinline__ void join(Pair pair) {
    const LanePair a = pair(as_u(m)), b = pair(as_u(l));
    const float la = as_f(b.first), lb = as_f(b.second);
    const float ma = la > 0.f ? as_f(a.first) : kNegBig, mb = lb > 0.f ? as_f(a.second) : kNegBig;
    const float top = fmaxf(ma, mb);
    const float wa = __builtin_amdgcn_exp2f(ma - top), wb = __builtin_amdgcn_exp2f(mb - top);
    l = la * wa + lb * wb;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const LanePair p = pair(as_u(acc[j]));
      acc[j] = as_f(p.first) * wa + as_f(p.second) * wb;
    }
    m = top;
  }
  __device__ __forceinline__ void finish(float* to, float* to_m, float* to_l, int lane) {
    join([&](uint32_t v) {
      const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false);   // lane ^ 8
      return (lane & 8) ? LanePair{other, v} : LanePair{v, other};
    });
    join([](uint32_t v) { return pair_across16(v); });
    join([](uint32_t v) { return pair_across32(v); });
    if (lane < 8) {
#pragma unroll
      for (int j = 0; j < 16; j += 4)
        *reinterpret_cast<float4*>(to + lane * 16 + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
      if (lane == 0) *to_m = m, *to_l = l;
    }
  }
};

// Up to eight query heads: lane l has channels 8 (l % 16) ..+7 of tokens l / 16 of every four.
struct ManyHeads {
  static constexpr int kSlots = kGroupHeads, kStride = kGroupStride;
  GroupState st;

  struct Regs {
    uint2 k[4], v[4];
  };
  __device__ __forceinline__ void init(char* stage, const char* query, int heads, int lane) {
    group_init(st, stage, query, heads, lane);
  }
  __device__ __forceinline__ static uint2 ld8(const char* p) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const u32x2_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p));
    return make_uint2(v.x, v.y);
  }
  __device__ __forceinline__ static void load(Regs& r, const char* k, const char* v, size_t first, size_t second, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.k[i] = ld8(k + (i < 2 ? first : second) + (i & 1) * 512 + lane * 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = ld8(v + (i < 2 ? first : second) + (i & 1) * 512 + lane * 8);
  }
  __device__ __forceinline__ void fold(Regs& r, const int (&left)[2], const float2 (&scale)[2], float scale_log2, int lane) {
    GroupRegs g;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g.k[i] = halves_of(r.k[i], scale[i >> 1].x);
      g.v[i] = halves_of(r.v[i], scale[i >> 1].y);
    }
    g.first = left[0];
    g.second = left[1];
    group_fold(st, g, scale_log2, lane);
  }
  __device__ __forceinline__ void finish(float* to, float* to_m, float* to_l, int lane) { group_finish(st, to, to_m, to_l, lane); }
};

template <class Head>
__global__ __launch_bounds__(kWaves* kWave, 2) void decode_e4m3_kernel(const DecodeArgs a) {
  constexpr int kSlots = Head::kSlots, kStride = Head::kStride;
  __shared__ __align__(16) float acc_lds[kWaves][kSlots * kStride];
  __shared__ float m_lds[kWaves][kSlots], l_lds[kWaves][kSlots];
  __shared__ uint32_t arrived;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  const int columns = a.kv_heads * a.subs;
  const int column = blockIdx.x % columns, index = blockIdx.x / columns;
  const int hk = column / a.subs, head0 = column % a.subs * kSlots;
  const int n_heads = min(kSlots, a.group - head0);
  Unit u;
  if (!find_unit(u, a, index, lane)) return;
  const size_t out_row = (size_t)u.b * a.num_heads + (size_t)hk * a.group + head0;

  Head st;
  st.init(reinterpret_cast<char*>(acc_lds[wave]), a.q + out_row * kRowBytes, n_heads, lane);
  const int32_t* table = a.page_table + (size_t)u.b * a.max_pages;
  const int32_t* list = a.topk != nullptr ? a.topk + ((size_t)u.b * a.kv_heads + hk) * a.k_pages : nullptr;
  const int eights_shift = a.page_shift - 3;   // log2 of a page's eights of tokens
  const int seq_pages = (u.seq_len + (1 << a.page_shift) - 1) >> a.page_shift;
  const int steps = u.end_tile - u.first_tile;
#pragma unroll 1
  for (int base = 0; base < steps; base += kWalkSteps) {
    const int n = min(steps - base, kWalkSteps);
    int block = 0, left = 0;
    float2 scale = make_float2(1.f, 1.f);
    {
      const int eight = ((u.first_tile + base + (lane >> 1)) * kWaves + wave) * 2 + (lane & 1);
      const int entry = eight >> eights_shift, in_page = eight & ((1 << eights_shift) - 1);
      int page = entry;
      if (list != nullptr) page = entry < a.listed ? list[entry] : -1;
      if ((lane >> 1) < n && page >= 0 && page < seq_pages) {
        const size_t at = (size_t)table[page] * a.kv_heads + hk;
        scale = a.scales[at];
        block = (int)((at << eights_shift) + in_page);
        left = u.seq_len - (page << a.page_shift) - in_page * 8;
      }
    }
    block = settled(block);
    left = settled(left);
    scale.x = as_f((uint32_t)settled((int)as_u(scale.x)));
    scale.y = as_f((uint32_t)settled((int)as_u(scale.y)));
    typename Head::Regs r[kSteps];
    auto load = [&](typename Head::Regs& to, int i) {
      i = min(i, n - 1);
      const size_t first = (size_t)(uint32_t)__builtin_amdgcn_readlane(block, 2 * i) * (8 * kRowBytes8);
      const size_t second = (size_t)(uint32_t)__builtin_amdgcn_readlane(block, 2 * i + 1) * (8 * kRowBytes8);
      Head::load(to, a.k_pool, a.v_pool, first, second, lane);
    };
    auto fold = [&](typename Head::Regs& from, int i) {
      const int there[2] = {__builtin_amdgcn_readlane(left, 2 * i), __builtin_amdgcn_readlane(left, 2 * i + 1)};
      const float2 by[2] = {make_float2(from_lane(scale.x, 2 * i), from_lane(scale.y, 2 * i)),
                            make_float2(from_lane(scale.x, 2 * i + 1), from_lane(scale.y, 2 * i + 1))};
      st.fold(from, there, by, a.scale_log2, lane);
    };
#pragma unroll
    for (int j = 0; j < kSteps; ++j) load(r[j], j);
    int i = 0;
#pragma unroll 1
    for (; i + 2 * kSteps <= n; i += kSteps)
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        fold(r[j], i + j);
        load(r[j], i + j + kSteps);
      }
    if (i + kSteps < n) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        fold(r[j], i + j);
        load(r[j], i + j + kSteps);
      }
      i += kSteps;
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
      if (i + j < n) fold(r[j], i + j);
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
  if (u.parts > 1) {
    const size_t part0 = ((size_t)index * columns + column) * kSlots;
    for (int slot = wave; slot < n_heads; slot += kWaves) {
      float2 ml;
      const float2 o = joined(slot, ml);
      dev_st2(a.part_acc + (part0 + slot) * kHeadDim + lane * 2, o);
      if (lane == 0) dev_st2(a.part_ml + (part0 + slot) * 2, ml);
    }
    wait_stores();
    __syncthreads();
    uint32_t* counter = reinterpret_cast<uint32_t*>(a.counters + ((size_t)u.b * columns + column) * kTeamWordStride);
    if (threadIdx.x == 0) arrived = team_arrive(counter, a.device_fences);
    __syncthreads();
    if (arrived != (uint32_t)u.parts - 1) return;
    team_acquire(a.device_fences);
    if (threadIdx.x == 0) team_reset(counter);
    // Parts wave, wave + 4, .. of every head; the weights a part a lane.
    const size_t first = ((size_t)(index - u.part + wave) * columns + column) * kSlots;
    const size_t step = (size_t)kWaves * columns * kSlots;
    const int mine = (u.parts - wave + kWaves - 1) / kWaves;
    for (int slot = 0; slot < n_heads; ++slot) {
      float top = kNegBig, sum = 0.f;
      float2 o = make_float2(0.f, 0.f);
      for (int base = 0; base < mine; base += kWave) {
        float2 ml = make_float2(kNegBig, 0.f);
        if (base + lane < mine) ml = dev_ld2(a.part_ml + (first + slot + (base + lane) * step) * 2);
        float next = ml.y > 0.f ? ml.x : kNegBig;
#pragma unroll
        for (int i = 1; i < kWave; i <<= 1) next = fmaxf(next, __shfl_xor(next, i));
        next = fmaxf(next, top);
        const float alpha = __builtin_amdgcn_exp2f(top - next);
        const float weight = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - next) : 0.f;
        float add = weight * ml.y;
#pragma unroll
        for (int i = 1; i < kWave; i <<= 1) add += __shfl_xor(add, i);
        sum = sum * alpha + add;
        o.x *= alpha, o.y *= alpha;
        top = next;
        const int n = min(mine - base, kWave);
#pragma unroll 1
        for (int i = 0; i < n; i += 16) {
          float2 x[16];
#pragma unroll
          for (int j = 0; j < 16; ++j)
            x[j] = dev_ld2(a.part_acc + (first + slot + (size_t)(base + min(i + j, n - 1)) * step) * kHeadDim + lane * 2);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float w = i + j < n ? from_lane(weight, i + j) : 0.f;
            o.x += w * x[j].x;
            o.y += w * x[j].y;
          }
        }
      }
      *reinterpret_cast<float2*>(&acc_lds[wave][slot * kStride + lane * 2]) = o;
      if (lane == 0) m_lds[wave][slot] = top, l_lds[wave][slot] = sum;
    }
    __syncthreads();
  }
  for (int slot = wave; slot < n_heads; slot += kWaves) {
    float2 ml;
    const float2 o = joined(slot, ml);
    const float factor = ml.y != 0.f ? 1.f / ml.y : 0.f;
    const size_t at = (out_row + slot) * kHeadDim + lane * 2;
    if (a.out_is_fp16)
      *reinterpret_cast<half2_t*>((_Float16*)a.out + at) = half2_t{half_of(o.x * factor), half_of(o.y * factor)};
    else
      *reinterpret_cast<float2*>((float*)a.out + at) = make_float2(o.x * factor, o.y * factor);
    if (a.lse != nullptr && lane == 0)
      a.lse[out_row + slot] = ml.y == 0.f ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) * kLn2;
  }
}

bool many_heads(const quest_cache& c) { return group_size(c) > 1; }
int columns_of(const quest_cache& c) { return kv_heads(c) * attention_subs(c); }
// Units of a column that are asked for: two work-groups on every compute unit.
int most_units_of(const quest_cache& c) {
  const int most = 512 / columns_of(c);
  return most > c.batch ? std::max(most, c.batch + 1) : 0;
}
size_t unit_bytes(const quest_cache& c) {
  return (size_t)columns_of(c) * (many_heads(c) ? kGroupHeads : 1) * (kHeadDim + 2) * sizeof(float);
}
// (The counters' part is as long as that of an fp16 cache of the shape, so that one workspace serves both.)
size_t counter_bytes(const quest_cache& c) { return decode_counter_bytes(c); }

}  // namespace

size_t decode_e4m3_workspace_bytes(const quest_cache& c) {
  const int units = most_units_of(c);
  return units > 0 ? counter_bytes(c) + units * unit_bytes(c) : 0;
}

bool decode_e4m3_fits_a_launch(const quest_cache& c) {
  return (int64_t)std::max(most_units_of(c), c.batch) * columns_of(c) < (1 << 24) - 1;   // 2^32 threads
}

int launch_decode_e4m3(const quest_cache& c, const void* q, const int32_t* topk_idx, int k_pages, float sm_scale, void* out,
                       int out_is_fp16, float* lse, void* workspace, size_t workspace_bytes, const char* who, hipStream_t s) {
  DecodeArgs a = {};
  fill_attn_args(a, c, q, sm_scale, out, out_is_fp16, lse);
  a.scales = (const float2*)c.scales;
  a.topk = topk_idx;
  a.k_pages = k_pages;
  a.listed = topk_idx != nullptr ? std::min(k_pages, c.max_pages_per_seq) : 0;
  a.most_units = most_units_of(c);
  const size_t counters = counter_bytes(c);
  const size_t room = workspace != nullptr && workspace_bytes > counters ? (workspace_bytes - counters) / unit_bytes(c) : 0;
  if (room < (size_t)a.most_units) a.most_units = room > (size_t)c.batch ? (int)room : 0;   // as far as it goes
  a.counters = (uint64_t*)workspace;
  a.part_acc = (float*)((char*)workspace + counters);
  const int units = std::max(a.most_units, c.batch);
  a.part_ml = a.part_acc + (size_t)units * columns_of(c) * (many_heads(c) ? kGroupHeads : 1) * kHeadDim;
  const dim3 grid((unsigned)((int64_t)units * columns_of(c))), block(kWaves * kWave);
  if (many_heads(c))
    hipLaunchKernelGGL(decode_e4m3_kernel<ManyHeads>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(decode_e4m3_kernel<OneHead>, grid, block, 0, s, a);
  return check_launch(who);
}

}  // namespace quest
