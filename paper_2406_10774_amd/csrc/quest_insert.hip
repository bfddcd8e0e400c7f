// Insertion of tokens with their rotation on the way, and insertion into pages of 8 bits (with or without rotation).
// (Insertion into fp16 pages as keys and values are given: quest_append.hip.)
//
// Rotation: of the first rotary_dim channels pair (x, y) becomes (x c - y s, x s + y c), c and s from the table's row of the token's
// position.  Products and the sum are rounded to fp32 one by one, so that the result is what the same three operations give anywhere
// (a fused multiply-add would be nearer to the exact value by less than the rounding to fp16 that follows).
//
// 8 bits: the scale of a page belongs to all of its tokens, so a wave has a whole (page, head) in registers before it rounds the first
// number.  A page that held tokens before keeps its scale unless the new ones need a larger one; then its old numbers are rounded again.
//
// Bound by memory: every number is read once and written once.  The waves of a work-group have adjacent heads; queries follow in the
// same launch, a wave having four tokens (whose table rows it then reads once) of kQHeads heads.  32749 tokens, pages of 16: 32 query / 8
// KV heads turned into pages of 8 bits 143 us (763 MB, 5.3 TB/s; a large copy 5.3), 32 heads into pages of 8 bits as they are 154 us (5.4).
// One token each of 16 sequences 5.0 us, of 32 / 8 heads turned into fp16 pages; 1 to 5 of 8 KV heads into pages of 8 bits 5.1 to 5.3:
// lengths -> page -> data -> store.  Rows alone (rotate_rows_kernel): 32768 of 32 heads 93 to 101 us (537 MB, 5.3 to 5.8 TB/s), 512 4.3.
//
// Without any length on the host: the pages of sequence b start at unit floor(cu[b] / S) + 2 b, which leaves
// room for the floor((n + S - 2) / S) + 1 pages that n >= 1 tokens can touch.
#include "quest_common.h"
#include "quest_e4m3.h"

namespace quest {

namespace {

constexpr int kPairsOf = 4;     // (page, head) pairs of a work-group: adjacent heads
constexpr int kRowWaves = 4;    // of a work-group that turns rows alone
constexpr int kQHeads = 4;

struct InsertArgs {
  char* k_pool;
  char* v_pool;
  char* meta;
  float2* scales;
  const int32_t* page_table;
  const int32_t* seq_lens;
  const int32_t* cu;
  const int32_t* rows;
  const char* k_new;
  const char* v_new;
  const char* q;
  char* q_out;
  int64_t new_stride, q_stride, q_out_stride;   // bytes between tokens
  int batch, kv_heads, q_heads, max_pages, total;
  int64_t num_phys_pages, pairs;                // pairs: (page, head) pairs at most
  int64_t insert_blocks;
  const float* table;
  const int32_t* positions;
  int num_positions, rotary, interleaved;
};

// The last sequence that starts at or before `what` (of its packed row, or its page's unit).
template <class Start>
__device__ __forceinline__ int sequence_at(const InsertArgs& a, int what, int lane, Start start) {
  int b = -1;
  for (int base = 0; base < a.batch; base += kWave) {
    const int i = base + lane;
    const bool before = i < a.batch && start(i < a.batch ? i : 0) <= what;
    const int n = __popcll(__ballot(before));
    b += n;
    if (n < kWave) break;
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// A lane's cosines and sines: it has channels 8 c .. 8 c + 7 of a token, c = lane % 16.
struct Turn {
  float4 cos0, cos1, sin0, sin1;   // (interleaved: the first of each)
  __device__ __forceinline__ void load(const InsertArgs& a, int position, int chunk) {
    const int half = a.rotary >> 1;
    if (chunk * 8 >= a.rotary) return;
    const bool there = position >= 0 && position < a.num_positions;
    const int first = a.interleaved ? chunk * 4 : chunk * 8 < half ? chunk * 8 : chunk * 8 - half;
    const float* row = a.table + (size_t)(there ? position : 0) * a.rotary + first;
    cos0 = *reinterpret_cast<const float4*>(row);
    sin0 = *reinterpret_cast<const float4*>(row + half);
    if (!a.interleaved) {
      cos1 = *reinterpret_cast<const float4*>(row + 4);
      sin1 = *reinterpret_cast<const float4*>(row + half + 4);
    }
    if (!there) {   // no number for a position without a row
      const float none = __builtin_nanf("");
      cos0 = cos1 = sin0 = sin1 = make_float4(none, none, none, none);
    }
  }
};

__device__ __forceinline__ uint32_t two_halves(float a, float b) {
  return __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});
}
// own c + other s, each operation rounded.
__device__ __forceinline__ float turned(float own, float c, float other, float s) {
#pragma clang fp contract(off)
  const float a = own * c, b = other * s;
  return a + b;
}
__device__ __forceinline__ float half_lo(uint32_t h) { return (float)__builtin_bit_cast(half2_t, h)[0]; }
__device__ __forceinline__ float half_hi(uint32_t h) { return (float)__builtin_bit_cast(half2_t, h)[1]; }

// The rotation of 8 channels; every lane of the wave has to be here (halves are exchanged between lanes).
__device__ __forceinline__ uint4 turn(const InsertArgs& a, uint4 v, const Turn& t, int chunk, int lane) {
  const bool stays = chunk * 8 >= a.rotary;
  uint4 r;
  if (a.interleaved) {
    auto pair = [&](uint32_t h, float c, float s) {
      const float x = half_lo(h), y = half_hi(h);
      return two_halves(turned(x, c, -y, s), turned(y, c, x, s));
    };
    r = make_uint4(pair(v.x, t.cos0.x, t.sin0.x), pair(v.y, t.cos0.y, t.sin0.y), pair(v.z, t.cos0.z, t.sin0.z),
                   pair(v.w, t.cos0.w, t.sin0.w));
  } else {
    const int by = a.rotary >> 4;   // lanes between the channels of a pair
    const bool second = chunk >= by;
    uint4 o;
    if (by == 8) {   // half a row of lanes away
      auto across = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false); };
      o = make_uint4(across(v.x), across(v.y), across(v.z), across(v.w));
    } else {
      const int from = (stays ? lane : second ? lane - by : lane + by) * 4;
      o = make_uint4(__builtin_amdgcn_ds_bpermute(from, v.x), __builtin_amdgcn_ds_bpermute(from, v.y),
                     __builtin_amdgcn_ds_bpermute(from, v.z), __builtin_amdgcn_ds_bpermute(from, v.w));
    }
    const float sign = second ? 1.f : -1.f;
    auto two = [&](uint32_t own, uint32_t other, float c0, float s0, float c1, float s1) {
      return two_halves(turned(half_lo(own), c0, half_lo(other), sign * s0), turned(half_hi(own), c1, half_hi(other), sign * s1));
    };
    r = make_uint4(two(v.x, o.x, t.cos0.x, t.sin0.x, t.cos0.y, t.sin0.y), two(v.y, o.y, t.cos0.z, t.sin0.z, t.cos0.w, t.sin0.w),
                   two(v.z, o.z, t.cos1.x, t.sin1.x, t.cos1.y, t.sin1.y), two(v.w, o.w, t.cos1.z, t.sin1.z, t.cos1.w, t.sin1.w));
  }
  return stays ? v : r;
}

// Queries (any packed rows): four tokens of kQHeads heads.
__device__ __forceinline__ void turn_rows(const InsertArgs& a, int64_t at, int lane) {
  const int sub = lane >> 4, chunk = lane & 15;
  const int groups = (a.q_heads + kQHeads - 1) / kQHeads;
  const int64_t four = at / groups;
  const int head0 = (int)(at - four * groups) * kQHeads;
  if (four * 4 >= a.total) return;
  const int row0 = (int)four * 4, rows_there = min(a.cu[a.batch], a.total);
  if (row0 >= rows_there) return;
  const int row = min(row0 + sub, rows_there - 1);
  const bool mine = row0 + sub < rows_there;
  uint4 v[kQHeads];
#pragma unroll
  for (int i = 0; i < kQHeads; ++i)
    v[i] = ld16_stream(a.q + row * a.q_stride + (int64_t)min(head0 + i, a.q_heads - 1) * kRowBytes + chunk * 16);
  int position;
  if (a.positions != nullptr) {
    position = a.positions[row];
  } else {
    int b = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int of = sequence_at(a, min(row0 + k, rows_there - 1), lane, [&](int i) { return a.cu[i]; });
      if (sub == k) b = of;
    }
    position = a.seq_lens[b] - (a.cu[b + 1] - row);
  }
  Turn t;
  t.load(a, position, chunk);
#pragma unroll
  for (int i = 0; i < kQHeads; ++i) {
    const uint4 r = turn(a, v[i], t, chunk, lane);
    if (mine && head0 + i < a.q_heads) st16(a.q_out + row * a.q_out_stride + (int64_t)(head0 + i) * kRowBytes + chunk * 16, r);
  }
}

__global__ __launch_bounds__(kRowWaves* kWave) void rotate_rows_kernel(const InsertArgs a) {
  turn_rows(a, (int64_t)blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane_id());
}

__device__ __forceinline__ uint32_t magnitude8(uint4 v) {
  return key_max2(key_max2(magnitude2(v.x), magnitude2(v.y)), key_max2(magnitude2(v.z), magnitude2(v.w)));
}
// The largest 16-bit magnitude of the wave.
__device__ __forceinline__ uint32_t largest_half(uint32_t m2) {
  m2 = key_max2(m2, m2 >> 16);
  m2 = key_max2(m2, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m2, 0x128, 0xf, 0xf, true));
  m2 = key_max2(m2, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m2, 0x124, 0xf, 0xf, true));
  m2 = key_max2(m2, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m2, 0x122, 0xf, 0xf, true));
  m2 = key_max2(m2, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m2, 0x121, 0xf, 0xf, true));
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)rows_key_max2(m2)) & 0xffffu;
}

// A wave's part of a page (keys or values) to 8 bits, with scale 2^e: slots first + 4 i + sub, channels 8 chunk ..+7 of x are new
// from slot `from` to slot `to`; those before hold numbers of scale `old`.
template <int kLoads>
__device__ __forceinline__ void round_part(char* block, const uint4 (&x)[kLoads], int first, int from, int to, float old, float scale,
                                           int lane) {
  const int sub = lane >> 4, chunk = lane & 15;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int slot = first + 4 * i + sub;
    uint2* at = reinterpret_cast<uint2*>(block + slot * kRowBytes8 + chunk * 8);
    if (slot >= from) {
      if (slot < to) *at = codes_of(at_most8(x[i]), scale);
    } else if (scale != old) {
      *at = codes_of(halves_of(*at, old), scale);
    }
  }
}

// How a page is shared out.  fp16 pages are one wave's, 16 tokens at a time.  Pages of 8 bits need all of their keys in registers, and
// all of their values: one wave's too, or (kApart) 16 tokens a wave, and what belongs to the page goes through LDS: pages of 64 tokens,
// turned, and pages of 32 and 64 of which the launch has no more than the SIMDs, where a wave's latency counts.  Of a turned page of 32
// tokens that is one wave's the keys are written before the values are asked for.
//   21722 tokens of 32 / 32 heads, 32 channels turned (32k of 32 / 8 heads, 128), pages of 32: so 182 (148) us; values asked for with the
//   keys 170 in the latter; apart 205 (157).  Pages of 64: apart 212 (163), as pages of 32 242 (203), in parts of 32 235 (174).  (Pages
//   of 16: 172 (141).) Without rotation, 32k tokens of 32 heads in pages of 32 (64): one wave 153 (158), apart 176 (177). One token each
//   of 16 sequences, 8 KV heads, pages of 64: one wave 6.7, apart 5.4; turned, pages of 32: 7.7 and 6.5.  1180 tokens of 32 heads (850
//   pairs of page and head) pages of 64 17.2 and 14.3; (1440 pairs) pages of 32 12.3 and 14.1.
//   Pairs are those that the launch has waves for, the most that there can be.  A step of one token a sequence has half as many or fewer,
//   but so many waves all the same; replayed, one wave and apart: 16 sequences of 40 heads (1280 pairs, 640 of them with a token) pages of 64
//   7.2 and 8.8, of 32 5.3 and 6.8, these turned 8.4 and 8.1; 65 of 8 heads 6.8 and 8.4, 5.3 and 6.7, 8.5 and 8.3; 40 of 8 heads (640)
//   pages of 32 5.0 and 5.8; 800 tokens of 32 heads (864) 6.7 and 8.8.
constexpr int kFewPairs = 1024;
template <int kS, bool k8, bool kRotate, bool kApart>
struct Shape {
  static constexpr int kParts = kApart ? kS / 16 : 1;                     // waves of a page
  static constexpr int kTokens = kS / kParts;                             // of a wave
  static constexpr int kPairs = kParts == 1 ? kPairsOf : 4 / kParts;      // of a work-group
  static constexpr int kWaves = kPairs * kParts;
  static constexpr int kEach = k8 ? kTokens : kTokens < 16 ? kTokens : 16;   // tokens at a time
};

template <int kS, bool k8, bool kRotate, bool kApart>
__global__ __launch_bounds__((Shape<kS, k8, kRotate, kApart>::kWaves * kWave)) void insert_kernel(const InsertArgs a) {
  using Of = Shape<kS, k8, kRotate, kApart>;
  constexpr int kParts = Of::kParts, kWaves = Of::kWaves, kEach = Of::kEach;
  constexpr int kLoads = kEach / 4;   // wave-wide loads of four tokens each
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (kRotate && blockIdx.x >= a.insert_blocks) {
    turn_rows(a, (blockIdx.x - a.insert_blocks) * kWaves + wave, lane);
    return;
  }
  const int64_t at = (int64_t)blockIdx.x * Of::kPairs + wave / kParts;
  const int part = wave % kParts;
  bool there = at < a.pairs;
  const int unit = there ? (int)(at / a.kv_heads) : 0;
  const int head = there ? (int)(at - (int64_t)unit * a.kv_heads) : 0;
  const int b = sequence_at(a, unit, lane, [&](int i) { return a.cu[i] / kS + 2 * i; });
  const int first_row = a.cu[b];
  const int tokens = a.cu[b + 1] - first_row;
  const int seq_len = a.seq_lens[b];
  const int first = seq_len - tokens;                              // position of the first new token
  const int page = first / kS + unit - (first_row / kS + 2 * b);
  there = there && tokens > 0 && first >= 0 && page <= (seq_len - 1) / kS && page < a.max_pages;   // (no page behind the row)
  if (kParts == 1 && !there) return;
  const int from = max(first - page * kS, 0), to = min(seq_len - page * kS, kS);   // the page's new slots
  const int phys = there ? a.page_table[(size_t)b * a.max_pages + page] : 0;
  const size_t block = (size_t)phys * a.kv_heads + head;
  const int sub = lane >> 4, chunk = lane & 15;

  uint4 k[kLoads], v[kLoads];
  uint4 mn = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
  uint4 mx = make_uint4(0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u);
  uint32_t most[2] = {0, 0};
  // Values asked for when the keys are turned leave registers for more waves (pages of 16 tokens 147 us, else 153; not where fp16 pages
  // give a wave several times 16 tokens one after the other, 163 and 159).
  constexpr bool kLate = kRotate && (k8 || kS <= 16);
  constexpr bool kKeysFirst = k8 && kRotate && kParts == 1 && kS > 16;
  // The new tokens from slot first_slot on: their keys, turned, and values; what the page's metadata and scales need of them.
  int row[kLoads];
  auto ask_values = [&] {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      v[i] = ld16_stream(a.v_new + row[i] * a.new_stride + (int64_t)head * kRowBytes + chunk * 16);
  };
  auto take = [&](int first_slot) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = first_slot + 4 * i + sub;
      const bool here = slot >= from && slot < to;
      row[i] = first_row + (here ? page * kS + slot - first : 0);
      int source = row[i];
      if (!kRotate && a.rows != nullptr) source = a.rows[source];
      const int64_t off = source * a.new_stride + (int64_t)head * kRowBytes + chunk * 16;
      k[i] = ld16_stream(a.k_new + off);
      if (!kLate) v[i] = ld16_stream(a.v_new + off);
    }
    if constexpr (kRotate) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        Turn t;
        t.load(a, a.positions != nullptr ? a.positions[row[i]] : first + row[i] - first_row, chunk);
        k[i] = turn(a, k[i], t, chunk, lane);
      }
      if (kLate && !kKeysFirst) {
        asm volatile("" ::: "memory");
        ask_values();
      }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = first_slot + 4 * i + sub;
      if (slot >= from && slot < to) {
        const uint4 key = order_key8(k[i]);
        mn = key_min8(mn, key);
        mx = key_max8(mx, key);
        if constexpr (k8) most[0] = key_max2(most[0], magnitude8(k[i]));
        if constexpr (k8 && kParts == 1 && !kKeysFirst) most[1] = key_max2(most[1], magnitude8(v[i]));
      }
    }
  };
  auto look_at_values = [&](int first_slot) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = first_slot + 4 * i + sub;
      if (slot >= from && slot < to) most[1] = key_max2(most[1], magnitude8(v[i]));
    }
  };
  if constexpr (k8) {
    const int first_slot = part * Of::kTokens;
    float2 old = make_float2(0.f, 0.f);
    if (there && from > 0) old = a.scales[block];
    const bool takes = there && first_slot + Of::kTokens > from && first_slot < to;
    if (takes) take(first_slot);
    float2 scale;
    auto scale_for = [&](uint32_t largest, float before) {
      const int e = exponent_for(largest);
      return scale_of(from > 0 ? max(e, exponent_of(before)) : e);
    };
    char* const k_block = a.k_pool + block * (kS * kRowBytes8);
    char* const v_block = a.v_pool + block * (kS * kRowBytes8);
    most[0] = largest_half(most[0]);
    if constexpr (kParts > 1) {
      // The keys' share of it first: they are written while the values are still on their way, which a barrier that waits for LDS alone
      // leaves alone.
      __shared__ uint4 bounds[kWaves][2][16];
      __shared__ uint32_t largest[kWaves][2];
      auto meet = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
      auto largest_of = [&](int which) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kParts; ++i) m = max(m, largest[wave - part + i][which]);
        return m;
      };
      mn = rows_key_min8(mn);
      mx = rows_key_max8(mx);
      if (lane < 32) bounds[wave][sub][chunk] = sub == 0 ? mn : mx;
      if (lane == 0) largest[wave][0] = most[0];
      meet();
      if (there) {
        scale.x = scale_for(largest_of(0), old.x);
        round_part<kLoads>(k_block, k, first_slot, from, to, old.x, scale.x, lane);
        if (part == 0)
#pragma unroll
          for (int i = 1; i < kParts; ++i) {
            mn = key_min8(mn, bounds[wave + i][0][chunk]);
            mx = key_max8(mx, bounds[wave + i][1][chunk]);
          }
      }
      if (takes) look_at_values(first_slot);
      most[1] = largest_half(most[1]);
      if (lane == 0) largest[wave][1] = most[1];
      meet();
      if (!there) return;
      scale.y = scale_for(largest_of(1), old.y);
      round_part<kLoads>(v_block, v, first_slot, from, to, old.y, scale.y, lane);
    } else {
      scale.x = scale_for(most[0], old.x);
      if constexpr (kKeysFirst) {
        round_part<kLoads>(k_block, k, first_slot, from, to, old.x, scale.x, lane);
        asm volatile("" ::: "memory");
        ask_values();
        look_at_values(first_slot);
      }
      most[1] = largest_half(most[1]);
      scale.y = scale_for(most[1], old.y);
      if (!kKeysFirst) round_part<kLoads>(k_block, k, first_slot, from, to, old.x, scale.x, lane);
      round_part<kLoads>(v_block, v, first_slot, from, to, old.y, scale.y, lane);
    }
    if (part == 0 && lane == 0) a.scales[block] = scale;
  } else {
#pragma unroll 1
    for (int first_slot = 0; first_slot < kS; first_slot += kEach) {
      if (first_slot + kEach <= from || first_slot >= to) continue;
      take(first_slot);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int slot = first_slot + 4 * i + sub;
        if (slot >= from && slot < to) {
          const size_t off = block * (kS * kRowBytes) + (size_t)slot * kRowBytes + chunk * 16;
          st16(a.k_pool + off, k[i]);
          st16(a.v_pool + off, v[i]);
        }
      }
    }
  }
  if (part != 0) return;
  mn = rows_key_min8(mn);
  mx = rows_key_max8(mx);
  if (lane < 32) {
    char* entry = a.meta + meta_offset(a.num_phys_pages, phys, head) + lane * 16;
    uint4 mine = sub == 0 ? mn : mx;
    if (from > 0) {
      const uint4 before = order_key8(ld16(entry));
      mine = sub == 0 ? key_min8(mine, before) : key_max8(mine, before);
    }
    st16(entry, order_key8(mine));
  }
}

// A launch has at most 2^32 - 1 threads.
bool fits_a_launch(int64_t blocks, int waves, const char* who) {
  if (blocks * waves * kWave <= UINT32_MAX) return true;
  set_error("%s: %lld work-groups of %d waves do not fit a launch", who, (long long)blocks, waves);
  return false;
}

int64_t waves_of_rows(const InsertArgs& a) { return ((int64_t)a.total + 3) / 4 * ((a.q_heads + kQHeads - 1) / kQHeads); }

template <int kS, bool k8, bool kRotate, bool kApart = false>
int launch_insert_as(InsertArgs& a, const char* who, hipStream_t s) {
  using Of = Shape<kS, k8, kRotate, kApart>;
  a.insert_blocks = (a.pairs + Of::kPairs - 1) / Of::kPairs;
  const int64_t rows = kRotate && a.q != nullptr ? (waves_of_rows(a) + Of::kWaves - 1) / Of::kWaves : 0;
  const int64_t blocks = a.insert_blocks + rows;
  if (!fits_a_launch(blocks, Of::kWaves, who)) return QUEST_ERR_SHAPE;
  hipLaunchKernelGGL((insert_kernel<kS, k8, kRotate, kApart>), dim3((unsigned)blocks), dim3(Of::kWaves * kWave), 0, s, a);
  return check_launch(who);
}
template <int kS, bool kRotate>
int launch_insert8(InsertArgs& a, const char* who, hipStream_t s) {
  if constexpr (kRotate && kS > 32) {
    return launch_insert_as<kS, true, kRotate, true>(a, who, s);
  } else {
    if constexpr (kS > 16)
      if (a.pairs <= kFewPairs) return launch_insert_as<kS, true, kRotate, true>(a, who, s);
    return launch_insert_as<kS, true, kRotate>(a, who, s);
  }
}
template <int kS>
int launch_insert_for(InsertArgs& a, bool pages8, bool rotate, const char* who, hipStream_t s) {
  if (!pages8) return launch_insert_as<kS, false, true>(a, who, s);
  return rotate ? launch_insert8<kS, true>(a, who, s) : launch_insert8<kS, false>(a, who, s);
}

InsertArgs rotation_args(const quest_cache& c, const PackedTokens& p, const quest_rotation* r) {
  InsertArgs a = {};
  a.seq_lens = c.seq_lens;
  a.cu = p.cu;
  a.batch = c.batch;
  a.total = p.total;
  if (r != nullptr) {
    a.table = r->table;
    a.positions = r->positions;
    a.num_positions = r->num_positions;
    a.rotary = r->rotary_dim;
    a.interleaved = r->interleaved != 0;
  }
  return a;
}

}  // namespace

int launch_insert(const quest_cache& c, const PackedTokens& p, const quest_rotation* rotation, const void* q, int64_t q_stride,
                  void* q_out, int64_t q_out_stride, const void* k_new, const void* v_new, int64_t new_stride,
                  const int32_t* rows, const char* who, hipStream_t s) {
  InsertArgs a = rotation_args(c, p, rotation);
  a.k_pool = (char*)c.k_pool;
  a.v_pool = (char*)c.v_pool;
  a.meta = (char*)c.meta;
  a.scales = e4m3_pages(c) ? (float2*)c.scales : nullptr;
  a.page_table = c.page_table;
  a.rows = rows;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.new_stride = new_stride * 2;
  a.q = (const char*)q;
  a.q_out = (char*)q_out;
  a.q_stride = q_stride * 2;
  a.q_out_stride = q_out_stride * 2;
  a.kv_heads = kv_heads(c);
  a.q_heads = c.num_heads;
  a.max_pages = c.max_pages_per_seq;
  a.num_phys_pages = c.num_phys_pages;
  a.pairs = ((int64_t)p.total / c.page_size + 2 * (int64_t)c.batch) * a.kv_heads;
  const bool pages8 = e4m3_pages(c), rotate = rotation != nullptr;
  switch (c.page_size) {
    case 8: return launch_insert_for<8>(a, pages8, rotate, who, s);
    case 32: return launch_insert_for<32>(a, pages8, rotate, who, s);
    case 64: return launch_insert_for<64>(a, pages8, rotate, who, s);
    default: return launch_insert_for<16>(a, pages8, rotate, who, s);
  }
}

int launch_rotate_rows(const quest_cache& c, const PackedTokens& p, const quest_rotation& rotation, const void* x, int64_t x_stride,
                       int heads, void* out, int64_t out_stride, hipStream_t s) {
  InsertArgs a = rotation_args(c, p, &rotation);
  a.q = (const char*)x;
  a.q_out = (char*)out;
  a.q_stride = x_stride * 2;
  a.q_out_stride = out_stride * 2;
  a.q_heads = heads;
  const int64_t blocks = (waves_of_rows(a) + kRowWaves - 1) / kRowWaves;
  if (!fits_a_launch(blocks, kRowWaves, "quest_rotate_tokens")) return QUEST_ERR_SHAPE;
  hipLaunchKernelGGL(rotate_rows_kernel, dim3((unsigned)blocks), dim3(kRowWaves * kWave), 0, s, a);
  return check_launch("quest_rotate_tokens");
}

}  // namespace quest
