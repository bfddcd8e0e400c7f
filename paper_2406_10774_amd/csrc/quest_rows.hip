// Attention of prompts (causal) and of trees of drafted tokens over the paged cache.  See quest_rows_core.h.
//
// Two kernels, chosen by the rows that a sequence has on average and by how much there is to do (plan_of):
//   many rows (shared_rows_kernel)  eight waves of 32 rows share the tiles of tokens, fetched once for 256 rows.  Bound by
//            the matrix cores and by power: 32k tokens of 32 query / 8 KV heads 8.45 to 8.65 ms, 1020 to 1040 TFLOP/s (a large
//            library product 1310), at 1.9 GHz; with zeros for data the clock stays at 2.4 GHz (7.0 ms where it was 8.2 to 8.5).
//   few rows (few_rows_kernel)      every wave of a work-group has all 32 rows and tiles of its own, so that four waves
//            stream tokens however few the rows are; their results are joined in LDS.  Bound by memory, or by the chain
//            of loads before the first tile: 26 drafts at 32k tokens of 32 heads 107 us, 5.0 TB/s.
// A row tile's tokens are walked in splits where that gives the compute units more to do; a row tile with more than one
// leaves partial results, which merge_rows_kernel joins (a launch of its own: 4 to 7 us, and up to 95 splits are
// joined by as many work-groups as there are rows, not by the last one to arrive).
#include <algorithm>
#include <type_traits>

#include "quest_common.h"
#include "quest_decode_core.h"
#include "quest_rows_core.h"

namespace quest {

namespace {

constexpr int kWaves = 4;                            // few_rows_kernel
constexpr int kFewRows = 32;
constexpr int kSharedWaves = 8;                      // shared_rows_kernel
constexpr int kSharedRows = 32 * kSharedWaves;
constexpr int kBuffers = 4;                          // tiles of tokens in LDS

// A work-group's part: a unit of one KV head.  Adjacent work-groups have adjacent heads: with a multiple of eight KV heads
// a head's units are all on one die, whose L2 then holds what its row tiles read at the same time.
template <bool kTree, int kRows>
struct Part {
  Sequence s;
  Stream<kTree> stream;
  int hk, unit, row0, rows, past, group, first_tile, end_tile;

  // position of a row's token (of the last one's, from there on)
  __device__ __forceinline__ int position(int row) const {
    return past + __builtin_amdgcn_readfirstlane(min(row, rows - 1) / group);
  }
  __device__ __forceinline__ bool whole() const { return stream.tiles <= s.chunk; }   // the row tile has no other split

  __device__ __forceinline__ bool find(const RowsArgs& a, const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens,
                                       const int32_t* __restrict__ page_table, const int32_t* __restrict__ topk, int lane) {
    hk = blockIdx.x % a.kv_heads;
    unit = blockIdx.x / a.kv_heads;
    if (!find_sequence<kTree, kRows, false>(s, a, cu, seq_lens, kTree && topk != nullptr, unit, lane)) return false;
    const int index = unit - s.before, slot = index / s.places<kTree>();
    int split = slot, behind = index - slot * s.places<kTree>();   // the row tile, counted from the last one
    if (s.paired<kTree>()) {
      // The one in the middle has its place alone.
      const int fewer = 2 * behind + 1 == s.row_tiles ? 0 : s.splits_of<kRows>(behind, a.group);
      split = slot < 2 * fewer ? slot >> 1 : slot - fewer;
      if (slot < 2 * fewer && (slot & 1)) behind = s.row_tiles - 1 - behind;
    }
    group = a.group;
    rows = s.tokens * group;
    row0 = (s.row_tiles - 1 - behind) * kRows;  // a prompt's last rows have the most work
    past = s.seq_len - s.tokens;
    stream.init(a, s, hk, position(row0 + kRows - 1), page_table, topk);
    first_tile = split * s.chunk;
    end_tile = s.chunk < stream.tiles - first_tile ? first_tile + s.chunk : stream.tiles;
    return first_tile < end_tile;   // (a pair may need fewer slots)
  }
  __device__ __forceinline__ size_t part_row(const RowsArgs& a, int in_tile) const {
    return ((size_t)unit * a.kv_heads + hk) * kRows + in_tile;
  }
};

// Many rows.  Two waves on each SIMD: while one of them has matrix products to do, the other is at its softmax, by
// turns that barriers keep: turn 2t is the first four waves' products (values of tile t - 1, logits of tile t) and
// the other four's softmax of tile t - 1, in turn 2t + 1 they change places.  In its turn of softmax of tile t a wave
// also asks for its share of tile t + 2, straight into LDS; it waits for that at the end of its next products, a turn
// before anyone reads it.  Four buffers: values of tile t - 2 are read until turn 2t - 1, its place is written from 2t + 1.
//
// A turn takes about 1900 cycles: the products 1450 (32 of 32 cycles; 32 KiB from LDS for each wave), the softmax 1000 and
// the fetch 300 to 700.  32k tokens of 32 / 8 heads took 12.2 ms with all waves in the same turn, 8.5 with the tiles through
// registers (this: 8.2), 9.7 in work-groups of 128 rows and no turns, two on a compute unit, and 9.9 with one
// wave of 64 rows on each SIMD and the softmax between its own products.  Reading keys or values of the next turn
// ahead changed it by less than 1 %.  (All before the sum of the weights as rounded, 16 instructions of the softmax, which adds 3 to 4 %.)
//
// k8: pages of 8 bits.  A wave has eight tokens of a tile, which are on their way to its registers for a whole step: in its turn of
// softmax of tile t it puts its share of tile t + 2 into LDS as fp16 numbers and asks for that of tile t + 3.  Tiles of drafted nodes, which
// come last, go straight to LDS as without k8.
template <bool kTree, bool kExact, bool k8>
__global__ __launch_bounds__(kSharedWaves* kWave, 2) void shared_rows_kernel(
    const RowsArgs a, const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ topk, const int64_t* __restrict__ mask) {
  constexpr int kLoads = kTileTokens / (4 * kSharedWaves);
  __shared__ __align__(16) char lds[kBuffers][2][kTileTokens * kRowBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  Part<kTree, kSharedRows> w;
  if (!w.find(a, cu, seq_lens, page_table, topk, lane)) return;
  const int row0 = w.row0 + wave * 32, row = row0 + (lane & 31);
  const bool there = row < w.rows;
  const int token = there ? row / a.group : 0;
  const int head = w.hk * a.group + (there ? row - token * a.group : 0);
  const int wave_first = w.position(row0);

  RowState<kExact, true> st;
  Walk<kTree, kTileTokens, k8> walk;
  walk.init(w.stream, w.first_tile * kTileTokens, kTileTokens);
  const int steps = w.end_tile - w.first_tile;
  uint64_t held = 0, held1 = 0, held2 = 0;   // of tiles t, t + 1, ..
  auto keys = [&](int step) { return lds[step & (kBuffers - 1)][0]; };
  auto values = [&](int step) { return lds[step & (kBuffers - 1)][1]; };
  // a wave's share of a tile: four tokens in each of kLoads pieces
  auto fetch = [&](int step) -> uint64_t {
    if (step >= steps) return 0;
    if (!walk.knows(step)) walk.find(w.stream, step, lane);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      walk.fetch(a, w.stream, w.hk, step, (i * kSharedWaves + wave) * 4, lane, lds_address(keys(step)),
                 lds_address(values(step)));
    return kTree ? walk.held(step, lane) : 0;
  };
  // k8: a wave's eight tokens of a tile, asked for and put into LDS
  static_assert(!k8 || kTileTokens == 8 * kSharedWaves, "eight tokens a wave");
  uint4 key8, value8;
  uint64_t held8 = 0;
  bool under_way = false;   // straight to LDS
  auto drafted = [&](int step) { return kTree && (w.first_tile + step) * kTileTokens >= w.stream.context; };
  auto ask8 = [&](int step) {
    if (step >= steps || drafted(step)) return;
    if (!walk.knows(step)) walk.find8(a, w.stream, w.hk, step, lane);
    walk.template load8<false>(a, w.stream, w.hk, step, wave * 8, lane, key8, value8);
    if (kTree) held8 = walk.held(step, lane);
  };
  auto put8 = [&](int step) -> uint64_t {
    if (step >= steps) return 0;
    if (drafted(step)) {
      under_way = true;
      return fetch(step);
    }
    walk.put8(walk.scales8(), step, wave * 8, lane, key8, value8, keys(step), values(step));
    return held8;
  };
  auto arrived = [&] {
    if constexpr (!k8) {
      dma_arrived<0>();
    } else if (kTree && under_way) {
      dma_arrived<0>();
      under_way = false;
    }
  };
  auto next = [&](int step) -> uint64_t {
    if constexpr (k8) {
      const uint64_t of_step = put8(step);
      ask8(step + 1);
      return of_step;
    } else {
      return fetch(step);
    }
  };
  if constexpr (k8) {
    walk.find8(a, w.stream, w.hk, 0, lane);
    st.init(a.q + (int64_t)(w.s.first + token) * a.q_stride + (int64_t)head * kRowBytes, lane);
    ask8(0);
    if constexpr (kTree) {
      held = put8(0);
      ask8(1);
    } else {
      const uint4 key0 = key8, value0 = value8;
      ask8(1);
      walk.put8(walk.scales8(), 0, wave * 8, lane, key0, value0, keys(0), values(0));
    }
    held1 = put8(1);
    ask8(2);
    st.ready(a.q_sign);
    arrived();
  } else {
    walk.find(w.stream, 0, lane);
    st.init(a.q + (int64_t)(w.s.first + token) * a.q_stride + (int64_t)head * kRowBytes, lane);
    held = fetch(0);
    held1 = fetch(1);
    st.ready(a.q_sign);
    dma_arrived<0>();
  }
  __syncthreads();
  const bool second = wave >= kSharedWaves / 2;
  if (second) __syncthreads();
  auto turn = [] {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  if (row0 < w.rows) {
    typename RowState<kExact, true>::template Weights<2> p;
    f32x16_t s[2];
    auto softmax = [&](int step) {
      if (!walk.whole(w.stream, held, step, wave_first))
        st.hide(s, walk.allow(w.stream, held, step, w.past + token, mask + (int64_t)(w.s.first + token) * a.mask_words, a.mask_words), lane);
      st.template weigh<2>(p, s, a);
      held = held1, held1 = held2;
    };
    auto rest = [&](int step) {
      arrived();
      __builtin_amdgcn_s_setprio(0);
      turn();
      held2 = next(step + 2);
      softmax(step);
      __builtin_amdgcn_s_setprio(1);   // products first where both waves could issue (1 % of the time)
      turn();
    };
    st.template logits<2>(s, keys(0), lane);
    rest(0);
    for (int step = 1; step < steps; ++step) {
      st.template add<2>(p, values(step - 1), lane);
      st.template logits<2>(s, keys(step), lane);
      rest(step);
    }
    st.template add<2>(p, values(steps - 1), lane);
  } else {
    for (int step = 0; step < steps; ++step) {
      arrived();
      turn();
      held2 = next(step + 2);
      held = held1, held1 = held2;
      turn();
    }
  }
  if (!second) __syncthreads();

  // Results: through LDS, so that 16 lanes write a row's 256 bytes together.  Two buffers that nobody reads any more have 8 KiB
  // for every wave; k_place spreads the lanes over the banks.
  if (row0 >= w.rows) return;
  const float total = st.total(), met = st.total_met();
  char* mine = lds[(steps + wave / 4) & (kBuffers - 1)][0] + wave % 4 * (32 * kRowBytes);
  const int r = lane & 31;
  auto write_rows = [&](char* to, int index, size_t row_bytes) {   // index: of the lane's row
    lds_in_order();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = i * 4 + (lane >> 4);
      const size_t row = (uint32_t)__builtin_amdgcn_ds_bpermute(at * 4, index);
      const uint4 v = ld16(mine + k_place(at, lane & 15));
      if (row0 + at < w.rows) st16(to + row * row_bytes + (lane & 15) * 16, v);
    }
    lds_in_order();
  };
  auto write_floats = [&](float factor, float* to, int index) {   // 64 channels, then the others
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      st.each4(factor, lane, [&](int d, float4 o) {
        if (d / 64 == half) *reinterpret_cast<float4*>(mine + k_place(r, d % 64 / 4)) = o;
      });
      write_rows((char*)to + half * 256, index, kHeadDim * sizeof(float));
    }
  };
  if (!w.whole()) {
    const size_t part = w.part_row(a, wave * 32);
    write_floats(kExact ? st.kUnscale : met > 0.f ? total / met : 1.f, a.part_acc + part * kHeadDim, r);   // (NaN stays in the sums)
    if (lane < 32 && there) *reinterpret_cast<float2*>(a.part_ml + (part + r) * 2) = make_float2(st.base, total);
    return;
  }
  const int out_row = (w.s.first + token) * (a.kv_heads * a.group) + head;
  const float factor = met > 0.f ? st.kUnscale / met : 0.f;
  if constexpr (kExact) {
    write_floats(factor, (float*)a.out, out_row);
  } else {
    st.each4(factor, lane, [&](int d, float4 o) { store_halves(mine + k_place(r, d / 8) + d % 8 * 2, o); });
    write_rows((char*)a.out, out_row, kHeadDim * 2);
  }
  if (a.lse != nullptr && lane < 32 && there) a.lse[out_row] = st.lse(st.base, total, a.scale);
}

// Few rows: tiles of 32 tokens, each wave its own; 16 KiB on the way to each wave's registers, 128 KiB for a compute unit.
// With 64 rows a wave (one work-group on a compute unit instead of two) 64 rows took as long as two tiles of 32: 61 us and 58
// at 65k tokens of 8 heads.  Weights keep 22 bits whatever the output's type, so that an fp16 output is the fp32 one rounded, as in
// the decode calls: a prompt of one token is as exact as a decode step.
template <bool kTree, bool kHalfOut, bool k8>
__global__ __launch_bounds__(kWaves* kWave, 2) void few_rows_kernel(
    const RowsArgs a, const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ topk, const int64_t* __restrict__ mask) {
  constexpr int kTokens = 32, kLoads = kTokens / 4;
  constexpr int kPasses = k8 && !kTree ? 2 : 1;   // of the waves' join
  constexpr int kStride = kHeadDim / kPasses + 4;
  constexpr int kStage = 2 * kTokens * (k8 && !kTree ? kRowBytes8 : kRowBytes), kJoin = kFewRows * kStride * 4;
  __shared__ __align__(16) char lds[kWaves * (kStage > kJoin ? kStage : kJoin)];
  __shared__ float ml[2][kWaves][kFewRows];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  Part<kTree, kFewRows> w;
  if (!w.find(a, cu, seq_lens, page_table, topk, lane)) return;
  int token, head;
  {
    const int row = w.row0 + (lane & 31);
    token = row < w.rows ? row / a.group : 0;
    head = w.hk * a.group + (row < w.rows ? row - token * a.group : 0);
  }
  const int first_position = w.position(w.row0);

  RowState<true, false> st;
  Walk<kTree, kTokens, k8> walk;
  walk.init(w.stream, w.first_tile * kTileTokens + wave * kTokens, kWaves * kTokens);
  const int steps = ((w.end_tile - w.first_tile) * (kTileTokens / kTokens) - wave + kWaves - 1) / kWaves;
  char* stage_k = lds + wave * kStage;
  char* stage_v = stage_k + kTokens * kRowBytes;
  uint64_t held = 0, held_next = 0;
  uint4 k[kLoads], v[kLoads];
  bool token_there[kLoads];
  auto load = [&](int step) {
    if (!walk.knows(step)) walk.find(w.stream, step, lane);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) token_there[i] = walk.load(a, w.stream, w.hk, step, i * 4, lane, k[i], v[i]);
    if (kTree) held_next = walk.held(step, lane);
  };
  auto put = [&] {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * 4 + (lane >> 4);
      st16(stage_k + k_place(at, lane & 15), k[i]);
      st16(stage_v + v_place(at, lane & 15), token_there[i] ? v[i] : make_uint4(0, 0, 0, 0));
    }
    lds_in_order();
  };
  auto fold = [&](int step) {
    const bool masked = !walk.whole(w.stream, held, step, first_position);
    uint64_t allow = ~0ull;
    if (masked)
      allow = walk.allow(w.stream, held, step, w.past + token, mask + (int64_t)(w.s.first + token) * a.mask_words, a.mask_words);
    st.template fold<1>(stage_k, stage_v, a, masked, allow, lane);
    lds_in_order();
  };
  if constexpr (k8) {
    // Pages of 8 bits: tiles lie in LDS as they came and become fp16 numbers on the way to a product, each number once, as a wave has all of
    // a tile's rows: half the LDS traffic of fp16 tiles.  26 tokens at 32k of 32 heads 57 us, with fp16 tiles 64 (40 heads, 9 to 77
    // tokens behind 35 to 2600: 38.6 and 44.2); two steps under way 64 (registers spill); three work-groups on a compute unit, with
    // queries in LDS, 63. (No load of the loop is ever skipped, so that the compiler knows how many are under way.)
    constexpr int kEights = kTokens / 8;
    // (the steps over cached tokens, which come before those over drafted nodes)
    const int cached = kTree ? min(max((w.stream.context - walk.start + walk.stride - 1) / walk.stride, 0), max(steps, 0)) : steps;
    char* stage_v8 = stage_k + kTokens * kRowBytes8;
    // Past the caches, unless other row tiles read the same tokens for long enough: one token a head at 32k of 32 heads so 52 us, else
    // 58; 32 times 10 tokens at 4000 of 32 / 8 heads (40 rows, two tiles; a split walks 63 tiles of tokens) 78 and through them 72, twice
    // 33 at 65k of 8 heads (64 tiles) 78 and 73; but 16 times 16 at 3000 of 32 / 8 heads (24) 35.1 and 35.9, 77 to 9 behind 2600 to 35 of
    // 40 heads (21) 37.4 and 38.2.
    const bool once = w.s.row_tiles == 1 || w.end_tile - w.first_tile < 32;
    auto load8 = [&](int step) {
      if (!walk.knows(step)) walk.find8(a, w.stream, w.hk, step, lane);
      if (once) {
#pragma unroll
        for (int i = 0; i < kEights; ++i) walk.template load8<true>(a, w.stream, w.hk, step, i * 8, lane, k[i], v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < kEights; ++i) walk.template load8<false>(a, w.stream, w.hk, step, i * 8, lane, k[i], v[i]);
      }
    };
    float k_scale, v_scale[2];   // of the lane's key, of its values
    auto put8 = [&](int step) {
#pragma unroll
      for (int i = 0; i < kEights; ++i) walk.put_codes(i * 8, lane, k[i], v[i], stage_k, stage_v8);
      k_scale = walk.scale_of_lane(walk.scale.x, step, st.token8(lane & 31) & 24);
#pragma unroll
      for (int i = 0; i < 2; ++i) v_scale[i] = walk.scale_of_lane(walk.scale.y, step, 16 * i + (lane >> 5) * 8);
      if (kTree) held = walk.held(step, lane);
      lds_in_order();
    };
    auto fold8 = [&](int step) {
      f32x16_t s[1];
      st.logits8(s, stage_k, k_scale, lane);
      if (!walk.whole(w.stream, held, step, first_position))
        st.hide8(s, (uint32_t)walk.allow(w.stream, held, step, w.past + token, mask + (int64_t)(w.s.first + token) * a.mask_words,
                                         a.mask_words), lane);
      typename RowState<true, false>::template Weights<1> p;
      st.template weigh<1>(p, s, a);
      st.add8(p, stage_v8, v_scale, lane);
      lds_in_order();
    };
    walk.find8(a, w.stream, w.hk, 0, lane);
    st.init(a.q + (int64_t)(w.s.first + token) * a.q_stride + (int64_t)head * kRowBytes, lane);
    if (!kTree || cached > 0) load8(0);
    st.ready(a.q_sign);
    int step = 0;
#pragma unroll 1
    for (; step + 1 < cached; ++step) {
      put8(step);
      load8(step + 1);
      fold8(step);
    }
    if (step < cached) {
      put8(step);
      fold8(step);
    }
    if constexpr (kTree)
      for (step = cached; step < steps; ++step) {
        load(step);
        held = held_next;
        put();
        fold(step);
      }
  } else {
    if (steps > 0) walk.find(w.stream, 0, lane);
    st.init(a.q + (int64_t)(w.s.first + token) * a.q_stride + (int64_t)head * kRowBytes, lane);
    if (steps > 0) load(0);
    st.ready(a.q_sign);
    for (int step = 0; step < steps; ++step) {
      held = held_next;
      put();
      if (step + 1 < steps) load(step + 1);
      fold(step);
    }
  }

  // Join the waves' results: eight threads a row, 16 channels each.
  __syncthreads();
  float* join = reinterpret_cast<float*>(lds);
  const float total = st.total();
  float* mine = join + (wave * kFewRows + (lane & 31)) * kStride;
  if (lane < kFewRows) {
    ml[0][wave][lane] = total > 0.f ? st.base : kNegBig;
    ml[1][wave][lane] = total;
  }
  constexpr int kFours = 4 / kPasses;
  const int in_tile = threadIdx.x >> 3, d0 = (threadIdx.x & 7) * (4 * kFours);
  const int row = w.row0 + in_tile;
  auto pass = [&](auto which) {
    constexpr int kFirst = decltype(which)::value * (kHeadDim / kPasses);
    if (kFirst > 0) __syncthreads();
    st.template each4<kFirst / 32, (kFirst + kHeadDim / kPasses) / 32>(
        RowState<true, false>::kUnscale, lane, [&](int d, float4 o) { *reinterpret_cast<float4*>(mine + (d - kFirst)) = o; });
    __syncthreads();
    if (row >= w.rows) return;
    float top = kNegBig, sum = 0.f, weight[kWaves];
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, ml[0][i][in_tile]);
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      weight[i] = __builtin_amdgcn_exp2f((ml[0][i][in_tile] - top) * a.scale);
      sum += weight[i] * ml[1][i][in_tile];
    }
    float4 o[kFours];
#pragma unroll
    for (int j = 0; j < kFours; ++j) {
      o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(join + (i * kFewRows + in_tile) * kStride + d0 + 4 * j);
        o[j].x += weight[i] * x.x, o[j].y += weight[i] * x.y, o[j].z += weight[i] * x.z, o[j].w += weight[i] * x.w;
      }
    }
    if (!w.whole()) {
      const size_t part = w.part_row(a, in_tile);
#pragma unroll
      for (int j = 0; j < kFours; ++j) *reinterpret_cast<float4*>(a.part_acc + part * kHeadDim + kFirst + d0 + 4 * j) = o[j];
      if (kFirst == 0 && d0 == 0) *reinterpret_cast<float2*>(a.part_ml + part * 2) = make_float2(top, sum);
      return;
    }
    const int tok = row / a.group;
    const size_t out_row = (size_t)(w.s.first + tok) * (a.kv_heads * a.group) + w.hk * a.group + (row - tok * a.group);
    const float factor = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int j = 0; j < kFours; ++j) {
      const float4 v = make_float4(o[j].x * factor, o[j].y * factor, o[j].z * factor, o[j].w * factor);
      const size_t at = out_row * kHeadDim + kFirst + d0 + 4 * j;
      if constexpr (kHalfOut)
        store_halves((_Float16*)a.out + at, v);
      else
        *reinterpret_cast<float4*>((float*)a.out + at) = v;
    }
    if (a.lse != nullptr && kFirst == 0 && d0 == 0) a.lse[out_row] = st.lse(top, sum, a.scale);
  };
  pass(std::integral_constant<int, 0>());
  if constexpr (kPasses > 1) pass(std::integral_constant<int, 1>());
}

// The partial results: a wave has some rows, one after the other, a lane a split for the weights, then two channels a
// lane.  A row's outputs are asked for with its weights (the first eight), and the next row's before they are used.
template <bool kTree, int kRows, int kMergeRows>
__global__ __launch_bounds__(256) void merge_rows_kernel(const RowsArgs a, const int32_t* __restrict__ cu,
                                                         const int32_t* __restrict__ seq_lens,
                                                         const int32_t* __restrict__ topk) {
  constexpr int kEach = kMergeRows / 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  const int hk = blockIdx.x % a.kv_heads;
  const int rest = blockIdx.x / a.kv_heads;
  const int tile = rest / (kRows / kMergeRows);
  const int in_tile = rest % (kRows / kMergeRows) * kMergeRows + wave * kEach;
  Sequence s;
  if (!find_sequence<kTree, kRows, true>(s, a, cu, seq_lens, topk != nullptr, tile, lane)) return;
  const int row0 = (tile - s.before) * kRows, rows = s.tokens * a.group;
  if (s.slots == 1 || row0 + in_tile >= rows) return;
  Stream<kTree> stream;
  stream.init(a, s, hk, s.seq_len - s.tokens + (min(row0 + kRows, rows) - 1) / a.group, nullptr, topk);
  const int parts = (stream.tiles + s.chunk - 1) / s.chunk;
  if (parts <= 1) return;  // written already, or rows that see nothing
  const size_t step = (size_t)s.places<kTree>() * a.kv_heads * kRows;   // rows between two splits' parts
  // The slot of split i: 2 i + odd for the first `turns`, then i + turns.
  int place = s.row_tiles - 1 - (tile - s.before), turns = 0, odd = 0;
  if (s.paired<kTree>()) {
    if (place > tile - s.before) {
      place = tile - s.before;
      turns = parts;
      odd = 1;
    } else if (place < tile - s.before) {
      turns = s.splits_of<kRows>(place, a.group);
    }
  }
  auto slots_on = [&](int i) { return i < turns ? 2 * i : i + turns; };   // from split 0's to split i's
  const size_t part0 = (((size_t)s.units_before + odd * s.places<kTree>() + place) * a.kv_heads + hk) * kRows + in_tile;
  const int n_rows = min(kEach, rows - row0 - in_tile);
  const float2* ml0 = reinterpret_cast<const float2*>(a.part_ml) + part0 + slots_on(min(lane, parts - 1)) * step;
  float2 first = *ml0;   // of a row's first 64 splits
#pragma unroll 1
  for (int r = 0; r < n_rows; ++r) {
    const float2* from = reinterpret_cast<const float2*>(a.part_acc + (part0 + r) * kHeadDim) + lane;
    int next = 0;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + part0 + r;
    float2 v[8];
    auto ask = [&] {   // the next eight parts' outputs
#pragma unroll
      for (int j = 0; j < 8; ++j, ++next) {
        v[j] = *from;
        if (next < parts - 1) from += next < turns ? step * kHeadDim : step * (kHeadDim / 2);
      }
    };
    ask();
    const float2 these = first;
    if (r + 1 < n_rows) first = ml0[r + 1];
    float top = these.y > 0.f ? these.x : kNegBig, sum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 1
    for (int base = kWave; base < parts; base += kWave) {
      const float2 x = ml[slots_on(min(base + lane, parts - 1)) * step];
      if (x.y > 0.f) top = fmaxf(top, x.x);
    }
#pragma unroll
    for (int i = 1; i < kWave; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
#pragma unroll 1
    for (int base = 0; base < parts; base += kWave) {
      const float2 x = base == 0 ? these : ml[slots_on(min(base + lane, parts - 1)) * step];
      const float weight = base + lane < parts && x.y > 0.f ? __builtin_amdgcn_exp2f((x.x - top) * a.scale) : 0.f;
      sum += weight * x.y;
      const int n = min(parts - base, kWave);
#pragma unroll 1
      for (int i = 0; i < n; i += 8) {
        float2 now[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) now[j] = v[j];
        if (next < parts) ask();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float w = i + j < n ? from_lane(weight, i + j) : 0.f;
          o0 += now[j].x * w;
          o1 += now[j].y * w;
        }
      }
    }
#pragma unroll
    for (int i = 1; i < kWave; i <<= 1) sum += __shfl_xor(sum, i);
    const int row = row0 + in_tile + r, token = row / a.group;
    const size_t out_row = (size_t)(s.first + token) * (a.kv_heads * a.group) + hk * a.group + (row - token * a.group);
    const float factor = sum > 0.f ? 1.f / sum : 0.f;
    const size_t at = out_row * kHeadDim + lane * 2;
    if (a.out_is_fp16)
      *reinterpret_cast<half2_t*>((_Float16*)a.out + at) = half2_t{half_of(o0 * factor), half_of(o1 * factor)};
    else
      *reinterpret_cast<float2*>((float*)a.out + at) = make_float2(o0 * factor, o1 * factor);
    if (a.lse != nullptr && lane == 0) a.lse[out_row] = RowState<true, false>::lse(top, sum, a.scale);
  }
}

// How a call is cut up, from what the host knows.  The figures are of 820 calls, from 6 to 12000 rows a sequence over contexts
// up to 60000 tokens by 1 to 64 heads, each with both kernels, with and without splits: the rules take 1 % longer than the
// best of the four on average.  (The lengths of a batch were from half or a quarter of the longest, page-table rows ended with it, and
// the small kernel rounded the weights of fp16 outputs, 1.00 to 1.12 times as fast as it is.)  The row of the page table is taken for the
// longest length: in wide tables short prompts have the large kernel and splits that find nothing to split (77 tokens of 32 heads in rows
// of 2048 pages 13.4 us, in rows of their own length 6.7).
//   Splits: where the row tiles leave compute units idle for long enough.  Idle is the share of the units without
//   a row tile times the row's tiles of tokens; a join costs as much as 8 to 12 of them (60 drafts of 8 heads at 600
//   tokens 12 us with splits and 15 without), 20 to 25 where more than a third of the units have a row tile (sixteen
//   sequences of 400 rows behind 2000 tokens: 37 us without, 43 with), and 30 to 50 where the splits do not fit the units
//   at once any more (400 tokens behind 600 of 32 / 8 heads 22 us without, 46 with; 24 nodes in fifteen sequences of 20000
//   tokens 340 without, 254 with).  None for rows of at most eight tiles.
//   So many that the work-groups fill the compute units once; an even share then ends at the same time
//   everywhere (26 drafts at 32k tokens: 105 us, with twice as many 110, four times 122).  Where there are row tiles for
//   more than half of that (many rows of trees: a quarter) their unequal ends weigh more than a start does, and the share
//   is cut into rounds: two, and four for many rows of trees (sixteen ragged trees of 1 to 2 tiles: 1830 us in one
//   round, 1245 in two, 1000 in four).
//   Kernel: the small one does a quarter of the large one's work in the same time where there is enough of it, but is a
//   third of it to start and to join.  It has calls of up to 64 rows a sequence (64 rows at 65k tokens of 8 heads:
//   56 us and 63 with the large one; 128 rows: 89 and 67), and those of less than 80 row tiles of the large one and
//   little work, counted in 256 rows by 64 tokens: 3000 (400 tokens behind 600 of 32 / 8 heads: 22 us and 33; fifteen
//   prompts of 250 to 500 tokens of 64 / 8 heads: 182 and 82), or 800 where the large one would split (60 tokens in ten
//   sequences of 6000 of 64 / 8 heads 160 and 153, one of 150 behind 3000 59 and 40).
//   Pages of 8 bits have the same borders, though the small kernel is faster on them and the large one is not.  The small and the large
//   one there, us (in brackets with fp32 outputs): 64 rows at 65k tokens of 8 heads 51 and 62 (50, 80), 128 rows 81 and 64 to 67 (81, 86 to
//   88), 256 145 and 87 (143, 118 to 121); 400 tokens behind 600 of 32 / 8 heads 21 and 38 (22, 44); 60 in ten sequences of 6000 of 64 / 8
//   heads 240 and 167 to 180 (237, 221 to 235), one of 150 behind 3000 52 and 41 (53, 50), fifteen prompts of 400 186 and 92 (200, 121); 77
//   in three of 2600, 40 heads, 49 and 68 (49, 92).
struct Plan {
  int rows;                     // of a row tile: kFewRows or kSharedRows
  int row_tiles;                // of a KV head, at most
  int most_units, least_chunk;  // of a KV head; 0 units: no splits
};
// Work-groups of a KV head that the compute units take at once: two few_rows_kernel each, or one shared_rows_kernel.
int at_once(int rows, const quest_cache& c) { return std::max(1, (rows == kFewRows ? 512 : 256) / kv_heads(c)); }
// Whether tokens are split where row tiles of `of` rows fill a share of the units, and into how many rounds.
bool worth_splits(int of, double fill, int64_t places) {
  const double idle = (double)places / kTileTokens * (1 - fill);
  const bool few = of == kFewRows;
  return places > 8 * kTileTokens && idle > (fill < 0.15 ? 8 : fill < 0.3 ? 12 : fill < 0.5 ? (few ? 25 : 20) : few ? 50 : 30);
}
int rounds_of(int of, int64_t row_tiles, int once, bool tree) {
  const int most = tree && of == kSharedRows ? 4 : 2;
  return row_tiles * most <= once ? 1 : most;
}
// k_pages: listed pages (0: all).
Plan plan_of(const quest_cache& c, int total_tokens, bool tree, int k_pages) {
  const int64_t rows = (int64_t)total_tokens * group_size(c), mean = (rows + c.batch - 1) / c.batch;
  const int64_t new_tokens = total_tokens / c.batch;
  const int64_t pages = k_pages > 0 ? std::min(k_pages, c.max_pages_per_seq) : c.max_pages_per_seq;
  const int64_t places = pages * c.page_size + (tree ? new_tokens : 0);   // that a row may attend to
  auto likely = [&](int of) { return std::max<int64_t>(c.batch, rows / of); };   // row tiles
  auto splits = [&](int of) { return worth_splits(of, (double)likely(of) / at_once(of, c), places); };
  const double wide = (double)rows * kv_heads(c) / kSharedRows;
  const double work = wide * (tree ? places : std::max(places - new_tokens / 2, places / 2)) / kTileTokens;
  Plan p;
  const bool few = mean <= 64 || (wide < 80 && work < (splits(kSharedRows) ? 800 : 3000));
  p.rows = few ? kFewRows : kSharedRows;
  p.row_tiles = (int)(rows / p.rows + c.batch);
  const int once = at_once(p.rows, c);
  p.least_chunk = few ? 2 : 8;
  p.most_units = splits(p.rows) ? std::max(once * rounds_of(p.rows, likely(p.rows), once, tree), p.row_tiles + (tree ? 1 : c.batch + 1)) : 0;
  return p;
}
int units_of(const Plan& p) { return std::max(p.row_tiles, p.most_units); }
size_t unit_bytes(int rows, const quest_cache& c) { return (size_t)kv_heads(c) * rows * (kHeadDim + 2) * sizeof(float); }

template <bool kTree, bool kExact, bool k8 = false>
int launch_rows(const quest_cache& c, RowsArgs& a, int total_tokens, const int32_t* topk, void* workspace, size_t bytes,
                const char* who, hipStream_t s) {
  Plan p = plan_of(c, total_tokens, kTree, topk != nullptr ? a.k_pages : 0);
  const size_t room = workspace != nullptr ? bytes / unit_bytes(p.rows, c) : 0;
  if (room < (size_t)units_of(p)) p.most_units = room > (size_t)p.row_tiles ? (int)room : 0;  // as far as it goes
  const bool exact = kExact || p.rows == kFewRows;
  a.below = (exact ? RowState<true, false>::kBelow : RowState<false, true>::kBelow) / a.scale;
  a.limit = (exact ? RowState<true, false>::kMove : RowState<false, true>::kMove) / a.scale;
  a.most_units = p.most_units;
  a.least_chunk = p.least_chunk;
  a.part_acc = (float*)workspace;
  a.part_ml = a.part_acc + (size_t)units_of(p) * a.kv_heads * p.rows * kHeadDim;
  const dim3 grid((unsigned)(units_of(p) * a.kv_heads)), block((p.rows == kSharedRows ? kSharedWaves : kWaves) * kWave);
  if (p.rows == kFewRows)
    hipLaunchKernelGGL((few_rows_kernel<kTree, !kExact, k8>), grid, block, 0, s, a, a.cu, a.seq_lens, c.page_table, topk, a.mask);
  else
    hipLaunchKernelGGL((shared_rows_kernel<kTree, kExact, k8>), grid, block, 0, s, a, a.cu, a.seq_lens, c.page_table, topk, a.mask);
  const int r = check_launch(who);
  if (r != QUEST_OK || p.most_units == 0) return r;
  const unsigned tiles = (unsigned)(p.row_tiles * a.kv_heads);
  // Few rows: work-groups of as few of them as the compute units take at once, 2048 work-groups, so that a wave has one row, two or four.
  // Four times 16 nodes over 128 listed pages of 32 / 8 heads (96 row tiles) 22.9 us with four rows, 26.0 with 16; 40 heads, 77 tokens
  // behind 2600 (280 row tiles) 50.2 with four rows, 47.5 with eight, 48.7 with 16.
  if (p.rows == kFewRows && tiles <= 256)
    hipLaunchKernelGGL((merge_rows_kernel<kTree, kFewRows, 4>), dim3(tiles * (kFewRows / 4)), dim3(256), 0, s, a, a.cu,
                       a.seq_lens, topk);
  else if (p.rows == kFewRows && tiles <= 512)
    hipLaunchKernelGGL((merge_rows_kernel<kTree, kFewRows, 8>), dim3(tiles * (kFewRows / 8)), dim3(256), 0, s, a, a.cu,
                       a.seq_lens, topk);
  else if (p.rows == kFewRows)
    hipLaunchKernelGGL((merge_rows_kernel<kTree, kFewRows, 16>), dim3(tiles * (kFewRows / 16)), dim3(256), 0, s, a, a.cu,
                       a.seq_lens, topk);
  else if (tiles <= 32)
    hipLaunchKernelGGL((merge_rows_kernel<kTree, kSharedRows, 4>), dim3(tiles * (kSharedRows / 4)), dim3(256), 0, s, a,
                       a.cu, a.seq_lens, topk);
  else
    hipLaunchKernelGGL((merge_rows_kernel<kTree, kSharedRows, 16>), dim3(tiles * (kSharedRows / 16)), dim3(256), 0, s, a,
                       a.cu, a.seq_lens, topk);
  return check_launch(who);
}

RowsArgs rows_args(const quest_cache& c, const PackedTokens& p, const void* q, int64_t q_stride, float sm_scale, void* out,
                   int out_is_fp16, float* lse) {
  RowsArgs a = {};
  a.q = (const char*)q;
  a.k_pool = (const char*)c.k_pool;
  a.v_pool = (const char*)c.v_pool;
  a.scales = e4m3_pages(c) ? (const float2*)c.scales : nullptr;
  a.cu = p.cu;
  a.seq_lens = c.seq_lens;
  a.out = out;
  a.lse = lse;
  a.q_stride = q_stride * 2;
  a.batch = c.batch;
  a.max_pages = c.max_pages_per_seq;
  a.page_shift = page_shift_of(c.page_size);
  a.kv_heads = kv_heads(c);
  a.group = group_size(c);
  a.out_is_fp16 = out_is_fp16;
  a.q_sign = sm_scale < 0.f ? 0x80008000u : 0u;
  a.scale = std::max(std::abs(sm_scale) * kLog2e, 1e-30f);  // scale 0: all weights alike
  return a;
}

}  // namespace

// The most that plan_of asks for in calls with any number of tokens up to this one: of each kernel that such a call may have, and
// only if any of them is split.  Fewer tokens have fewer row tiles, and row tiles that fill the units are not split.
size_t tokens_workspace_bytes(const quest_cache& c, int total_tokens) {
  const int64_t rows = (int64_t)total_tokens * group_size(c);
  const int64_t places = (int64_t)c.max_pages_per_seq * c.page_size + total_tokens / c.batch;
  auto most = [&](int of) -> size_t {
    const int once = at_once(of, c);
    if (!worth_splits(of, (double)c.batch / once, places)) return 0;
    const int64_t tiles = std::min<int64_t>(rows / of, once);
    const int rounds = rounds_of(of, std::max<int64_t>(tiles, c.batch), once, true);
    return (size_t)std::max<int64_t>((int64_t)once * rounds, tiles + 2 * (int64_t)c.batch + 1) * unit_bytes(of, c);
  };
  const double wide = (double)rows * kv_heads(c) / kSharedRows;
  const bool many = rows > 64 * (int64_t)c.batch && (wide >= 80 || wide * places / kTileTokens >= 800);
  return total_tokens == 0 ? 0 : std::max(most(kFewRows), many ? most(kSharedRows) : 0);
}

bool rows_fit_a_launch(const quest_cache& c, int total_tokens) {
  return ((int64_t)total_tokens * group_size(c) + 2 * kSharedRows * (int64_t)c.batch) * kv_heads(c) <= INT32_MAX;
}

int launch_prompt(const quest_cache& c, const PackedTokens& p, const void* q, int64_t q_stride, float sm_scale, void* out,
                  int out_is_fp16, float* lse, void* workspace, size_t workspace_bytes, hipStream_t s) {
  RowsArgs a = rows_args(c, p, q, q_stride, sm_scale, out, out_is_fp16, lse);
  const auto launch = e4m3_pages(c) ? (out_is_fp16 ? launch_rows<false, false, true> : launch_rows<false, true, true>)
                                    : (out_is_fp16 ? launch_rows<false, false> : launch_rows<false, true>);
  return launch(c, a, p.total, nullptr, workspace, workspace_bytes, "quest_prompt_attention", s);
}

int launch_tree(const quest_cache& c, const PackedTokens& p, const void* q, int64_t q_stride, const void* k_new,
                const void* v_new, int64_t new_stride, const int64_t* mask, int mask_words, const int32_t* topk_idx, int k_pages,
                float sm_scale, void* out, int out_is_fp16, float* lse, void* workspace, size_t workspace_bytes,
                hipStream_t s) {
  RowsArgs a = rows_args(c, p, q, q_stride, sm_scale, out, out_is_fp16, lse);
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.new_stride = new_stride * 2;
  a.mask = mask;
  a.mask_words = mask_words;
  a.k_pages = k_pages;
  const auto launch = e4m3_pages(c) ? (out_is_fp16 ? launch_rows<true, false, true> : launch_rows<true, true, true>)
                                    : (out_is_fp16 ? launch_rows<true, false> : launch_rows<true, true>);
  return launch(c, a, p.total, topk_idx, workspace, workspace_bytes, "quest_tree_attention", s);
}

}  // namespace quest
