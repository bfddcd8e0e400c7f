// Attention of prompts (causal) and of trees of drafted tokens over the paged cache.  See quest_rows_core.h.
#include <algorithm>

#include "quest_common.h"
#include "quest_decode_core.h"
#include "quest_rows_core.h"

namespace quest {

namespace {

constexpr int kSharedWaves = 4;                       // waves of 32 rows that share the tiles of tokens
constexpr int kSharedRows = 32 * kSharedWaves;

// What the threads of a work-group fetch of a tile of 64 tokens: 16 tokens in each of four loads, four tokens (in
// one page) a wave.
constexpr int kLoads = kTileTokens / (4 * kSharedWaves);

struct Tile {
  uint4 k[kLoads], v[kLoads];
};

template <bool kTree, bool kExact>
__global__ __launch_bounds__(kSharedWaves* kWave, 2) void shared_rows_kernel(
    const RowsArgs a, const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ topk, const int64_t* __restrict__ mask) {
  __shared__ __align__(16) char lds[2][2][kTileTokens * kRowBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  const int hk = blockIdx.x % a.kv_heads;
  const int split = blockIdx.x / a.kv_heads % a.splits;
  const int slot = a.slots - 1 - (int)(blockIdx.x / a.kv_heads / a.splits);  // a prompt's last rows have the most work
  RowTile t;
  if (!find_tile<kSharedRows>(t, cu, a.batch, a.group, slot, lane)) return;
  const int32_t* table = page_table + (size_t)t.b * a.max_pages;
  const int seq_len = seq_lens[t.b];
  const int page_mask = (1 << a.page_shift) - 1;

  // this lane's row, and the tokens that the wave's and the work-group's rows attend to
  const int row = t.row0 + wave * 32 + (lane & 31);
  const bool there = row < t.rows;
  const int token = there ? row / a.group : t.tokens - 1;
  const int head = hk * a.group + (there ? row - token * a.group : 0);
  const int past = seq_len - t.tokens;                                  // prompts: tokens before the new ones
  const int wave_first = past + min(t.row0 + wave * 32, t.rows - 1) / a.group;
  const int wave_last = past + min(t.row0 + wave * 32 + 31, t.rows - 1) / a.group;
  const int group_last = past + min(t.row0 + kSharedRows - 1, t.rows - 1) / a.group;
  // tiles: of the context, then (trees) of the drafted tokens
  const int limit = kTree ? seq_len : group_last + 1;
  const bool list = kTree && topk != nullptr;
  const int32_t* pages = list ? topk + ((size_t)t.b * a.kv_heads + hk) * a.k_pages : nullptr;
  const int seq_pages = (seq_len + page_mask) >> a.page_shift;
  const int context_tiles =
      list ? (int)((((int64_t)min(a.k_pages, a.max_pages) << a.page_shift) + kTileTokens - 1) / kTileTokens)
           : (limit + kTileTokens - 1) / kTileTokens;
  const int all_tiles = context_tiles + (kTree ? (t.tokens + kTileTokens - 1) / kTileTokens : 0);
  const int first_tile = (int)((int64_t)all_tiles * split / a.splits);
  const int end_tile = (int)((int64_t)all_tiles * (split + 1) / a.splits);

  RowState<kExact> st;
  st.init(a.q + (int64_t)(t.first + token) * a.q_stride + (int64_t)head * kRowBytes, there, a.q_sign, lane);

  // The physical page (and how many of the four tokens are there) of each of a tile's loads.
  int phys[kLoads], count[kLoads];
  auto find_pages = [&](int tile) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = tile * kTileTokens + i * (4 * kSharedWaves) + wave * 4;
      if (kTree && tile >= context_tiles) {
        count[i] = t.tokens - (at - context_tiles * kTileTokens);
      } else if (list) {
        const int entry = at >> a.page_shift;
        const int page = entry < min(a.k_pages, a.max_pages) ? pages[entry] : -1;
        const bool valid = page >= 0 && page < seq_pages;
        count[i] = valid ? seq_len - (page << a.page_shift) - (at & page_mask) : 0;
        phys[i] = valid ? table[page] : 0;
      } else {
        count[i] = limit - at;
        phys[i] = table[min(at, limit - 1) >> a.page_shift];
      }
    }
  };
  auto load = [&](Tile& r, int tile) {
    const int sub = lane >> 4, chunk = lane & 15;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = tile * kTileTokens + i * (4 * kSharedWaves) + wave * 4;
      const char *k, *v;
      if (kTree && tile >= context_tiles) {
        const int node = min(at - context_tiles * kTileTokens + sub, t.tokens - 1);
        const int64_t off = (int64_t)(t.first + node) * a.new_stride + (int64_t)hk * kRowBytes + chunk * 16;
        k = a.k_new + off;
        v = a.v_new + off;
      } else {
        const size_t off =
            ((((size_t)phys[i] * a.kv_heads + hk) << a.page_shift) + (at & page_mask) + sub) * kRowBytes + chunk * 16;
        k = a.k_pool + off;
        v = a.v_pool + off;
      }
      r.k[i] = ld16(k);
      r.v[i] = ld16(v);
      if (sub >= count[i]) r.v[i] = make_uint4(0, 0, 0, 0);  // stale slots may hold anything
    }
  };
  auto store = [&](const Tile& r, int buffer) {
    const int chunk = lane & 15;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * (4 * kSharedWaves) + wave * 4 + (lane >> 4);
      st16(lds[buffer][0] + k_place(at, chunk), r.k[i]);
      st16(lds[buffer][1] + v_place(at, chunk), r.v[i]);
    }
  };

  if (first_tile < end_tile) {
    Tile next;
    find_pages(first_tile);
    load(next, first_tile);
    store(next, 0);
    __syncthreads();
    for (int tile = first_tile; tile < end_tile; ++tile) {
      const int buffer = (tile - first_tile) & 1;
      if (tile + 1 < end_tile) {
        find_pages(tile + 1);
        load(next, tile + 1);
      }
      const int t0 = tile * kTileTokens;
      bool masked = false, skip = false;
      uint64_t allow = ~0ull;
      auto first_bits = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
      if (!kTree) {
        masked = t0 + kTileTokens - 1 > wave_first;
        skip = t0 > wave_last;
        if (masked) allow = first_bits(past + token + 1 - t0);
      } else if (tile >= context_tiles) {
        masked = true;
        const int words = tile - context_tiles;
        allow = words < a.mask_words ? (uint64_t)mask[(int64_t)(t.first + token) * a.mask_words + words] : 0;
        allow &= first_bits(t.tokens - words * kTileTokens);
      } else if (list) {
        const int entry = (t0 + lane) >> a.page_shift;
        const int page = entry < min(a.k_pages, a.max_pages) ? pages[entry] : -1;
        allow = __ballot(page >= 0 && page < seq_pages &&
                         ((int64_t)page << a.page_shift) + ((t0 + lane) & page_mask) < seq_len);
        masked = allow != ~0ull;
      } else {
        masked = t0 + kTileTokens > limit;
        allow = first_bits(limit - t0);
      }
      if (!skip) st.template fold<2>(lds[buffer][0], lds[buffer][1], a.scale_log2, masked, allow, lane);
      if (tile + 1 < end_tile) store(next, buffer ^ 1);
      __syncthreads();
    }
  }

  const float total = st.total();
  if (a.splits > 1) {
    const size_t part = (((size_t)split * a.slots + slot) * a.kv_heads + hk) * kSharedRows + wave * 32 + (lane & 31);
    if (there) {
      st.each4(RowState<kExact>::kUnscale, lane,
               [&](int d, float4 v) { *reinterpret_cast<float4*>(a.part_acc + part * kHeadDim + d) = v; });
      if (lane < 32) *reinterpret_cast<float2*>(a.part_ml + part * 2) = make_float2(st.ref, total);
    }
    return;
  }
  if (!there) return;
  const size_t out_row = (size_t)(t.first + token) * (a.kv_heads * a.group) + head;
  const float factor = total > 0.f ? RowState<kExact>::kUnscale / total : 0.f;
  st.each4(factor, lane, [&](int d, float4 v) { store4(a.out, a.out_is_fp16, out_row * kHeadDim + d, v); });
  if (a.lse != nullptr && lane < 32)
    a.lse[out_row] = total > 0.f ? (st.ref + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
}

// The splits of each row: a wave a row, two channels a lane.
template <int kRows>
__global__ __launch_bounds__(256) void merge_rows_kernel(const RowsArgs a, const int32_t* __restrict__ cu) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id();
  const int hk = blockIdx.x % a.kv_heads;
  const int rest = blockIdx.x / a.kv_heads;
  const int in_tile = rest % (kRows / 4) * 4 + wave;
  const int slot = rest / (kRows / 4);
  RowTile t;
  if (!find_tile<kRows>(t, cu, a.batch, a.group, slot, lane)) return;
  const int row = t.row0 + in_tile;
  if (row >= t.rows) return;
  const size_t part0 = ((size_t)slot * a.kv_heads + hk) * kRows + in_tile;
  const size_t step = (size_t)a.slots * a.kv_heads * kRows;
  float top = kNegBig;
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (part0 + s * step) * 2);
    if (ml.y > 0.f) top = fmaxf(top, ml.x);
  }
  float sum = 0.f, o0 = 0.f, o1 = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (part0 + s * step) * 2);
    if (!(ml.y > 0.f)) continue;
    const float w = __builtin_amdgcn_exp2f(ml.x - top);
    const float2 v = *reinterpret_cast<const float2*>(a.part_acc + (part0 + s * step) * kHeadDim + lane * 2);
    sum += ml.y * w;
    o0 += v.x * w;
    o1 += v.y * w;
  }
  const int token = row / a.group;
  const size_t out_row = (size_t)(t.first + token) * (a.kv_heads * a.group) + hk * a.group + (row - token * a.group);
  const float factor = sum > 0.f ? 1.f / sum : 0.f;
  store_out2(a.out, a.out_is_fp16, out_row * kHeadDim + lane * 2, o0 * factor, o1 * factor);
  if (a.lse != nullptr && lane == 0)
    a.lse[out_row] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

constexpr int kMaxSplits = 64;

int64_t slots_of(const quest_cache& c, int total_tokens, int rows) {
  return (int64_t)total_tokens * group_size(c) / rows + c.batch;
}

// Splits of the tokens: as many work-groups as the compute units hold at once, two each.
int splits_of(const quest_cache& c, int total_tokens) {
  const int64_t groups = slots_of(c, total_tokens, kSharedRows) * kv_heads(c);
  const int64_t tiles = ((int64_t)c.max_pages_per_seq * c.page_size + kTileTokens - 1) / kTileTokens;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / groups, tiles, kMaxSplits}));
}

size_t split_bytes(const quest_cache& c, int total_tokens) {
  return (size_t)slots_of(c, total_tokens, kSharedRows) * kv_heads(c) * kSharedRows * (kHeadDim + 2) * sizeof(float);
}

template <bool kTree>
int launch_rows(const quest_cache& c, RowsArgs& a, int total_tokens, const int32_t* topk, void* workspace,
                size_t bytes, const char* who, hipStream_t s) {
  a.slots = (int)slots_of(c, total_tokens, kSharedRows);
  a.splits = splits_of(c, total_tokens);
  const size_t one = split_bytes(c, total_tokens);
  if (workspace == nullptr) bytes = 0;
  a.splits = (int)std::min<size_t>(a.splits, std::max<size_t>(1, bytes / one));
  a.part_acc = (float*)workspace;
  a.part_ml = a.part_acc + (size_t)a.splits * a.slots * a.kv_heads * kSharedRows * kHeadDim;
  const dim3 grid((unsigned)(a.slots * a.splits * a.kv_heads)), block(kSharedWaves * kWave);
  if (a.out_is_fp16)
    hipLaunchKernelGGL((shared_rows_kernel<kTree, false>), grid, block, 0, s, a, a.cu, a.seq_lens, c.page_table, topk, a.mask);
  else
    hipLaunchKernelGGL((shared_rows_kernel<kTree, true>), grid, block, 0, s, a, a.cu, a.seq_lens, c.page_table, topk, a.mask);
  const int r = check_launch(who);
  if (r != QUEST_OK || a.splits == 1) return r;
  hipLaunchKernelGGL(merge_rows_kernel<kSharedRows>, dim3((unsigned)(a.slots * (kSharedRows / 4) * a.kv_heads)), dim3(256), 0, s, a,
                     a.cu);
  return check_launch(who);
}

RowsArgs rows_args(const quest_cache& c, const PackedTokens& p, const void* q, int64_t q_stride, float sm_scale, void* out,
                   int out_is_fp16, float* lse) {
  RowsArgs a = {};
  a.q = (const char*)q;
  a.k_pool = (const char*)c.k_pool;
  a.v_pool = (const char*)c.v_pool;
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
  a.scale_log2 = std::max(std::abs(sm_scale) * kLog2e, 1e-30f);  // scale 0: all weights alike
  return a;
}

}  // namespace

size_t tokens_workspace_bytes(const quest_cache& c, int total_tokens) {
  const int splits = splits_of(c, total_tokens);
  return splits > 1 ? splits * split_bytes(c, total_tokens) : 0;
}

bool rows_fit_a_launch(const quest_cache& c, int total_tokens) {
  return slots_of(c, total_tokens, kSharedRows) * (kSharedRows / 4) * kv_heads(c) <= INT32_MAX;
}

int launch_prompt(const quest_cache& c, const PackedTokens& p, const void* q, int64_t q_stride, float sm_scale, void* out,
                  int out_is_fp16, float* lse, void* workspace, size_t workspace_bytes, hipStream_t s) {
  RowsArgs a = rows_args(c, p, q, q_stride, sm_scale, out, out_is_fp16, lse);
  return launch_rows<false>(c, a, p.total, nullptr, workspace, workspace_bytes, "quest_prompt_attention", s);
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
  return launch_rows<true>(c, a, p.total, topk_idx, workspace, workspace_bytes, "quest_tree_attention", s);
}

}  // namespace quest
