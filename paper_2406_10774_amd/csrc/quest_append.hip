// Insertion of many tokens a sequence into the paged cache: a prompt, the next part of one, accepted drafts.
//
// Keys and values go to their slots, and every page that receives a token gets its channel-wise minimum
// and maximum, folded with what the entry holds where the page had tokens before (the insertion half of
// Algorithm 1 of arXiv 2406.10774, a page at a time: order_key2 makes the result independent of how).
//
// Bound by memory: each byte of a new token is read once and written once, metadata from registers.  A wave
// has one (page, head); the waves of a work-group have adjacent heads, whose 256-byte rows are adjacent in the
// packed arrays and whose blocks are adjacent in the pools.  32749 tokens of 32 heads: 1.1 GB in 197 us, 5.6 TB/s
// (a large copy: 4.9).  A few tokens of 16 sequences: 4.1 us, lengths -> page and row -> data -> store.
//
// Without any length on the host: the pages of sequence b start at unit floor(cu[b] / S) + 2 b, which leaves
// room for the floor((n + S - 2) / S) + 1 pages that n >= 1 tokens can touch.
#include "quest_common.h"

namespace quest {

namespace {

constexpr int kAppendWaves = 4;

template <int kS>
__global__ __launch_bounds__(kAppendWaves* kWave) void append_tokens_kernel(
    char* __restrict__ k_pool, char* __restrict__ v_pool, char* __restrict__ meta,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ cu,
    const int32_t* __restrict__ rows, const char* __restrict__ k_new, const char* __restrict__ v_new,
    int64_t new_stride, int batch, int num_heads, int max_pages, int64_t num_phys_pages, int64_t waves) {
  constexpr int kLoads = kS < 16 ? kS / 4 : 4;  // wave-wide loads of four tokens each at a time
  const int lane = lane_id();
  const int64_t at = (int64_t)blockIdx.x * kAppendWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= waves) return;
  const int unit = (int)(at / num_heads);
  const int head = (int)(at - (int64_t)unit * num_heads);
  int b = -1;
  for (int base = 0; base < batch; base += kWave) {  // the last sequence that starts at or before the unit
    const int i = base + lane;
    const bool before = i < batch && cu[i < batch ? i : 0] / kS + 2 * i <= unit;
    const int n = __popcll(__ballot(before));
    b += n;
    if (n < kWave) break;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int first_row = cu[b];
  const int tokens = cu[b + 1] - first_row;
  const int seq_len = seq_lens[b];
  const int first = seq_len - tokens;                              // position of the first new token
  const int page = first / kS + unit - (first_row / kS + 2 * b);
  if (tokens <= 0 || first < 0 || page > (seq_len - 1) / kS || page >= max_pages) return;   // (no page behind the row)
  const int from = max(first - page * kS, 0), to = min(seq_len - page * kS, kS);   // the page's new slots
  const int phys = page_table[(size_t)b * max_pages + page];
  const size_t block = ((size_t)phys * num_heads + head) * (kS * kRowBytes);
  const int sub = lane >> 4, chunk = lane & 15;

  uint4 mn = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
  uint4 mx = make_uint4(0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u);
#pragma unroll 1
  for (int s0 = 0; s0 < kS; s0 += 4 * kLoads) {
    if (s0 + 4 * kLoads <= from || s0 >= to) continue;
    uint4 k[kLoads], v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = s0 + 4 * i + sub;
      const bool here = slot >= from && slot < to;
      int row = first_row + (here ? page * kS + slot - first : 0);
      if (rows != nullptr) row = rows[row];
      const int64_t off = row * new_stride + head * kRowBytes + chunk * 16;
      k[i] = ld16_stream(k_new + off);
      v[i] = ld16_stream(v_new + off);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = s0 + 4 * i + sub;
      if (slot >= from && slot < to) {
        const size_t off = block + (size_t)slot * kRowBytes + chunk * 16;
        st16(k_pool + off, k[i]);
        st16(v_pool + off, v[i]);
        const uint4 key = order_key8(k[i]);
        mn = key_min8(mn, key);
        mx = key_max8(mx, key);
      }
    }
  }
  mn = rows_key_min8(mn);
  mx = rows_key_max8(mx);
  if (lane < 32) {
    char* entry = meta + meta_offset(num_phys_pages, phys, head) + lane * 16;
    uint4 mine = sub == 0 ? mn : mx;
    if (from > 0) {
      const uint4 old = order_key8(ld16(entry));
      mine = sub == 0 ? key_min8(mine, old) : key_max8(mine, old);
    }
    st16(entry, order_key8(mine));
  }
}

template <int kS>
int launch_append_tokens_for(const quest_cache& c, const PackedTokens& p, const void* k_new, const void* v_new,
                             int64_t new_stride, const int32_t* rows, hipStream_t s) {
  const int64_t waves = ((int64_t)p.total / kS + 2 * (int64_t)c.batch) * kv_heads(c);
  hipLaunchKernelGGL(append_tokens_kernel<kS>, dim3((unsigned)((waves + kAppendWaves - 1) / kAppendWaves)),
                     dim3(kAppendWaves * kWave), 0, s, (char*)c.k_pool, (char*)c.v_pool, (char*)c.meta, c.page_table,
                     c.seq_lens, p.cu, rows, (const char*)k_new, (const char*)v_new, new_stride * 2, c.batch,
                     kv_heads(c), c.max_pages_per_seq, c.num_phys_pages, waves);
  return check_launch("quest_append_tokens");
}

}  // namespace

int launch_append_tokens(const quest_cache& c, const PackedTokens& p, const void* k_new, const void* v_new,
                         int64_t new_stride, const int32_t* rows, hipStream_t s) {
  switch (c.page_size) {
    case 8: return launch_append_tokens_for<8>(c, p, k_new, v_new, new_stride, rows, s);
    case 32: return launch_append_tokens_for<32>(c, p, k_new, v_new, new_stride, rows, s);
    case 64: return launch_append_tokens_for<64>(c, p, k_new, v_new, new_stride, rows, s);
    default: return launch_append_tokens_for<16>(c, p, k_new, v_new, new_stride, rows, s);
  }
}

}  // namespace quest
