// Attention that cached keys have been given (arXiv 2409.15355, Section 2.5's final block, and the answer's tokens after it): for a
// sequence's query rows (token i, head h of the KV head) and its key t <= p(i)
//   w_t = decay w_t + sum_rows exp(scale <q_row, k_t> - lse_row).
//
// A work item is a range of keys of one KV head, of a group's prefix (for the rows of its sequences, or of some of them, whose weights lie apart)
// or of what a sequence has behind it.  S = Q K^T by v_mfma_f32_32x32x16_bf16 with the keys as columns: a lane owns a key, its
// registers run over the rows, so the sum over rows is a lane's own and is stored as 128 consecutive bytes a half-wave.  A wave's
// keys come straight from the pages into its registers, once; the query rows go round through LDS in tiles of 32, for all waves.
#include "ba_device.h"
#include "ba_lds.h"
#include "ba_long.h"

namespace ba {
namespace {

constexpr int kWThreads = 256;
typedef __attribute__((address_space(3))) float lds_f;
typedef __attribute__((address_space(3))) int32_t lds_i;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4;
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x4_t lds_i32x4;
typedef const __attribute__((address_space(3))) bf16x8_t lds_bf16x8;

__device__ __forceinline__ int clamped_length(const int32_t *seq_len, int cap, int seq) { return max(0, min(seq_len[seq], cap)); }

struct WeightsItem {
  int seq0, n_mem;    // the sequences whose rows it takes
  int table_seq;      // the one whose pages it reads
  int kvh;
  int key0, key_end;  // keys from key0 on, below key_end
  int step;           // how much further on it goes on, if it does
  int part;
};
template <int KEYS, typename Groups>
__device__ __forceinline__ WeightsItem weights_item(const KeyWeightsParams &p, const Groups &groups) {
  WeightsItem it;
  it.part = 0;
  if ((int)blockIdx.x < p.prefix_items) {
    const int id = (int)blockIdx.x;
    int lo = 0, hi = groups.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.item0[mid] <= id) lo = mid; else hi = mid;
    }
    const int rel = id - groups.item0[lo];
    it.seq0 = it.table_seq = groups.seq0[lo];
    it.n_mem = groups.members[lo];
    it.kvh = rel % p.n_kv_heads;
    int chunk = rel / p.n_kv_heads;
    if (it.n_mem > p.item_members) {
      const int parts = (it.n_mem + p.item_members - 1) / p.item_members, first = chunk % parts * p.item_members;
      chunk /= parts;
      it.seq0 += first;
      it.n_mem = min(p.item_members, it.n_mem - first);
    }
    it.key0 = chunk * KEYS;
    it.key_end = groups.prefix[lo];
    it.step = 1 << 30;
  } else {
    int rel = (int)blockIdx.x - p.prefix_items;
    it.kvh = rel % p.n_kv_heads;
    rel /= p.n_kv_heads;
    const int chunk = rel % p.own_chunks;
    rel /= p.own_chunks;
    it.seq0 = it.table_seq = rel % p.n_seqs;
    it.part = rel / p.n_seqs;
    it.n_mem = 1;
    int lo = 0, hi = groups.n;  // its group
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.seq0[mid] <= it.seq0) lo = mid; else hi = mid;
    }
    const bool in = groups.n > 0 && groups.seq0[lo] <= it.seq0 && it.seq0 < groups.seq0[lo] + groups.members[lo];
    it.key0 = (in ? groups.prefix[lo] : 0) + chunk * KEYS;
    it.key_end = clamped_length(p.seq_len, p.cap, it.seq0);
    it.step = p.own_chunks * KEYS;
  }
  return it;
}
// A wave's keys, the B operand: lane = key, chunk 2 kk + half of its row.
template <int D, int NT>
struct WaveKeys {
  int key[NT];
  bool there[NT];
  bf16x8_t frag[NT][D / 16];
  __device__ __forceinline__ void load(const KeyWeightsParams &p, const WeightsItem &it, int key0, int lane) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      key[t] = key0 + t * 32 + (lane & 31);
      const int k = min(key[t], it.key_end - 1), page_at = (int)fast_div((uint32_t)k, p.pages.page_div);
      int page = page_at < p.pages.max_pages ? p.pages.table[it.table_seq * p.pages.stride + page_at] : -1;
      there[t] = page >= 0 && page < p.pages.n_pages;
      page = there[t] ? page : 0;  // (some row that is there: its sums are dropped)
      const char *row = (const char *)(p.k.base + it.kvh * p.k.sh) + ((uint64_t)(uint32_t)page * p.k.page_b16 << 4) +
                        (uint64_t)(uint32_t)(k - page_at * p.pages.page_rows) * p.k.rb + (lane >> 5) * 16;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) frag[t][kk] = *reinterpret_cast<const bf16x8_t *>(row + kk * 32);
    }
  }
};

// Query rows go from memory straight into LDS, two tiles ahead.
constexpr int kRowsTiles = 2, kRowsBuffers = 3;
static_assert(kWThreads / 64 * 32 * kRowsTiles == kWeightsManyKeys && kWThreads / 64 * 32 == kWeightsFewKeys, "what the plan counts with");
// 16 bytes a lane from `from` to LDS bytes [lds_base + 16 lane, +16), as lds_dma16
__device__ __forceinline__ void lds_dma16_lane(const char *from, uint32_t lds_base) {
  lds_base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_base);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds_base) : "memory");
}

// ---- few rows a sequence: 32 keys a wave ----------------------------------------------------------------------------
// A sequence's rows begin at a multiple of 4 (of 8 if it has more than 4): a quad of accumulators is one sequence's, and a tile of rows is
// several's.  32 keys a wave, not 64: those leave registers for five workgroups a compute unit, and what a tile does for its rows -
// notes, masks, the weights of sequences that end in it - goes on in the others while one waits.
// Bound by HBM where it shares a prefix: what every sequence was given before comes in, what it is given now goes out.  64 sequences of four rows on
// 31,744 keys, 8 heads of 128, 64 keys a wave 88 us, 32 keys 60 (149 MB in, 66 out; vector units 39 %, matrix units 14 % of the cycles).  One token
// of one sequence (2,064 keys): a launch, a call takes 4.3 us.
// kEven: without padding, and 32 rows on is the same head, so every tile lies as far from the one before.
template <int D>
struct FewLds {
  static constexpr int kNoted = 16, kNotes = 3 * 32 * 4;  // tiles whose notes lie in LDS at a time; bytes of a tile's
  static constexpr int kBytes = kRowsBuffers * 32 * D * 2 + kNoted * (kNotes + 4);
};
template <int D, bool kFour, bool kEven>
__device__ __forceinline__ void key_weights_few(const KeyWeightsParams &p, const WeightsItem &item, lds_char *const smem, int tid) {
  constexpr int NB = kRowsBuffers;
  constexpr int CPR = D / 8, KCH = D / 16, ROWB = D * 2, LPR = 256 / ROWB, RPI = 1024 / ROWB;  // RPI: rows of a load instruction
  constexpr int OPS = 32 / RPI / (kWThreads / 64);                                             // of a wave and tile
  constexpr uint32_t TB = 32 * ROWB;
  constexpr int kNoted = FewLds<D>::kNoted, kNotes = FewLds<D>::kNotes;
  lds_char *const notes_at = smem + NB * TB;
  lds_i *const all_at = (lds_i *)(notes_at + kNoted * kNotes);
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hf = lane >> 5;
  const int item_last = min(item.key_end, item.key0 + kWeightsFewKeys) - 1;
  const int n_rows = item.n_mem * p.padded, n_tiles = (n_rows + 31) / 32;

  // row r: its sequence, token and head; false: padding (a row that is there in its place)
  auto place = [&](int r, int &j, int &i, int64_t &tok, int &head) __attribute__((always_inline)) {
    const bool there = r < n_rows;
    r = min(r, n_rows - 1);
    j = (int)fast_div((uint32_t)r, p.padded_div);
    const int at = min(r - j * p.padded, p.rows - 1);
    i = (int)fast_div((uint32_t)at, p.group_div);
    tok = (int64_t)(item.seq0 + j) * p.nq + i;
    head = item.kvh * p.group + at - i * p.group;
    return there && r - j * p.padded < p.rows;
  };
  auto where = [&](int u, int tile) __attribute__((always_inline)) {
    const int row = (wave * OPS + u) * RPI + lane / CPR;
    int j, i, head;
    int64_t tok;
    place(tile * 32 + row, j, i, tok, head);
    return (const char *)(p.q + tok * p.q_st + head * p.q_sh) + (((lane % CPR) ^ ((row / LPR) & (CPR - 1))) << 4);
  };
  const char *from_even[OPS];
  const int64_t tile_step = 32 / p.group * p.q_st * 2;
  if constexpr (kEven)
#pragma unroll
    for (int u = 0; u < OPS; ++u) from_even[u] = where(u, 0);
  auto issue = [&](uint32_t to, int tile) __attribute__((always_inline)) {
    const bool whole = kEven && tile * 32 + 32 <= n_rows;  // (the last one may reach beyond the rows)
#pragma unroll
    for (int u = 0; u < OPS; ++u) {
      const char *from;
      if (whole) from = from_even[u], from_even[u] += tile_step;
      else from = where(u, tile);
      lds_dma16_lane(from, (uint32_t)(uintptr_t)smem + to + (wave * OPS + u) * 1024);
    }
  };
  // what the rows of the next kNoted tiles have beside them: -lse in log2 units, the key that each ends before, the sequence's length; whether all
  // keys are old ones, seen by all rows of a tile
  auto note = [&](int tile0) __attribute__((always_inline)) {
#pragma unroll 1
    for (int n = tid; n < min(kNoted, n_tiles - tile0) * 32; n += kWThreads) {
      int j, i, head;
      int64_t tok;
      const bool there = place(tile0 * 32 + n, j, i, tok, head);
      const float lse = p.lse[tok * (p.n_kv_heads * p.group) + head];
      const int len = clamped_length(p.seq_len, p.cap, item.seq0 + j), limit = there && lse != -INFINITY ? len - p.nq + i + 1 : 0;
      lds_char *const to = notes_at + n / 32 * kNotes;
      ((lds_f *)to)[n % 32] = -lse * 1.4426950408889634f;
      ((lds_i *)to)[32 + n % 32] = limit;
      ((lds_i *)to)[64 + n % 32] = len;
      const uint64_t see_all = __builtin_amdgcn_ballot_w64(limit > item_last && len - p.nq > item_last);  // (two tiles to a wave)
      if (n % 32 == 0) all_at[n / 32] = (uint32_t)(see_all >> (lane & 32)) == ~0u;
    }
  };
  issue(0, 0);
  WaveKeys<D, 1> k;
  k.load(p, item, item.key0 + wave * 32, lane);
  const int key = k.key[0];
  note(0);

  const uint32_t q_rd = col * ROWB + ((hf ^ ((col / LPR) & (CPR - 1))) << 4);  // (chunk pairs kk on are an exclusive or away)
  float sum = 0.f;
  int j = 0, left = p.padded;  // (more than 4 rows a sequence: the one that the next eight rows belong to, its rows from there on)
  const int64_t from_seq = p.n_kv_heads * p.w_stride, list = ((int64_t)item.seq0 * p.n_kv_heads + item.kvh) * p.w_stride;
  const int64_t mine = list + key + (kFour ? hf * from_seq : 0);
  const bool stores = key <= item_last && (kFour || hf == 0);
  // which sequences end in a tile, and what they had: asked for a tile ahead (whether it counts is seen later)
  int64_t at[4], next_at[4];  // of their weights, behind `mine`; -1: none ends with these eight rows
  float old[4], next_old[4];
  auto ahead = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      next_at[i] = -1;
      if (tile * 32 + i * 8 < n_rows) {
        if constexpr (kFour) next_at[i] = (tile * 8 + i * 2) * from_seq;
        else if ((left -= 8) == 0) next_at[i] = j++ * from_seq, left = p.padded;
      }
      next_old[i] = 0.f;
      if (p.w_in && next_at[i] >= 0 && stores && (!kFour || tile * 32 + i * 8 + hf * 4 < n_rows)) next_old[i] = (p.w_in + mine)[next_at[i]];
    }
  };
  ahead(0);
  if (n_tiles > 1) issue(TB, 1);
  lds_wait();
  uint32_t buffer = 0;
#pragma unroll 1
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (tile + 1 < n_tiles) dma_wait<OPS>(); else dma_wait<0>();
    wg_barrier();  // the tile is there, and its notes; nobody needs the one before
    if (tile > 0 && tile % kNoted == 0) {
      note(tile);
      lds_wait();
      wg_barrier();
    }
    const uint32_t from = q_rd + buffer;
    buffer = buffer == (NB - 1) * TB ? 0 : buffer + TB;
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = next_at[i], old[i] = next_old[i];
    if (tile + 1 < n_tiles) ahead(tile + 1);
    if (tile + 2 < n_tiles) issue(buffer == (NB - 1) * TB ? 0 : buffer + TB, tile + 2);
    lds_char *const beside = notes_at + tile % kNoted * kNotes;
    f32x16_t s;
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) {
      const f32x16_t zero = {};
      const bf16x8_t qf = *(lds_bf16x8 *)(smem + (from ^ (kk << 5)));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, k.frag[0][kk], kk ? s : zero, 0, 0, 0);
    }
    auto sums = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // this lane's rows: tile * 32 + i * 8 + hf * 4 + (0 .. 3)
        if (decltype(masked)::value && tile * 32 + i * 8 >= n_rows) break;  // (a tile with rows behind the last is masked)
        const f32x4_t nl = *(const lds_f32x4 *)(beside + (i * 8 + hf * 4) * 4);
        i32x4_t limit = {0, 0, 0, 0};
        if constexpr (decltype(masked)::value) limit = *(const lds_i32x4 *)(beside + (32 + i * 8 + hf * 4) * 4);
        float e[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          e[c] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i * 4 + c], p.scale_log2e, nl[c]));
          if constexpr (decltype(masked)::value) e[c] = key < limit[c] ? e[c] : 0.f;
        }
        sum += (e[0] + e[1]) + (e[2] + e[3]);
        if (at[i] >= 0) {
          float total = sum;
          if constexpr (!kFour) total += other_half(total);
          sum = 0.f;
          total = k.there[0] ? total : 0.f;
          if constexpr (decltype(masked)::value) {
            const int len = ((const lds_i *)beside)[64 + i * 8 + (kFour ? hf * 4 : 0)];
            if (stores && key < len && (!kFour || tile * 32 + i * 8 + hf * 4 < n_rows))
              (p.w_out + mine)[at[i]] = __builtin_fmaf(p.decay, key < len - p.nq ? old[i] : 0.f, total);
          } else {
            if (stores) (p.w_out + mine)[at[i]] = __builtin_fmaf(p.decay, old[i], total);
          }
        }
      }
    };
    if (__builtin_amdgcn_readfirstlane(all_at[tile % kNoted]) != 0) sums(std::false_type{});
    else sums(std::true_type{});
  }
}
// kOn: a workgroup goes on with further keys of its sequence.
template <int D, bool kFour, bool kEven, bool kOn, typename Groups>
__global__ __launch_bounds__(kWThreads, 4) void key_weights_kernel(KeyWeightsParams p, Groups groups) {
  __shared__ __attribute__((aligned(1024))) char smem[FewLds<D>::kBytes];
  WeightsItem item = weights_item<kWeightsFewKeys>(p, groups);
  if (item.key0 >= item.key_end) return;
  if constexpr (!kOn) {
    key_weights_few<D, kFour, kEven>(p, item, (lds_char *)smem, threadIdx.x);
  } else {
#pragma unroll 1
    while (true) {
      int tid = threadIdx.x;  // (all is computed again by every pass: kept, it would cost a wave a SIMD)
      asm volatile("" : "+v"(tid), "+s"(item.seq0), "+s"(item.n_mem), "+s"(item.table_seq), "+s"(item.kvh), "+s"(item.key0), "+s"(item.key_end));
      key_weights_few<D, kFour, kEven>(p, item, (lds_char *)smem, tid);
      item.key0 += item.step;
      if (item.key0 >= item.key_end) return;
      wg_barrier();  // (what lies in LDS has been read)
    }
  }
}

// ---- many rows a sequence: 64 keys a wave ---------------------------------------------------------------------------
// A score costs its exponential (half the vector rate), a scaling and an addition.  Bound by vector and matrix units together: 1,024 rows over 32,000
// keys, 8 heads of 128, 80 us (840 TFLOP/s), matrix units 42 %, vector units 56 % of the cycles, and by what the part may draw: a tile's products
// between the exponentials of the one before, two waves a SIMD, take 24 % more cycles and the same time, at 2.26 GHz instead of 1.85.  With 32 keys a
// wave 139: an LDS read a product, not for two.
// kEven: a sequence's rows are whole tiles, and 32 rows on is the same head, so every tile lies as far from the one before.
template <int D, bool kEven, typename Groups>
__global__ __launch_bounds__(kWThreads, kEven ? 4 : 3) void key_weights_many_kernel(KeyWeightsParams p, Groups groups) {
  constexpr int NT = kRowsTiles, NB = kRowsBuffers;
  constexpr int CPR = D / 8, KCH = D / 16, ROWB = D * 2, LPR = 256 / ROWB, RPI = 1024 / ROWB;  // RPI: rows of a load instruction
  constexpr int OPS = 32 / RPI / (kWThreads / 64);                                             // of a wave and tile
  constexpr uint32_t TB = 32 * ROWB;
  constexpr int kNoted = 32, kNotes = 2 * 32 * 4;  // tiles whose notes lie in LDS at a time; bytes of a tile's
  __shared__ __attribute__((aligned(1024))) char smem_generic[NB * TB + kNoted * (kNotes + 4)];
  lds_char *const smem = (lds_char *)smem_generic, *const notes_at = smem + NB * TB;
  lds_i *const all_at = (lds_i *)(notes_at + kNoted * kNotes);
  const WeightsItem item = weights_item<kWeightsManyKeys>(p, groups);
  if (item.key0 >= item.key_end) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hf = lane >> 5;
  const int item_last = min(item.key_end, item.key0 + kWeightsManyKeys) - 1;
  const int per_seq = (p.rows + 31) / 32;  // tiles of a sequence (the last one may end early)
  const int tile_first = item.part * p.part_tiles;
  const int n_tiles = p.part_tiles ? min(p.part_tiles, per_seq - tile_first) : item.n_mem * per_seq;

  // row r of sequence j: its token, its head
  auto place = [&](int j, int r, int64_t &tok, int &head) __attribute__((always_inline)) {
    const int i = (int)fast_div((uint32_t)r, p.group_div);
    tok = (int64_t)(item.seq0 + j) * p.nq + i;
    head = item.kvh * p.group + r - i * p.group;
    return i;
  };
  // (kEven: a tile's first row, the same in all lanes, and how far behind it a lane's piece lies)
  const int64_t tile_step = 32 / p.group * p.q_st * 2;
  const char *from_even = (const char *)(p.q + (int64_t)item.seq0 * p.nq * p.q_st + (int64_t)item.kvh * p.group * p.q_sh) + tile_first * tile_step;
  uint32_t behind[OPS];
  // tile `at` of sequence j: rows at * 32 + (0 .. 31) of it, the last one again behind it (and masked)
  auto where = [&](int u, int j, int at) __attribute__((always_inline)) {
    const int row = (wave * OPS + u) * RPI + lane / CPR;
    int64_t tok;
    int head;
    place(j, min(at * 32 + row, p.rows - 1), tok, head);
    return (const char *)(p.q + tok * p.q_st + head * p.q_sh) + (((lane % CPR) ^ ((row / LPR) & (CPR - 1))) << 4);
  };
  if constexpr (kEven)
#pragma unroll
    for (int u = 0; u < OPS; ++u) {
      const int row = (wave * OPS + u) * RPI + lane / CPR, i = (int)fast_div((uint32_t)row, p.group_div);
      behind[u] = (uint32_t)(i * p.q_st + (row - i * p.group) * p.q_sh) * 2 + (((lane % CPR) ^ ((row / LPR) & (CPR - 1))) << 4);
    }
  int j_in = 0, at_in = tile_first;  // the tile that is asked for next
  auto issue = [&](uint32_t to) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < OPS; ++u) {
      const uint32_t lds = (uint32_t)(uintptr_t)smem + to + (wave * OPS + u) * 1024;
      if constexpr (kEven) lds_dma16(from_even, behind[u], lds);
      else lds_dma16_lane(where(u, j_in, at_in), lds);
    }
    if constexpr (kEven) from_even += tile_step;
    if (++at_in == per_seq) at_in = 0, ++j_in;
  };
  // what the rows of the next kNoted tiles have beside them: -lse in log2 units, the key that each ends before, whether a tile's rows see all keys
  auto note = [&](int tile0) __attribute__((always_inline)) {
#pragma unroll 1
    for (int n = threadIdx.x; n < min(kNoted, n_tiles - tile0) * 32; n += kWThreads) {
      const int tile = tile_first + tile0 + n / 32, j = tile / per_seq, r = (tile - j * per_seq) * 32 + n % 32;
      int64_t tok;
      int head;
      const int i = place(j, min(r, p.rows - 1), tok, head);
      const float lse = p.lse[tok * (p.n_kv_heads * p.group) + head];
      const int limit = r < p.rows && lse != -INFINITY ? clamped_length(p.seq_len, p.cap, item.seq0 + j) - p.nq + i + 1 : 0;
      lds_char *const to = notes_at + n / 32 * kNotes;
      ((lds_f *)to)[n % 32] = -lse * 1.4426950408889634f;
      ((lds_i *)to)[32 + n % 32] = limit;
      const uint64_t see_all = __builtin_amdgcn_ballot_w64(limit > item_last);  // (two tiles to a wave)
      if (n % 32 == 0) all_at[n / 32] = (uint32_t)(see_all >> (lane & 32)) == ~0u;
    }
  };
  issue(0);
  WaveKeys<D, NT> k;
  k.load(p, item, item.key0 + wave * NT * 32, lane);
  const int my_key = item.key0 + wave * NT * 32 + col;
  auto key = [&](int t) __attribute__((always_inline)) { return my_key + t * 32; };
  note(0);
  if (n_tiles > 1) issue(TB);
  lds_wait();

  const uint32_t q_rd = col * ROWB + ((hf ^ ((col / LPR) & (CPR - 1))) << 4);  // (chunk pairs kk on are an exclusive or away)
  float sum[NT] = {};
  int j = 0, at = tile_first;
  uint32_t buffer = 0;
#pragma unroll 1
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (tile + 1 < n_tiles) dma_wait<OPS>(); else dma_wait<0>();
    wg_barrier();  // the tile is there, and its notes; nobody needs the one before
    if (tile > 0 && tile % kNoted == 0) {
      note(tile);
      lds_wait();
      wg_barrier();
    }
    const uint32_t from = q_rd + buffer;
    buffer = buffer == (NB - 1) * TB ? 0 : buffer + TB;
    if (tile + 2 < n_tiles) issue(buffer == (NB - 1) * TB ? 0 : buffer + TB);
    lds_char *const beside = notes_at + tile % kNoted * kNotes;
    f32x16_t s[NT];
    auto q_frag = [&](int kk) __attribute__((always_inline)) { return *(lds_bf16x8 *)(smem + (from ^ (kk << 5))); };
    constexpr int kWin = 2;  // fragments on their way from LDS
    bf16x8_t qf[kWin];
    qf[0] = q_frag(0);
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) {
      const f32x16_t zero = {};
      if (kk + 1 < KCH) qf[(kk + 1) % kWin] = q_frag(kk + 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kk % kWin], k.frag[t][kk], kk ? s[t] : zero, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    auto sums = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // this lane's rows: i * 8 + hf * 4 + (0 .. 3)
        const f32x4_t nl = *(const lds_f32x4 *)(beside + (i * 8 + hf * 4) * 4);
        i32x4_t lim = {0, 0, 0, 0};
        if constexpr (decltype(masked)::value) lim = *(const lds_i32x4 *)(beside + (32 + i * 8 + hf * 4) * 4);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float e[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            e[c] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i * 4 + c], p.scale_log2e, nl[c]));
            if constexpr (decltype(masked)::value) e[c] = key(t) < lim[c] ? e[c] : 0.f;
          }
          sum[t] += (e[0] + e[1]) + (e[2] + e[3]);
        }
        __builtin_amdgcn_sched_barrier(0);  // (as few of them on their way as the registers have room for)
      }
    };
    if (__builtin_amdgcn_readfirstlane(all_at[tile % kNoted]) != 0) sums(std::false_type{});
    else sums(std::true_type{});
    if (++at == per_seq && !p.part_tiles) {
      const int len = clamped_length(p.seq_len, p.cap, item.seq0 + j);
      const int64_t list = ((int64_t)(item.seq0 + j) * p.n_kv_heads + item.kvh) * p.w_stride;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float total = sum[t] + other_half(sum[t]);
        sum[t] = 0.f;
        if (hf == 0 && key(t) <= item_last && key(t) < len) {
          const float old = p.w_in && key(t) < len - p.nq ? p.w_in[list + key(t)] : 0.f;
          p.w_out[list + key(t)] = __builtin_fmaf(p.decay, old, k.there[t] ? total : 0.f);
        }
      }
      at = 0, ++j;
    }
  }
  if (p.part_tiles) {
    const int64_t list = (((int64_t)item.part * p.n_seqs + item.seq0) * p.n_kv_heads + item.kvh) * p.cap;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float total = sum[t] + other_half(sum[t]);
      if (hf == 0 && key(t) <= item_last) p.part[list + key(t)] = k.there[t] ? total : 0.f;
    }
  }
}

// A sequence's parts, added up in their order.
__global__ __launch_bounds__(kWThreads) void key_weights_merge_kernel(KeyWeightsParams p, int chunks) {
  const int list = blockIdx.x / chunks, seq = list / p.n_kv_heads, key = blockIdx.x % chunks * kWThreads + threadIdx.x;
  const int len = clamped_length(p.seq_len, p.cap, seq);
  if (key >= len) return;
  const int64_t at = (int64_t)list * p.w_stride + key, step = (int64_t)p.n_seqs * p.n_kv_heads * p.cap;
  const float old = p.w_in && key < len - p.nq ? p.w_in[at] : 0.f;
  const float *from = p.part + (int64_t)list * p.cap + key;
  float sum = 0.f;
#pragma unroll 8
  for (int i = 0; i < p.row_parts; ++i) sum += from[i * step];
  p.w_out[at] = __builtin_fmaf(p.decay, old, sum);
}

template <int D, typename Groups>
hipError_t launch_d(const KeyWeightsParams &p, const Groups &g, bool many, hipStream_t stream) {
  const int64_t items = p.prefix_items + (int64_t)p.n_seqs * p.n_kv_heads * p.own_chunks * p.row_parts;
  if (items < 1 || items > kMaxWorkgroups) return hipErrorInvalidValue;
  // (a tile's rows in 32 bits behind the first)
  const bool near = (32 / p.group + 1) * p.q_st + p.group * p.q_sh < ((int64_t)1 << 30);
  if (many && p.rows % 32 == 0 && 32 % p.group == 0 && near) key_weights_many_kernel<D, true, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
  else if (many) key_weights_many_kernel<D, false, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
  else {
    auto launch = [&](auto four, auto even) {
      if (p.own_go_on) key_weights_kernel<D, decltype(four)::value, decltype(even)::value, true, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
      else key_weights_kernel<D, decltype(four)::value, decltype(even)::value, false, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
    };
    const bool even = p.rows == p.padded && 32 % p.group == 0;
    if (p.padded == 4) even ? launch(std::true_type{}, std::true_type{}) : launch(std::true_type{}, std::false_type{});
    else even ? launch(std::false_type{}, std::true_type{}) : launch(std::false_type{}, std::false_type{});
  }
  return hipGetLastError();
}

}  // namespace

template <typename Groups>
hipError_t launch_key_weights(const KeyWeightsParams &p, const Groups &g, int head_dim, bool many, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(p, g, many, stream) : launch_d<64>(p, g, many, stream);
}
hipError_t launch_key_weights_merge(const KeyWeightsParams &p, hipStream_t stream) {
  const int64_t chunks = ((int64_t)p.cap + kWThreads - 1) / kWThreads, wgs = (int64_t)p.n_seqs * p.n_kv_heads * chunks;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  key_weights_merge_kernel<<<(unsigned)wgs, kWThreads, 0, stream>>>(p, (int)chunks);
  return hipGetLastError();
}
template hipError_t launch_key_weights(const KeyWeightsParams &, const PagedGroups &, int, bool, hipStream_t);
template hipError_t launch_key_weights(const KeyWeightsParams &, const PagedGroupsSmall &, int, bool, hipStream_t);

}  // namespace ba
