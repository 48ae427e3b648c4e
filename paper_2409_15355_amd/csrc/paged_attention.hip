// Attention of one or a few query tokens of many sequences over the pages of a key/value cache, where groups of
// sequences begin with the same pages (arXiv 2409.15355, Section 2.5's final block, token by token: many questions over one set of
// passages).  For token t at position pos(t), head h: o = sum_{s <= pos} softmax_s(scale <q, k_s>) v_s.
//
// A work item is a tile of packed rows (row = token * G + head in group) of one KV head over a range of keys:
//   - of a group's prefix, for the rows of all its sequences: its keys are read once for all of them;
//   - of what a sequence has behind the prefix, for its own rows.
// Every item leaves, per row, its output, reference and sum; paged_merge_kernel adds a row's parts up in their order.
//
// Two walks, by the item's rows:
//   - up to kPagedStreamRows rows, bound by the stream of keys and values: the four waves of a workgroup take tiles of 16 keys in turn,
//     each through LDS of its own and without a barrier, 16 rows an MFMA (v_mfma_f32_16x16x32_bf16 for S^T = K Q^T, 16x16x16 for
//     O^T = V^T P^T), and add their sums up at the end;
//   - beyond, bound by the products: the waves take 32 rows each (v_mfma_f32_32x32x16_bf16) of 128 and share tiles of 32 keys.
// Two workgroups a compute unit either way.  Keys and values come from the pages straight into LDS; the item's part of the page table lies
// in LDS.  Tiles begin at multiples of 16 keys, so where a page's rows are a multiple of 16 a load instruction's rows are all of one page and
// its address is a scalar (kAligned); otherwise every lane looks its own row's page up.
// The exponentials come out as the operand of the second product.  Scores, softmax and sums in 32 bits; P is rounded to bf16 for the
// second product (the format of V), parts between the launches to fp16 (see row_end).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "ba_device.h"
#include "ba_lds.h"
#include "ba_paged.h"

namespace ba {
namespace {

constexpr int kPWaves = 4;
constexpr int kPThreads = kPWaves * 64;
constexpr float kRebaseAbove = 1099511627776.0f;  // 2^40: a lane's sum over a tile beyond this moves the row's reference
constexpr int kTilesB = 65536;                    // LDS of the tiles, then the page table's part

template <int D>
struct PGeo {
  static constexpr int CPR = D / 8;        // 16-byte chunks per row
  static constexpr int ROWB = D * 2;       // bytes per K/V row in LDS
  static constexpr int LPR = 256 / ROWB;   // rows per 256-byte LDS line
  static constexpr int RPI = 1024 / ROWB;  // rows filled by one LDS-direct wave instruction
};
typedef __attribute__((address_space(3))) int32_t lds_int;
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
typedef const __attribute__((address_space(3))) bf16x8_t lds_bf16x8;

// lds_dma16, kPast: past the caches; and with an address per lane (rows of different pages)
template <bool kPast>
__device__ __forceinline__ void lds_dma16_page(const char *base, uint32_t offset, uint32_t lds_base) {
  if constexpr (!kPast) {
    lds_dma16(base, offset, lds_base);
  } else {
    const uint64_t b = (uint64_t)base;
    const uint64_t bu = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) << 32) |
                        (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b);
    lds_base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_base);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(offset), "s"(bu), "s"(lds_base) : "memory");
  }
}
template <bool kPast>
__device__ __forceinline__ void lds_dma16_from(const char *from, uint32_t lds_base) {
  lds_base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_base);
  if constexpr (kPast)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(from), "s"(lds_base) : "memory");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds_base) : "memory");
}
// value held by lane ^ 16
__device__ __forceinline__ float other_sixteen(float x) {
  const uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return (threadIdx.x & 16) ? __uint_as_float(r[0]) : __uint_as_float(r[1]);
}

// index of the group that sequence `seq` belongs to, or -1
template <typename Groups>
__device__ __forceinline__ int group_of(const Groups &g, int seq) {
  int lo = 0, hi = g.n;  // the last group that begins at or before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (g.seq0[mid] <= seq) lo = mid; else hi = mid;
  }
  return g.n > 0 && g.seq0[lo] <= seq && seq < g.seq0[lo] + g.members[lo] ? lo : -1;
}
__device__ __forceinline__ int length_of(const PagedAttnParams &p, int seq) { return max(0, min(p.seq_len[seq], p.cap)); }

struct PagedItem {
  int seq0;           // its rows are those of the sequences from this one on; its pages this one's
  int n_rows, row0;   // rows of the problem, first row of the tile
  int kvh, part;
  int k_lo, k0, k1;   // keys [k_lo, k1), tiles from k0 (a multiple of 16) on
  int page0;          // first entry of the page table in LDS
  bool holes;         // some pages are not there
};
// Row r of an item's problem.
struct PagedRow {
  int64_t tok;
  int head;
  int limit;  // it sees the item's keys below this
};
__device__ __forceinline__ PagedRow paged_row(const PagedAttnParams &p, const PagedItem &it, int r) {
  PagedRow w;
  const int tok = (int)fast_div((uint32_t)r, p.group_div), seq = (int)fast_div((uint32_t)tok, p.nq_div);
  w.tok = (int64_t)it.seq0 * p.nq + tok;
  w.head = it.kvh * p.group + r - tok * p.group;
  w.limit = min(it.k1, length_of(p, it.seq0 + seq) - p.nq + (tok - seq * p.nq) + 1);
  return w;
}
// Pages that a list names, ascending: what the walk takes for a sequence is the listed pages one after the other.
struct SelectedItem : PagedItem {
  lds_char *list;  // numbers of the item's pages within the sequence
  int n_list;
};
// (the tokens that a row sees are the first ones of that sequence, too: those of the pages before the one its last token is in, and
// what it sees of that one)
__device__ __forceinline__ PagedRow paged_row(const PagedAttnParams &p, const SelectedItem &it, int r) {
  PagedRow w = paged_row(p, static_cast<const PagedItem &>(it), r);
  const int tok = (int)fast_div((uint32_t)r, p.group_div), seq = (int)fast_div((uint32_t)tok, p.nq_div);
  const int limit = max(0, length_of(p, it.seq0 + seq) - p.nq + (tok - seq * p.nq) + 1);
  const int page = (int)fast_div((uint32_t)limit, p.page_div);
  const lds_int *const list = (const lds_int *)it.list;
  w.limit = 0;
  if (it.n_list <= 0) return w;
  int lo = 0, hi = it.n_list;  // the first that is not before it
  if (list[hi - 1] < page) lo = hi;
  while (hi > lo) {
    const int mid = (lo + hi) >> 1;
    if (list[mid] < page) lo = mid + 1; else hi = mid;
  }
  const int64_t keys = (int64_t)(it.page0 + lo) * p.page_rows + (lo < it.n_list && list[lo] == page ? limit - page * p.page_rows : 0);
  w.limit = lo == it.n_list ? it.k1 : (int)(keys < it.k1 ? keys : it.k1);
  return w;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = min(x, __shfl_xor(x, m));
  return __builtin_amdgcn_readfirstlane(x);
}

// Where rows of the item's keys lie, and the loads of a run of them that does not cross a multiple of 16: wave instructions of RPI rows
// each, lane l fetching one chunk of row l / CPR.
template <int D, bool kAligned>
struct PagedSource {
  using G = PGeo<D>;
  const PagedAttnParams &p;
  const PagedItem &it;
  lds_char *table;
  const char *k, *v;
  __device__ __forceinline__ PagedSource(const PagedAttnParams &p_, const PagedItem &it_, lds_char *table_)
      : p(p_), it(it_), table(table_), k((const char *)(p_.k + it_.kvh * p_.k_sh)), v((const char *)(p_.v + it_.kvh * p_.v_sh)) {}
  // the page of a key, -1: not there
  __device__ __forceinline__ int page_of(int key, int &row) const {
    const int i = (int)fast_div((uint32_t)key, p.page_div);
    row = key - i * p.page_rows;
    return ((const lds_int *)table)[i - it.page0];
  }
  // where a row of page `page` lies behind page 0's
  static __device__ __forceinline__ uint64_t behind(int page, uint32_t page_b16, int row, uint32_t rb) {
    return ((uint64_t)(uint32_t)page * page_b16 << 4) + (uint64_t)(uint32_t)row * rb;
  }
  // Where the rows from a key on lie: asked for ahead of the loads, which would wait for LDS otherwise.
  struct Run {
    int key, page, row;
  };
  __device__ __forceinline__ Run run_at(int key) const {
    Run r = {key, 0, 0};
    if constexpr (kAligned) {
      // (rows behind the item's last lie in the same page, whole blocks of 16 behind it are its last block once more; pages that are
      // not there: page 0.  All of them are masked)
      key = __builtin_amdgcn_readfirstlane(key);
      r.page = page_of(min(key & ~15, (it.k1 - 1) & ~15) | (key & 15), r.row);
    }
    return r;
  }
  // N wave instructions of keys and of values, a run's rows; chunks(u, &kchunk, &vchunk): what this lane fetches of its row in the u-th
  template <int N, typename Chunks>
  __device__ __forceinline__ void fetch(const Run &run, int lane_row, uint32_t k_to, uint32_t v_to, Chunks &&chunks) const {
    if (p.past_caches) fetch_p<N, true>(run, lane_row, k_to, v_to, chunks);
    else fetch_p<N, false>(run, lane_row, k_to, v_to, chunks);
  }
  template <int N, bool kPast, typename Chunks>
  __device__ __forceinline__ void fetch_p(const Run &run, int lane_row, uint32_t k_to, uint32_t v_to, Chunks &&chunks) const {
    if constexpr (kAligned) {
      const int page = max(0, __builtin_amdgcn_readfirstlane(run.page));
      const char *k0 = k + behind(page, p.k_page_b16, run.row, p.k_rb), *v0 = v + behind(page, p.v_page_b16, run.row, p.v_rb);
#pragma unroll
      for (int u = 0; u < N; ++u) {
        uint32_t kc, vc;
        chunks(u, kc, vc);
        lds_dma16_page<kPast>(k0, (uint32_t)(u * G::RPI + lane_row) * p.k_rb + kc, k_to + u * 1024);
        lds_dma16_page<kPast>(v0, (uint32_t)(u * G::RPI + lane_row) * p.v_rb + vc, v_to + u * 1024);
      }
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) {
        uint32_t kc, vc;
        chunks(u, kc, vc);
        int row;
        const int page = max(0, page_of(min(run.key + u * G::RPI + lane_row, it.k1 - 1), row));
        lds_dma16_from<kPast>(k + behind(page, p.k_page_b16, row, p.k_rb) + kc, k_to + u * 1024);
        lds_dma16_from<kPast>(v + behind(page, p.v_page_b16, row, p.v_rb) + vc, v_to + u * 1024);
      }
    }
  }
  // bit i: key + i is one of the item's, and its page is there
  template <int N>
  __device__ __forceinline__ uint32_t there(int key, int lane) const {
    const int at = key + (lane & (N - 1));
    int row;
    const bool ok = at >= it.k_lo && at < it.k1 && (!it.holes || page_of(max(it.k_lo, min(at, it.k1 - 1)), row) >= 0);
    return (uint32_t)__builtin_amdgcn_ballot_w64(ok) & (N == 32 ? ~0u : (1u << (N & 31)) - 1u);
  }
};
__device__ __forceinline__ uint32_t below(int lim) { return lim <= 0 ? 0u : lim >= 32 ? ~0u : (1u << lim) - 1u; }

// A row's result: E consecutive dimensions of it at a time, of D.  top: the largest finite size among all D of o.
// Parts are kept as fp16, divided by their sum and by a power of two that brings the largest into [2^13, 2^14): an element of a part is off by
// 2^-11 of itself, or 2^-38 of the part's largest where that is more; the result by 2^-11 of sum p |v|, a quarter of what rounding P to bf16
// may take.  Half the memory traffic of 32 bits (64 sequences over 31,744 shared keys, 32 over 8 heads of 128: 33 MB out and in
// again, of 130 MB of keys and values).
struct RowEnd {
  float m, l, inv, mult, scale;
};
// (An infinity or a NaN in one dimension stays what it is, and the others keep their power of two.)
__device__ __forceinline__ float finite_size(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
__device__ __forceinline__ RowEnd row_end(const PagedAttnParams &p, float m, float l, float top) {
  RowEnd e = {m, l, l == 0.f ? 0.f : 1.f / l, 1.f, 1.f};
  if (!p.direct) {
    const int exp = max(-100, __builtin_amdgcn_frexp_expf(top * e.inv));
    e.mult = e.inv * __builtin_ldexpf(1.f, 14 - exp);
    e.scale = __builtin_ldexpf(1.f, exp - 14);
  }
  return e;
}
template <int D, int E>
__device__ __forceinline__ void write_row(const PagedAttnParams &p, const PagedItem &it, const PagedRow &r, const RowEnd &end, int d, const float *o,
                                          bool first) {
  const int64_t row = r.tok * (p.n_kv_heads * p.group) + r.head;
  if (p.direct) {
    uint16_t *to = p.o + r.tok * p.o_st + r.head * p.o_sh + d;
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<u32x2_t *>(to + e) =
          u32x2_t{pack_bf16(o[e] * end.inv, o[e + 1] * end.inv), pack_bf16(o[e + 2] * end.inv, o[e + 3] * end.inv)};
    if (p.lse && first) p.lse[row] = end.l == 0.f ? -INFINITY : (end.m + __builtin_amdgcn_logf(end.l)) * 0.6931471805599453f;
  } else {
    const int64_t at = it.part * p.part_rows + row;
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<u32x2_t *>(p.part_o + at * D + d + e) =
          u32x2_t{pack_f16(o[e] * end.mult, o[e + 1] * end.mult), pack_f16(o[e + 2] * end.mult, o[e + 3] * end.mult)};
    if (first) *reinterpret_cast<f32x4_t *>(p.part_ml + at * 4) = f32x4_t{end.l == 0.f ? -INFINITY : end.m, end.l, end.scale, 0.f};
  }
}
// the largest of each run of 16 lanes, in every lane of the run
__device__ __forceinline__ float max_over_sixteen(float x) {
  auto with = [&](auto ctrl) __attribute__((always_inline)) {
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)));
  };
  with(std::integral_constant<int, 0xb1>{});   // (as sum_over_lanes)
  with(std::integral_constant<int, 0x4e>{});
  with(std::integral_constant<int, 0x141>{});
  with(std::integral_constant<int, 0x140>{});
  return x;
}

// ---- few rows: RG groups of 16 ------------------------------------------------------------------------------------------
// Bound by memory: two products of G * tokens rows a key, 16 KB of tiles in flight a wave and 128 a compute unit.  A barrier a tile would
// tie the waves' loads together; they meet only at the end.  32 over 8 heads of 128: 128 sequences of up to 8,000 keys, 1.98 GB, 324 us,
// 6.1 TB/s; 1 of 2,064 keys 6.5 us, of them launch 2.4, the page table 0.8, keys and products 1.8, the end 1.6.
// stage(): puts the item's part of the page table into LDS (the rows are asked for first, and arrive meanwhile)
template <int D, bool kAligned, int RG, typename Item, typename Stage>
__device__ __forceinline__ void walk_stream(const PagedAttnParams &p, Item &it, lds_char *smem, int lane, int wave, Stage &&stage) {
  using G = PGeo<D>;
  constexpr int KK = D / 32, DS = D / 16;
  constexpr uint32_t TB = 16 * G::ROWB;              // a tile of keys, then one of values
  constexpr int NB = kTilesB / kPWaves / (2 * TB);   // tiles of a wave in LDS
  constexpr int OPS = 16 / G::RPI;                   // load instructions per tile and kind
  const PagedSource<D, kAligned> src(p, it, smem + kTilesB);
  const int col = lane & 15, quad = lane >> 4;
  const int n_tiles = (it.k1 - it.k0 + 15) / 16;
  const int n = n_tiles > wave ? (n_tiles - wave + kPWaves - 1) / kPWaves : 0;  // this wave's: wave, wave + 4, ...
  const uint32_t ring = wave * (NB * 2 * TB);

  auto run_of = [&](int i) __attribute__((always_inline)) { return src.run_at(it.k0 + (wave + i * kPWaves) * 16); };
  auto issue = [&](int i, const auto &run) __attribute__((always_inline)) {
    const uint32_t to = (uint32_t)(uintptr_t)smem + ring + (uint32_t)(i % NB) * (2 * TB);
    int ln = lane;
    src.template fetch<OPS>(run, ln / G::CPR, to, to + TB, [&](int u, uint32_t &kchunk, uint32_t &vchunk) __attribute__((always_inline)) {
      const int line = (u * G::RPI + ln / G::CPR) / G::LPR, pos = ln % G::CPR;
      kchunk = (uint32_t)(pos ^ (line & (G::CPR - 1))) << 4;
      vchunk = (uint32_t)((((pos >> 1) ^ (line & (G::CPR / 2 - 1))) << 1) | (pos & 1)) << 4;
    });
  };
  bf16x8_t qf[RG][KK];
  int limit[RG], least = 0x7fffffff;
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    const PagedRow r = paged_row(p, it, min(it.row0 + g * 16 + col, it.n_rows - 1));
    limit[g] = r.limit;
    least = min(least, r.limit);
    const uint16_t *row = p.q + r.tok * p.q_st + r.head * p.q_sh + quad * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[g][kk] = *reinterpret_cast<const bf16x8_t *>(row + kk * 32);
  }
  stage();
#pragma unroll
  for (int g = 0; g < RG; ++g)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[g][kk]));  // (waited for here, not inside the loop)
#pragma unroll 1
  for (int i = 0; i < min(n, NB); ++i) issue(i, run_of(i));
  least = wave_min(least);

  uint32_t k_rd[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) k_rd[kk] = ring + col * G::ROWB + (((kk * 4 + quad) ^ ((col / G::LPR) & (G::CPR - 1))) << 4);
  const int v_row = quad * 4 + (col >> 2), v_swz = (v_row / G::LPR) & (G::CPR / 2 - 1);
  const uint32_t v_rd = ring + TB + v_row * G::ROWB + (lane & 3) * 8;
  f32x4_t o[RG][DS];
  float mb[RG], l[RG];
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    mb[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) o[g][ds] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const uint32_t buf = (uint32_t)(i % NB) * (2 * TB);
    const int newer = min(NB, n - i) - 1;  // tiles on their way behind this one
    if (newer == 0) dma_wait<0>();
    else if (NB == 2 || newer == 1) dma_wait<2 * OPS>();
    else if (newer == 2) dma_wait<4 * OPS>();
    else dma_wait<6 * OPS>();
    const int key0 = it.k0 + (wave + i * kPWaves) * 16;
    const auto ahead = run_of(i + NB);
    bf16x8_t kf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kf[kk] = *(lds_bf16x8 *)(smem + (k_rd[kk] + buf));
    s16x4_t vf[DS];
    uint32_t swz = v_swz;
    auto v_frag = [&](int ds) __attribute__((always_inline)) {
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(smem + (v_rd + buf + ((ds ^ swz) << 5))));
    };
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) vf[ds] = v_frag(ds);
    const bool masked = it.holes || key0 < it.k_lo || key0 + 16 > least;
    const uint32_t there = masked ? src.template there<16>(key0, lane) : 0xffffu;
    // the tile is in registers: its place takes the one that is NB further on
    lds_wait();
    if (i + NB < n) issue(i + NB, ahead);
    // A masked probability is zero, but zero times an infinity or a NaN is not: values of keys that a row does not see must
    // not reach its sums, and are set to zero.
    bool apart = false;  // the rows see different keys of the tile
    if (masked) {
      const int lim0 = __builtin_amdgcn_readfirstlane(limit[0] - key0);
#pragma unroll
      for (int g = 0; g < RG; ++g) apart |= __builtin_amdgcn_ballot_w64(below(limit[g] - key0) != below(lim0)) != 0;
      const uint32_t seen = (apart ? there : there & below(lim0)) >> (quad * 4);
      const u32x2_t keep = {(seen & 1 ? 0xffffu : 0u) | (seen & 2 ? 0xffff0000u : 0u), (seen & 4 ? 0xffffu : 0u) | (seen & 8 ? 0xffff0000u : 0u)};
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) vf[ds] = __builtin_bit_cast(s16x4_t, __builtin_bit_cast(u32x2_t, vf[ds]) & keep);
    }
#pragma unroll
    for (int g = 0; g < RG; ++g) {
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kk], qf[g][kk], s, 0, 0, 0);
      const int lim = limit[g] - key0;
      if (masked) {
        const uint32_t mine = (there & below(lim)) >> (quad * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!((mine >> e) & 1)) s[e] = -INFINITY;
      }
      // the reference: the row's maximum in the first tile of which it sees a key, raised where an exponential threatens to overflow
      auto row_max = [&]() __attribute__((always_inline)) {
        float m = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        m = fmaxf(m, other_sixteen(m));
        return fmaxf(m, other_half(m)) * p.scale_log2e;
      };
      if (__builtin_amdgcn_ballot_w64(mb[g] == -INFINITY) != 0) {
        const float m = row_max();
        if (mb[g] == -INFINITY) mb[g] = m;
      }
      float e4[4], sum;
      auto exponentials = [&]() __attribute__((always_inline)) {
        const float ref = mb[g] == -INFINITY ? 0.f : mb[g];
#pragma unroll
        for (int e = 0; e < 4; ++e) e4[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], p.scale_log2e, -ref));
        sum = (e4[0] + e4[1]) + (e4[2] + e4[3]);
      };
      exponentials();
      const uint64_t above = __builtin_amdgcn_ballot_w64(!(sum < kRebaseAbove));
      if (above != 0) {
        // (the rows of these lanes and no others: what another row's scores are changes no bit of this one)
        const uint32_t rows = (uint32_t)above | (uint32_t)(above >> 32);
        const float m = ((rows | rows >> 16) >> col) & 1 ? fmaxf(row_max(), mb[g]) : mb[g];
        const float alpha = m == mb[g] ? 1.f : __builtin_amdgcn_exp2f(mb[g] - m);
        mb[g] = m;
        l[g] *= alpha;
#pragma unroll
        for (int ds = 0; ds < DS; ++ds)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[g][ds][e] *= alpha;
        exponentials();
      }
      l[g] += sum;
      const u32x2_t w = {pack_bf16(e4[0], e4[1]), pack_bf16(e4[2], e4[3])};
      const s16x4_t pf = __builtin_bit_cast(s16x4_t, w);
      if (!apart) {
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) o[g][ds] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf[ds], pf, o[g][ds], 0, 0, 0);
      } else {
        // the rows that see the same keys go together
        uint64_t left = ~0ull;
#pragma unroll 1
        while (left) {
          const int their_lim = __builtin_amdgcn_readlane(lim, __builtin_ctzll(left));
          const bool mine = lim == their_lim;
          left &= ~__builtin_amdgcn_ballot_w64(mine);
          const uint32_t seen = below(their_lim) >> (quad * 4);
          if (their_lim <= 0) continue;
          const u32x2_t keep = {(seen & 1 ? 0xffffu : 0u) | (seen & 2 ? 0xffff0000u : 0u), (seen & 4 ? 0xffffu : 0u) | (seen & 8 ? 0xffff0000u : 0u)};
#pragma unroll
          for (int ds = 0; ds < DS; ++ds) {
            const s16x4_t f = __builtin_bit_cast(s16x4_t, __builtin_bit_cast(u32x2_t, vf[ds]) & keep);
            const f32x4_t add = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(f, pf, f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][ds][e] += mine ? add[e] : 0.f;
          }
        }
      }
    }
  }

  // ---- the waves' sums, 16 rows at a time ----------------------------------------------------------------------
  constexpr int OST = D + 4;  // (floats from row to row: 16 bytes on, off the last one's banks)
  static_assert((size_t)kPWaves * 16 * (OST + 2) * 4 <= kTilesB, "the waves' sums fit the tiles' place");
  lds_float *const os = (lds_float *)smem, *const mls = os + kPWaves * 16 * OST;
  constexpr int E = D / 16;
  const int tid = wave * 64 + lane, row = tid / 16, d = tid % 16 * E;
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    if (it.row0 + g * 16 >= it.n_rows) break;
    __syncthreads();  // (everybody is done with the tiles, or with the rows before)
    float lt = l[g] + other_sixteen(l[g]);
    lt += other_half(lt);
    if (quad == 0) {
      mls[(wave * 16 + col) * 2] = lt == 0.f ? -INFINITY : mb[g];
      mls[(wave * 16 + col) * 2 + 1] = lt;
    }
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) *(lds_f32x4 *)(os + (wave * 16 + col) * OST + ds * 16 + quad * 4) = o[g][ds];
    __syncthreads();
    float m = -INFINITY, lsum = 0.f, acc[E];
#pragma unroll
    for (int w = 0; w < kPWaves; ++w) m = fmaxf(m, mls[(w * 16 + row) * 2]);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kPWaves; ++w) {
      const float lw = mls[(w * 16 + row) * 2 + 1];
      const float f = lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mls[(w * 16 + row) * 2] - m);
      lsum += lw * f;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const f32x4_t x = *(const lds_f32x4 *)(os + (w * 16 + row) * OST + d + e);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[e + c] += lw == 0.f ? 0.f : x[c] * f;
      }
    }
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, finite_size(acc[e]));
    const RowEnd end = row_end(p, m, lsum, max_over_sixteen(top));
    const int r = it.row0 + g * 16 + row;
    if (r < it.n_rows) write_row<D, E>(p, it, paged_row(p, it, r), end, d, acc, d == 0);
  }
}

// ---- many rows: 32 a wave, tiles of 32 keys shared by the four -----------------------------------------------------------
// A key is read from memory once for 128 rows, and from LDS once for 32.  32 over 8 heads of 128, 64 sequences on 31,744 keys: 33.4 GFLOP in
// 58.7 us, 570 TFLOP/s.  The matrix units are busy for 17 of them, vector instructions take 21 and LDS reads 9 (counters): what it waits for is a
// wave's own chain (the tile behind a barrier, the softmax between two products), of which two waves a SIMD cover each other's only
// in part.  Three workgroups a compute unit need 168 registers and 48 KB: 512 rows 87 us against 91, but 256 rows 58.5 against 51.9; eight
// waves that take turns at the matrix units, with 64 keys a tile, and with the sequences' own items among theirs: 58.4 against 58.2.
// The next tile's score products between this one's exponentials: no change.
template <int D, bool kAligned, typename Item, typename Stage>
__device__ __forceinline__ void walk_shared(const PagedAttnParams &p, Item &it, lds_char *smem, int lane, int wave, Stage &&stage) {
  using G = PGeo<D>;
  constexpr int KCH = D / 16, DT = D / 32, GPR = G::ROWB / 64;
  constexpr uint32_t TB = 32 * G::ROWB;
  constexpr int NB = 4;  // tiles in LDS
  static_assert(NB * 2 * TB <= kTilesB, "the tiles fit");
  constexpr int IPW = 32 / G::RPI / kPWaves;
  const PagedSource<D, kAligned> src(p, it, smem + kTilesB);
  const int col = lane & 31, hf = lane >> 5;
  const int n_t = (it.k1 - it.k0 + 31) / 32;
  auto run_of = [&](int t) __attribute__((always_inline)) { return src.run_at(it.k0 + t * 32 + wave * 8); };
  auto issue = [&](int t, const auto &run) __attribute__((always_inline)) {
    const uint32_t to = (uint32_t)(uintptr_t)smem + (uint32_t)(t % NB) * (2 * TB) + wave * IPW * 1024;
    static_assert(IPW * G::RPI == 8, "a wave's rows do not cross a multiple of 16");
    src.template fetch<IPW>(run, lane / G::CPR, to, to + TB, [&](int u, uint32_t &kchunk, uint32_t &vchunk) __attribute__((always_inline)) {
      const int line = (wave * 8 + u * G::RPI + lane / G::CPR) / G::LPR, pos = lane % G::CPR;
      kchunk = (uint32_t)(pos ^ (line & (G::CPR - 1))) << 4;
      vchunk = (uint32_t)((((pos >> 2) ^ (line & (GPR - 1))) << 2) | (pos & 3)) << 4;
    });
  };
  constexpr int OPS = 2 * IPW;  // of a wave and tile
  const int wave_row0 = it.row0 + wave * 32;
  const bool live = wave_row0 < it.n_rows;
  const PagedRow me = paged_row(p, it, min(wave_row0 + col, it.n_rows - 1));
  const int least = wave_min(me.limit);
  bf16x8_t qf[KCH];  // Q rows, the B operand of S^T = K Q^T: lane = row, chunk 2 kk + hf
  {
    const uint16_t *row = p.q + me.tok * p.q_st + me.head * p.q_sh + hf * 8;
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) qf[kk] = *reinterpret_cast<const bf16x8_t *>(row + kk * 16);
    stage();
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) asm volatile("" : "+v"(qf[kk]));
  }
#pragma unroll 1
  for (int t = 0; t < min(n_t, NB - 1); ++t) issue(t, run_of(t));
  // where this lane's fragments begin; chunk pairs kk and slabs dt on are an exclusive or away (the swizzle is one, too)
  const uint32_t k_rd = col * G::ROWB + ((hf ^ ((col / G::LPR) & (G::CPR - 1))) << 4);
  const int v_row = hf * 4 + ((lane & 15) >> 2);
  const uint32_t v_rd = v_row * G::ROWB + (((v_row / G::LPR) & (GPR - 1)) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  f32x16_t oacc[DT], s;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;
  bf16x8_t pf[2];
  float mb = -INFINITY;  // the row's reference, log2 units; not set before the row has seen a key
  float l_run = 0.f;     // this lane's share of the running sum of exponentials
  constexpr int kWin = 4;  // fragments on their way from LDS
  auto place = [&](int t) __attribute__((always_inline)) { return (uint32_t)(t % NB) * (2 * TB); };
  auto v_frag = [&](uint32_t vofs, int st) __attribute__((always_inline)) {
    typedef short s16x8_t __attribute__((ext_vector_type(8)));
    const int kc = st / DT, dt = st % DT;
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(smem + ((v_rd + vofs) ^ (dt << 6)) + kc * 16 * G::ROWB));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(smem + ((v_rd + vofs) ^ (dt << 6)) + (kc * 16 + 8) * G::ROWB));
    return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto scores = [&](int t) __attribute__((always_inline)) {
    const uint32_t kofs = place(t);
    auto k_frag = [&](int kk) __attribute__((always_inline)) { return *(lds_bf16x8 *)(smem + ((k_rd + kofs) ^ (kk << 5))); };
    bf16x8_t fr[kWin];
#pragma unroll
    for (int kk = 0; kk < kWin; ++kk) fr[kk] = k_frag(kk);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) {
      const f32x16_t zero = {};
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[kk % kWin], qf[kk], kk ? s : zero, 0, 0, 0);
      if (kk + kWin < KCH) fr[kk % kWin] = k_frag(kk + kWin);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto exponentials = [&]() __attribute__((always_inline)) {
    auto row_max = [&]() __attribute__((always_inline)) {
      float m = s[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) m = fmaxf(m, s[v]);
      return fmaxf(m, other_half(m)) * p.scale_log2e;
    };
    // the reference: the row's maximum in the first tile of which it sees a key, raised where an exponential threatens to overflow
    if (__builtin_amdgcn_ballot_w64(mb == -INFINITY) != 0) {
      const float m = row_max();
      if (mb == -INFINITY) mb = m;
    }
    float sum;
    auto powers = [&]() __attribute__((always_inline)) {
      const float ref = mb == -INFINITY ? 0.f : mb;
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e * 8 + 2 * i], p.scale_log2e, -ref));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e * 8 + 2 * i + 1], p.scale_log2e, -ref));
          s0 += p0;
          s1 += p1;
          w[i] = pack_bf16(p0, p1);
        }
        pf[e] = __builtin_bit_cast(bf16x8_t, w);
      }
      sum = s0 + s1;
    };
    powers();
    const uint64_t above = __builtin_amdgcn_ballot_w64(!(sum < kRebaseAbove));
    if (above != 0) {
      // (the rows of these lanes and no others: what another row's scores are changes no bit of this one)
      const float m = (((uint32_t)above | (uint32_t)(above >> 32)) >> col) & 1 ? fmaxf(row_max(), mb) : mb;
      const float alpha = m == mb ? 1.f : __builtin_amdgcn_exp2f(mb - m);
      mb = m;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
      powers();
    }
    l_run += sum;
  };
  // tile t has landed (every wave's share), nobody needs tile t - 1
  auto next_tile = [&](int t) __attribute__((always_inline)) {
    const int newer = min(NB - 1, n_t - t) - 1;
    if (newer == 0) dma_wait<0>();
    else if (newer == 1) dma_wait<OPS>();
    else dma_wait<2 * OPS>();
    wg_barrier();
  };
  // Tiles before t_part: all of the wave's rows see all of their keys.  (Apart from the others: one loop for both would keep a second set
  // of sums, and move 64 registers a tile.)
  const int t_part = !live || it.holes || it.k_lo > it.k0 ? 0 : max(0, min(n_t, (least - it.k0) / 32));
#pragma unroll 1
  for (int t = 0; t < t_part; ++t) {
    next_tile(t);
    const auto ahead = run_of(t + NB - 1);
    scores(t);
    if (t + NB - 1 < n_t) issue(t + NB - 1, ahead);  // (in the shadow of the products)
    const uint32_t vofs = place(t) + TB;
    bf16x8_t vf[kWin];
#pragma unroll
    for (int st = 0; st < 2; ++st) vf[st] = v_frag(vofs, st);
    __builtin_amdgcn_sched_barrier(0);
    exponentials();
#pragma unroll
    for (int st = 2; st < kWin; ++st) vf[st] = v_frag(vofs, st);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < 2 * DT; ++st) {
      oacc[st % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[st % kWin], pf[st / DT], oacc[st % DT], 0, 0, 0);
      if (st + kWin < 2 * DT) vf[st % kWin] = v_frag(vofs, st + kWin);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll 1
  for (int t = t_part; t < n_t; ++t) {
    next_tile(t);
    if (t + NB - 1 < n_t) issue(t + NB - 1, run_of(t + NB - 1));
    if (!live) continue;
    const int key0 = it.k0 + t * 32, lim = max(0, min(32, me.limit - key0));
    const uint32_t there = src.template there<32>(key0, lane);
    scores(t);
    {  // keys that this lane's row does not see at -infinity
      const uint32_t seen = (there & below(lim)) >> (hf * 4);
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (!((seen >> ((v >> 2) * 8 + (v & 3))) & 1)) s[v] = -INFINITY;
    }
    exponentials();
    // A masked probability is zero, but zero times an infinity or a NaN is not: values of keys that a row does not see must not
    // reach its sums.  The rows that see the same keys go together, with every other key's values at zero.
    uint64_t left = ~0ull;
#pragma unroll 1
    while (left) {
      const int their_lim = __builtin_amdgcn_readlane(lim, __builtin_ctzll(left));
      const bool same = lim == their_lim;
      left &= ~__builtin_amdgcn_ballot_w64(same);
      const uint32_t seen = there & below(their_lim);
      if (seen == 0) continue;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x16_t add = {};
#pragma unroll
        for (int kc = 0; kc < 2; ++kc) {
          const uint32_t mask = seen >> (kc * 16 + hf * 4);
          u32x4_t f = __builtin_bit_cast(u32x4_t, v_frag(place(t) + TB, kc * DT + dt));
#pragma unroll
          for (int e = 0; e < 4; ++e) {  // keys (e / 2) * 8 + (e % 2) * 2 and the next
            const uint32_t two = mask >> (e / 2 * 8 + e % 2 * 2);
            f[e] &= (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
          }
          add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f), pf[kc], add, 0, 0, 0);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] += same ? add[v] : 0.f;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (!live) return;
  float top = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, finite_size(oacc[dt][v]));
  const RowEnd end = row_end(p, mb, l_run + other_half(l_run), fmaxf(top, other_half(top)));
  if (wave_row0 + col >= it.n_rows) return;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const float o4[4] = {oacc[dt][q4 * 4], oacc[dt][q4 * 4 + 1], oacc[dt][q4 * 4 + 2], oacc[dt][q4 * 4 + 3]};
      write_row<D, 4>(p, it, me, end, dt * 32 + q4 * 8 + hf * 4, o4, dt == 0 && q4 == 0 && hf == 0);
    }
}

template <int D, bool kAligned, typename Groups>
__global__ __launch_bounds__(kPThreads, 2) void paged_attn_kernel(PagedAttnParams p, Groups groups) {
  extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
  lds_char *smem = (lds_char *)smem_generic;
  PagedItem it;
  if ((int)blockIdx.x < p.prefix_items) {
    // the row tiles of one range of keys share it: regroup the ids, which go round the 8 XCDs, so that each gets a run of items
    const uint32_t n = (uint32_t)p.prefix_items, q = n / 8, r = n % 8, x = blockIdx.x % 8;
    const int id = (int)(x * q + min(x, r) + blockIdx.x / 8);
    int lo = 0, hi = groups.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.item0[mid] <= id) lo = mid; else hi = mid;
    }
    it.seq0 = groups.seq0[lo];
    it.n_rows = groups.members[lo] * p.nq * p.group;
    const int tile = paged_tile_rows(it.n_rows), n_rt = (it.n_rows + tile - 1) / tile;
    int rel = id - groups.item0[lo];
    it.row0 = rel % n_rt * tile;
    rel /= n_rt;
    it.part = rel % groups.splits[lo];
    it.kvh = rel / groups.splits[lo];
    it.k_lo = it.k0 = it.part * p.chunk;
    it.k1 = min(groups.prefix[lo], it.k0 + p.chunk);
  } else {
    int rel = (int)blockIdx.x - p.prefix_items;
    it.kvh = rel % p.n_kv_heads;
    rel /= p.n_kv_heads;
    it.n_rows = p.nq * p.group;
    it.row0 = rel % p.own_row_tiles * paged_tile_rows(it.n_rows);
    rel /= p.own_row_tiles;
    it.seq0 = rel % p.n_seqs;
    it.part = rel / p.n_seqs;
    const int g = group_of(groups, it.seq0), prefix = g < 0 ? 0 : groups.prefix[g];
    // (cut at multiples of the chunk behind the multiple of 16 that the prefix ends above)
    it.k0 = prefix / 16 * 16 + it.part * p.own_chunk;
    it.k1 = min(p.cap, it.k0 + p.own_chunk);  // (as far as the sequence may reach: see below)
    it.k_lo = max(prefix, it.k0);
    if (g >= 0) it.part += groups.splits[g];
  }
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // ---- the item's part of the page table; the entries are asked for together with the sequence's length -----------------------
  it.page0 = (int)fast_div((uint32_t)it.k0, p.page_div);
  const int32_t *const table = p.page_table + it.seq0 * p.stride_table + it.page0;
  auto n_pages = [&]() __attribute__((always_inline)) { return it.k1 > it.k0 ? (int)fast_div((uint32_t)(it.k1 - 1), p.page_div) - it.page0 + 1 : 0; };
  int id = -1;
  if ((int)threadIdx.x < n_pages()) id = table[threadIdx.x];
  if ((int)blockIdx.x >= p.prefix_items) {
    it.k1 = min(it.k1, length_of(p, it.seq0));
    if (it.k_lo >= it.k1) {
      if (!p.direct) return;  // (the merge knows)
      it.k0 = it.k_lo = it.k1 = 0;
    }
  }
  auto stage = [&]() __attribute__((always_inline)) {
    const int n = n_pages();
    int bad = 0;
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kPThreads) {
      if (i >= kPThreads) id = table[i];
      const bool ok = id >= 0 && id < p.n_pages;
      ((lds_int *)(smem + kTilesB))[i] = ok ? id : -1;
      bad |= !ok;
    }
    it.holes = __syncthreads_or(bad) != 0;
  };
  const int rows = it.n_rows - it.row0;
  if (it.n_rows > kPagedStreamRows) walk_shared<D, kAligned>(p, it, smem, lane, wave, stage);
  else if (rows > 16) walk_stream<D, kAligned, 2>(p, it, smem, lane, wave, stage);
  else walk_stream<D, kAligned, 1>(p, it, smem, lane, wave, stage);
}

// The same over listed pages: an item is a range of the keys of the listed pages one after the other.  Entries from the first one on that is
// negative or not above the one in front of it are nobody's.  Bound by HBM: 128 sequences of 2,048 listed keys, 8 heads of 128, 995 MB,
// 163 us, 6.1 TB/s; 24 of 1,536, 152 MB, 31 us; for one of 2,048 by latency, 7.2 us and the merge.
template <int D, bool kAligned>
__global__ __launch_bounds__(kPThreads, 2) void paged_selected_kernel(PagedAttnParams p, PagedSelection sel) {
  extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
  lds_char *smem = (lds_char *)smem_generic;
  SelectedItem it;
  int rel = (int)blockIdx.x;
  it.kvh = rel % p.n_kv_heads;
  rel /= p.n_kv_heads;
  it.n_rows = p.nq * p.group;
  it.row0 = rel % p.own_row_tiles * paged_tile_rows(it.n_rows);
  rel /= p.own_row_tiles;
  it.seq0 = rel % p.n_seqs;
  it.part = rel / p.n_seqs;
  it.k_lo = it.k0 = it.part * p.own_chunk;
  it.page0 = (int)fast_div((uint32_t)it.k0, p.page_div);
  it.k1 = min(min(sel.keys, it.k0 + p.own_chunk), length_of(p, it.seq0));
  if (it.k0 >= it.k1) {
    if (!p.direct) return;  // (the merge knows)
    it.k_lo = it.k0 = it.k1 = it.page0 = 0;
  }
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = it.k1 > it.k0 ? (int)fast_div((uint32_t)(it.k1 - 1), p.page_div) - it.page0 + 1 : 0;
  const int32_t *const list = sel.pages + ((int64_t)it.seq0 * p.n_kv_heads + it.kvh) * sel.n, *const table = p.page_table + it.seq0 * p.stride_table;
  lds_int *const ids = (lds_int *)(smem + kTilesB), *const entries = ids + n, *const ends = entries + n;
  it.list = (lds_char *)entries;
  int valid = it.page0 + n, bad = 0;
#pragma unroll 1
  for (int i = threadIdx.x; i < it.page0 + n; i += kPThreads) {
    const int e = list[i], before = i ? list[i - 1] : -1;
    if (e <= before) valid = min(valid, i);
    if (i < it.page0) continue;
    const int id = e >= 0 && e < sel.max_pages ? table[e] : -1;
    const bool ok = id >= 0 && id < p.n_pages;
    ids[i - it.page0] = ok ? id : -1;
    entries[i - it.page0] = e;
    bad |= !ok;
  }
  valid = wave_min(valid);
  if (lane == 0) ends[wave] = valid;
  it.holes = __syncthreads_or(bad) != 0;
  valid = min(min(ends[0], ends[1]), min(ends[2], ends[3]));
  it.n_list = max(0, valid - it.page0);
  const int64_t valid_keys = (int64_t)valid * p.page_rows;
  if (valid_keys < it.k1) it.k1 = (int)valid_keys;
  if (it.k1 <= it.k0) it.k_lo = it.k0 = it.k1 = 0;
  auto stage = [] {};
  const int rows = it.n_rows - it.row0;
  if (it.n_rows > kPagedStreamRows) walk_shared<D, kAligned>(p, it, smem, lane, wave, stage);
  else if (rows > 16) walk_stream<D, kAligned, 2>(p, it, smem, lane, wave, stage);
  else walk_stream<D, kAligned, 1>(p, it, smem, lane, wave, stage);
}
// parts of a sequence's rows
__device__ __forceinline__ int parts_of(const PagedAttnParams &p, const PagedSelection &sel, int seq) {
  return (min(sel.keys, length_of(p, seq)) + p.own_chunk - 1) / p.own_chunk;
}
template <typename Groups>
__device__ __forceinline__ int parts_of(const PagedAttnParams &p, const Groups &groups, int seq) {
  const int g = group_of(groups, seq);
  const int prefix = g < 0 ? 0 : groups.prefix[g];
  // (a sequence that ends in its prefix has no part of its own)
  const int len = length_of(p, seq), own = len > prefix ? (len - prefix / 16 * 16 + p.own_chunk - 1) / p.own_chunk : 0;
  return (g < 0 ? 0 : groups.splits[g]) + own;
}

// o = sum_i w_i o_i / sum_i w_i over a row's parts, w_i = 2^(m_i - m) l_i, m = max m_i: sixteen lanes a row, kWays times over (every
// kWays-th part each).  References and sums arrive together, a lane per part, ahead of the outputs.
// Bound by launch and by the way to memory and back twice: 32 rows of 33 parts 4.3 us; 2,048 rows of 33 parts, 16 MB, 6.4.
constexpr int kMergeThreads = 256, kMergeLanes = 16;
template <int D, int kWays, typename Groups>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedAttnParams p, Groups groups) {
  constexpr int L = kMergeLanes, E = D / L, kRows = kMergeThreads / L / kWays;
  const int lane = threadIdx.x % L, way = threadIdx.x / L % kWays, slot = threadIdx.x / L / kWays, hq = p.n_kv_heads * p.group;
  const int64_t my_row = (int64_t)blockIdx.x * kRows + slot, row = min(my_row, p.part_rows - 1);
  const int tok = (int)(row / hq), head = (int)(row - (int64_t)tok * hq);
  const int seq = (int)fast_div((uint32_t)tok, p.nq_div);
  const int parts = parts_of(p, groups, seq);
  const int n = parts > way ? (parts - way + kWays - 1) / kWays : 0;  // this way's: way, way + kWays, ...
  auto end_of = [&](int i) __attribute__((always_inline)) {
    return i < n ? *reinterpret_cast<const f32x4_t *>(p.part_ml + ((way + (int64_t)i * kWays) * p.part_rows + row) * 4) : f32x4_t{-INFINITY, 0.f, 0.f, 0.f};
  };
  const f32x4_t first = end_of(lane);
  float m = first[0], l = first[1];
  for (int i = lane + L; i < n; i += L) {
    const f32x4_t e = end_of(i);
    const float to = fmaxf(m, e[0]);
    l = (l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - to)) + (e[1] == 0.f ? 0.f : e[1] * __builtin_amdgcn_exp2f(e[0] - to));
    m = to;
  }
  const float top = max_over_sixteen(m);
  l = sum_over_lanes<L>(l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - top));
  m = top;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i0 = 0; i0 < n; i0 += L) {
    const f32x4_t e = i0 ? end_of(i0 + lane) : first;
    const float w = e[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(e[0] - m) * (e[1] * inv) * e[2];
    const int here = min(L, n - i0);
    const uint16_t *from = p.part_o + ((way + (int64_t)i0 * kWays) * p.part_rows + row) * D + lane * E;
    constexpr int kAhead = kWays > 1 ? 4 : 8;
#pragma unroll 1
    for (int i = 0; i < here; i += kAhead) {
      uint32_t x[kAhead][E / 2];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint16_t *at = from + min(i + u, here - 1) * (kWays * p.part_rows * D);
#pragma unroll
        for (int c = 0; c < E / 2; c += 2) {
          const u32x2_t h = *reinterpret_cast<const u32x2_t *>(at + 2 * c);
          x[u][c] = h[0], x[u][c + 1] = h[1];
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float wi = __shfl(w, i + u, L);  // (lanes without a part, and parts that saw nothing: zero)
#pragma unroll
        for (int c = 0; c < E / 2; ++c) {
          o[2 * c] += wi == 0.f ? 0.f : f16_lo(x[u][c]) * wi;
          o[2 * c + 1] += wi == 0.f ? 0.f : f16_hi(x[u][c]) * wi;
        }
      }
    }
  }
  if constexpr (kWays > 1) {
    // two dimensions of a row to a thread
    typedef float pair_t __attribute__((ext_vector_type(2)));
    __shared__ __attribute__((aligned(16))) float all_o[kRows][kWays][D];
    __shared__ pair_t all_ml[kRows][kWays];
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4_t *>(&all_o[slot][way][lane * E + e]) = f32x4_t{o[e], o[e + 1], o[e + 2], o[e + 3]};
    if (lane == 0) all_ml[slot][way] = pair_t{m, l};
    __syncthreads();
    const int mine = threadIdx.x / (D / 2), d = threadIdx.x % (D / 2) * 2;
    const int64_t to_row = (int64_t)blockIdx.x * kRows + mine;
    if (mine >= kRows || to_row >= p.part_rows) return;
    float a = 0.f, b = 0.f;
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWays; ++w) m = fmaxf(m, all_ml[mine][w][0]);
#pragma unroll
    for (int w = 0; w < kWays; ++w) {
      const pair_t ml = all_ml[mine][w], x = *reinterpret_cast<const pair_t *>(&all_o[mine][w][d]);
      const float f = ml[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m) * ml[1];
      l += f;
      a += f == 0.f ? 0.f : x[0] * f;
      b += f == 0.f ? 0.f : x[1] * f;
    }
    const float all = l == 0.f ? 0.f : 1.f / l;
    const int64_t to_tok = to_row / hq;
    *reinterpret_cast<uint32_t *>(p.o + to_tok * p.o_st + (to_row - to_tok * hq) * p.o_sh + d) = pack_bf16(a * all, b * all);
    if (p.lse && d == 0) p.lse[to_row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  } else {
    if (my_row >= p.part_rows) return;
    uint16_t *to = p.o + tok * p.o_st + head * p.o_sh + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<u32x2_t *>(to + e) = u32x2_t{pack_bf16(o[e], o[e + 1]), pack_bf16(o[e + 2], o[e + 3])};
    if (p.lse && lane == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

// LDS behind the tiles: entries of the page table for `pages` pages
template <int D, bool kAligned, typename Groups>
struct AttnKernel {
  static constexpr int kMaxPages = kPagedMaxChunk + 2;
  static constexpr size_t table_bytes(int pages) { return (size_t)pages * 4; }
  static constexpr auto *kernel = &paged_attn_kernel<D, kAligned, Groups>;
};
template <int D, bool kAligned>
struct AttnKernel<D, kAligned, PagedSelection> {
  static constexpr int kMaxPages = kSelectedMaxPages;
  static constexpr size_t table_bytes(int pages) { return (size_t)pages * 8 + kPWaves * 4; }
  static constexpr auto *kernel = &paged_selected_kernel<D, kAligned>;
};
template <int D, bool kAligned, typename Groups>
hipError_t launch_attn_a(const PagedAttnParams &p, const Groups &g, unsigned items, size_t lds, hipStream_t stream) {
  // (a launch of more than 64 KB of LDS has to be allowed first, on every device)
  static std::atomic<bool> told[16];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev >= 16 || !told[dev].load(std::memory_order_acquire)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(AttnKernel<D, kAligned, Groups>::kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                            kTilesB + (int)AttnKernel<D, kAligned, Groups>::table_bytes(AttnKernel<D, kAligned, Groups>::kMaxPages));
    if (e != hipSuccess) return e;
    if (dev < 16) told[dev].store(true, std::memory_order_release);
  }
  AttnKernel<D, kAligned, Groups>::kernel<<<items, kPThreads, lds, stream>>>(p, g);
  return hipGetLastError();
}
template <int D, typename Groups>
hipError_t launch_attn_d(const PagedAttnParams &p, const Groups &g, hipStream_t stream) {
  const int64_t items = p.prefix_items + (int64_t)p.n_seqs * p.n_kv_heads * p.own_row_tiles * p.own_splits;
  const int32_t chunk = std::max(p.chunk, p.own_chunk);
  using Kernel = AttnKernel<D, true, Groups>;
  if (items < 1 || items > kMaxWorkgroups || chunk / p.page_rows + 2 > Kernel::kMaxPages) return hipErrorInvalidValue;
  const size_t lds = kTilesB + Kernel::table_bytes(chunk / p.page_rows + 2);  // (a range may begin and end inside a page)
  static_assert(2 * (kTilesB + Kernel::table_bytes(Kernel::kMaxPages)) <= 160 * 1024, "two workgroups a compute unit");
  return p.page_rows % 16 == 0 ? launch_attn_a<D, true>(p, g, (unsigned)items, lds, stream) : launch_attn_a<D, false>(p, g, (unsigned)items, lds, stream);
}
template <int D, int kWays, typename Groups>
hipError_t launch_merge_w(const PagedAttnParams &p, const Groups &g, hipStream_t stream) {
  constexpr int kRows = kMergeThreads / kMergeLanes / kWays;
  static_assert(kRows * kWays == kPagedMergeRows && kMergeThreads == 256, "what the size of a call is checked with");
  const int64_t wgs = (p.part_rows + kRows - 1) / kRows;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  paged_merge_kernel<D, kWays, Groups><<<(unsigned)wgs, kMergeThreads, 0, stream>>>(p, g);
  return hipGetLastError();
}
// By rows and parts, us with 1 / 4 / 16 ways: 32 rows of 33 parts 8.0 / 4.5 / 4.4, of 250 39 / 14.4 / 6.0; 128 of 63 11.4 / 5.5 / 4.7; 512 of
// 16 4.8 / 4.8 / 4.8, of 64 11.9 / 6.0 / 5.7; 1,024 of 64 11.8 / 6.6 / 8.0; 2,048 of 33 7.8 / 6.4 / 10.1; 4,096 of 17 7.5 /
// 8.2 / 15.1; 8,192 of 2 5.0 / 8.6 / 18.4.
template <int D, typename Groups>
hipError_t launch_merge_d(const PagedAttnParams &p, const Groups &g, hipStream_t stream) {
  if (p.max_parts >= 32 && p.part_rows <= 512) return launch_merge_w<D, 16>(p, g, stream);
  if (p.max_parts >= 8 && p.part_rows <= 2048) return launch_merge_w<D, 4>(p, g, stream);
  return launch_merge_w<D, 1>(p, g, stream);
}

}  // namespace

template <typename Groups>
hipError_t launch_paged_attention(const PagedAttnParams &p, const Groups &g, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_attn_d<128>(p, g, stream) : launch_attn_d<64>(p, g, stream);
}
template <typename Groups>
hipError_t launch_paged_merge(const PagedAttnParams &p, const Groups &g, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_merge_d<128>(p, g, stream) : launch_merge_d<64>(p, g, stream);
}
template hipError_t launch_paged_attention(const PagedAttnParams &, const PagedGroups &, int, hipStream_t);
template hipError_t launch_paged_attention(const PagedAttnParams &, const PagedGroupsSmall &, int, hipStream_t);
template hipError_t launch_paged_merge(const PagedAttnParams &, const PagedGroups &, int, hipStream_t);
template hipError_t launch_paged_merge(const PagedAttnParams &, const PagedGroupsSmall &, int, hipStream_t);
template hipError_t launch_paged_attention(const PagedAttnParams &, const PagedSelection &, int, hipStream_t);
template hipError_t launch_paged_merge(const PagedAttnParams &, const PagedSelection &, int, hipStream_t);

}  // namespace ba
