// Attention of one or a few query tokens of many sequences over the pages of a key/value cache, where groups of
// sequences begin with the same pages (arXiv 2409.15355, Section 2.5's final block, token by token: many questions over one set of
// passages).  For token t at position pos(t), head h: o = sum_{s <= pos} softmax_s(scale <q, k_s>) v_s.
//
// A work item is 128 packed rows (row = token * G + head in group) of one KV head over a range of keys:
//   - of a group's prefix, for the rows of all its sequences: its keys are read once for all of them;
//   - of what a sequence has behind the prefix, for its own rows.
// Every item leaves, per row, its output, reference and sum; paged_merge_kernel adds a row's parts up in their order.
// Keys and values come from the pages straight into LDS, two tiles of 32 keys ahead; the item's part of the page table lies in LDS.
// Scores are S^T = K Q^T with v_mfma_f32_32x32x16_bf16 (keys along registers, rows along lanes), the exponentials are then the
// operand of O^T = V^T P^T.  Scores, softmax, sums and parts in 32 bits; P is rounded to bf16 for the second product.
#include <type_traits>

#include "ba_device.h"
#include "ba_lds.h"
#include "ba_paged.h"

namespace ba {
namespace {

constexpr int kPWaves = kPagedTileRows / 32;
constexpr int kPThreads = kPWaves * 64;
constexpr int kPKeys = kPagedTileKeys;
constexpr int kPBuf = 3;
constexpr float kRebaseAbove = 1099511627776.0f;  // 2^40: a tile sum beyond this moves the reference

template <int D>
struct PGeo {
  static constexpr int KCH = D / 16;       // k-steps of the QK contraction
  static constexpr int DT = D / 32;        // 32-row slabs of O^T
  static constexpr int CPR = D / 8;        // 16-byte chunks per row
  static constexpr int ROWB = D * 2;       // bytes per K/V row in LDS
  static constexpr int LPR = 256 / ROWB;   // rows per 256-byte LDS line
  static constexpr int GPR = ROWB / 64;    // 64-byte granules per row
  static constexpr int TILEB = kPKeys * ROWB;
  static constexpr int RPI = 1024 / ROWB;  // rows filled by one LDS-direct wave instruction
  static constexpr int IPW = kPKeys / RPI / kPWaves;
  static constexpr int TABLE = 2 * kPBuf * TILEB;  // where the page table's part lies
};

// lds_dma16 with an address per lane: rows of different pages
__device__ __forceinline__ void lds_dma16_from(const char *from, uint32_t lds_base) {
  lds_base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_base);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds_base) : "memory");
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

template <int D, typename Groups>
__global__ __launch_bounds__(kPThreads, D == 64 ? 3 : 2) void paged_attn_kernel(PagedAttnParams p, Groups groups) {
  using G = PGeo<D>;
  extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
  lds_char *smem = (lds_char *)smem_generic;
  constexpr uint32_t TB = G::TILEB;
  typedef __attribute__((address_space(3))) int32_t lds_int;

  // ---- which work item ----------------------------------------------------------------------------
  int seq0, n_rows, row0, kvh, k0, k1, part;
  if ((int)blockIdx.x < p.prefix_items) {
    // the row tiles of one range of keys share it: regroup the ids, which go round the 8 XCDs, so that each gets a run of items
    const uint32_t n = (uint32_t)p.prefix_items, q = n / 8, r = n % 8, x = blockIdx.x % 8;
    const int id = (int)(x * q + min(x, r) + blockIdx.x / 8);
    int lo = 0, hi = groups.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.item0[mid] <= id) lo = mid; else hi = mid;
    }
    seq0 = groups.seq0[lo];
    n_rows = groups.members[lo] * p.nq * p.group;
    const int n_rt = (n_rows + kPagedTileRows - 1) / kPagedTileRows;
    int rel = id - groups.item0[lo];
    row0 = rel % n_rt * kPagedTileRows;
    rel /= n_rt;
    part = rel % groups.splits[lo];
    kvh = rel / groups.splits[lo];
    k0 = part * p.chunk;
    k1 = min(groups.prefix[lo], k0 + p.chunk);
  } else {
    int rel = (int)blockIdx.x - p.prefix_items;
    kvh = rel % p.n_kv_heads;
    rel /= p.n_kv_heads;
    row0 = rel % p.own_row_tiles * kPagedTileRows;
    rel /= p.own_row_tiles;
    seq0 = rel % p.n_seqs;
    part = rel / p.n_seqs;
    n_rows = p.nq * p.group;
    const int g = group_of(groups, seq0), prefix = g < 0 ? 0 : groups.prefix[g];
    k0 = prefix + part * p.chunk;
    k1 = min(length_of(p, seq0), k0 + p.chunk);
    if (g >= 0) part += groups.splits[g];
    if (k0 >= k1 && !p.direct) return;  // (the merge knows)
    k1 = max(k0, k1);
  }
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hf = lane >> 5;
  const int n_t = (k1 - k0 + kPKeys - 1) / kPKeys;

  // ---- this lane's row: its token, the keys it sees ---------------------------------------------------
  const int wave_row0 = row0 + wave * 32;
  const bool live = wave_row0 < n_rows;
  const int my_row = min(wave_row0 + col, n_rows - 1);
  const int tok = (int)fast_div((uint32_t)my_row, p.group_div);
  const int64_t q_tok = (int64_t)seq0 * p.nq + tok;
  const int q_head = kvh * p.group + my_row - tok * p.group;
  const int rel_seq = (int)fast_div((uint32_t)tok, p.nq_div);
  const int limit = min(k1, length_of(p, seq0 + rel_seq) - p.nq + (tok - rel_seq * p.nq) + 1);  // keys below it
  int least = limit;  // of the wave's rows
#pragma unroll
  for (int m = 1; m < 64; m *= 2) least = min(least, __shfl_xor(least, m));
  least = __builtin_amdgcn_readfirstlane(least);

  bf16x8_t qf[G::KCH];  // Q rows, the B operand of S^T = K Q^T: lane = row, chunk 2 kk + hf
  {
    const uint16_t *row = p.q + q_tok * p.q_st + q_head * p.q_sh + hf * 8;
#pragma unroll
    for (int kk = 0; kk < G::KCH; ++kk) qf[kk] = *reinterpret_cast<const bf16x8_t *>(row + kk * 16);
  }

  // ---- the item's part of the page table --------------------------------------------------------------
  const int page0 = (int)fast_div((uint32_t)k0, p.page_div);
  bool holes = false;
  if (k1 > k0) {
    const int n_pages = (int)fast_div((uint32_t)(k1 - 1), p.page_div) - page0 + 1;
    const int32_t *table = p.page_table + seq0 * p.stride_table + page0;
    int bad = 0;
    for (int i = threadIdx.x; i < n_pages; i += kPThreads) {
      const int id = table[i];
      const bool ok = id >= 0 && id < p.n_pages;
      ((lds_int *)(smem + G::TABLE))[i] = ok ? id : -1;
      bad |= !ok;
    }
    holes = __syncthreads_or(bad) != 0;
  }

  // ---- tile fill (swizzled on the global side) and fragment reads, as in the other attention kernels ----
  uint32_t k_rd[G::KCH];
  {
    const int swz = (col / G::LPR) & (G::CPR - 1);
#pragma unroll
    for (int kk = 0; kk < G::KCH; ++kk) k_rd[kk] = col * G::ROWB + (((kk * 2 + hf) ^ swz) << 4);
  }
  uint32_t v_rd[G::DT];
  {
    const int vrow = hf * 4 + ((lane & 15) >> 2);
    const int vwithin = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    const int swz = (vrow / G::LPR) & (G::GPR - 1);
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt) v_rd[dt] = vrow * G::ROWB + ((dt ^ swz) << 6) + vwithin;
  }
  const char *k_base = (const char *)(p.k + kvh * p.k_sh), *v_base = (const char *)(p.v + kvh * p.v_sh);
  const uint32_t lds_copy = (uint32_t)(uintptr_t)smem + wave * G::IPW * 1024;
  auto page_of = [&](int key, int &row) __attribute__((always_inline)) {
    const int i = (int)fast_div((uint32_t)key, p.page_div);
    row = key - i * p.page_rows;
    return ((const lds_int *)(smem + G::TABLE))[i - page0];
  };
  auto issue_copy = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < G::IPW; ++u) {
      const int r = (wave * G::IPW + u) * G::RPI + lane / G::CPR, pos = lane % G::CPR;
      const uint32_t kchunk = (uint32_t)(pos ^ ((r / G::LPR) & (G::CPR - 1))) << 4;
      const uint32_t vchunk = (uint32_t)((((pos >> 2) ^ ((r / G::LPR) & (G::GPR - 1))) << 2) | (pos & 3)) << 4;
      int row;
      // (rows behind the range take its last one; pages that are not there take page 0: both are masked)
      const int page = max(0, page_of(min(k0 + t * kPKeys + r, k1 - 1), row));
      lds_dma16_from(k_base + page * p.k_page_b + ((uint64_t)(uint32_t)row * p.k_rb + kchunk), lds_copy + (uint32_t)buf * (2 * TB) + u * 1024);
      lds_dma16_from(v_base + page * p.v_page_b + ((uint64_t)(uint32_t)row * p.v_rb + vchunk), lds_copy + (uint32_t)buf * (2 * TB) + TB + u * 1024);
    }
  };
  constexpr int kOpsPerTile = 2 * G::IPW;
#pragma unroll
  for (int kk = 0; kk < G::KCH; ++kk) asm volatile("" : "+v"(qf[kk]));  // the rows are waited for here, not inside the loop
  if (n_t > 0) issue_copy(0, 0);
  if (n_t > 1) issue_copy(1, 1);
  __builtin_amdgcn_sched_barrier(0);

  // ---- running state ------------------------------------------------------------------------------------
  f32x16_t oacc[G::DT];
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;
  float mb = -INFINITY;  // the row's reference, log2 units; not set before the row has seen a key
  float l_run = 0.f;     // this lane's share of the running sum of exponentials

  int buf = 0;
#pragma unroll 1
  for (int t = 0; t < n_t; ++t) {
    if (t + 1 < n_t) dma_wait<kOpsPerTile>(); else dma_wait<0>();
    wg_barrier();  // every wave's share of tile t has landed, and every wave is done with tile t - 1
    if (t + 2 < n_t) issue_copy(t + 2, buf == 0 ? 2 : buf - 1);
    if (live) {
      const uint32_t kofs = (uint32_t)buf * (2 * TB), vofs = kofs + TB;
      const int key0 = k0 + t * kPKeys;
      f32x16_t s;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
      for (int kk = 0; kk < G::KCH; ++kk)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const __attribute__((address_space(3))) bf16x8_t *>(smem + (k_rd[kk] + kofs)), qf[kk], s, 0, 0, 0);
      // keys that this lane's row does not see at -infinity
      const bool masked = holes || key0 + kPKeys > least;
      const int lim = limit - key0;
      uint32_t there = ~0u;  // keys whose page is there
      if (masked) {
        if (holes) {
          int row;
          there = (uint32_t)__builtin_amdgcn_ballot_w64(page_of(min(key0 + col, k1 - 1), row) >= 0);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = (v >> 2) * 8 + hf * 4 + (v & 3);
          if (key >= lim || !((there >> key) & 1)) s[v] = -INFINITY;
        }
      }
      // the reference: the row's maximum in the first tile of which it sees a key, raised where an exponential threatens to overflow
      auto row_max = [&]() __attribute__((always_inline)) {
        float m = s[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) m = fmaxf(m, s[v]);
        return fmaxf(m, other_half(m)) * p.scale_log2e;
      };
      if (__builtin_amdgcn_ballot_w64(mb == -INFINITY) != 0) {
        const float m = row_max();
        if (mb == -INFINITY) mb = m;
      }
      bf16x8_t pf[2];
      float sum;
      auto exponentials = [&]() __attribute__((always_inline)) {
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
      exponentials();
      if (__builtin_amdgcn_ballot_w64(!(sum < kRebaseAbove)) != 0) {
        // (only the rows concerned: what another row's scores are changes no bit of this one)
        const float m = !(sum + other_half(sum) < kRebaseAbove) ? fmaxf(row_max(), mb) : mb;
        const float alpha = m == mb ? 1.f : __builtin_amdgcn_exp2f(mb - m);
        mb = m;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < G::DT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
        exponentials();
      }
      l_run += sum;
      auto v_frag = [&](int kc, int dt) __attribute__((always_inline)) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(smem + (v_rd[dt] + vofs) + kc * 16 * G::ROWB));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(smem + (v_rd[dt] + vofs) + (kc * 16 + 8) * G::ROWB));
        return (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      };
      if (!masked) {
#pragma unroll
        for (int st = 0; st < 2 * G::DT; ++st)
          oacc[st % G::DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v_frag(st / G::DT, st % G::DT)), pf[st / G::DT],
                                                                      oacc[st % G::DT], 0, 0, 0);
      } else {
        // A masked probability is zero, but zero times an infinity or a NaN is not: values of keys that a row does not see must
        // not reach its sums.  The rows that see the same keys go together, with every other key's values at zero.
        uint64_t left = ~0ull;
#pragma unroll 1
        while (left) {
          const int their_lim = __builtin_amdgcn_readlane(lim, __builtin_ctzll(left));
          const bool mine = lim == their_lim;
          left &= ~__builtin_amdgcn_ballot_w64(mine);
          const uint32_t seen = there & (their_lim <= 0 ? 0u : their_lim >= 32 ? ~0u : (1u << their_lim) - 1u);
          if (seen == 0) continue;
#pragma unroll
          for (int dt = 0; dt < G::DT; ++dt) {
            f32x16_t add;
#pragma unroll
            for (int v = 0; v < 16; ++v) add[v] = 0.f;
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
              auto f = v_frag(kc, dt);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (!((seen >> (kc * 16 + (e >> 2) * 8 + hf * 4 + (e & 3))) & 1)) f[e] = 0;
              add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f), pf[kc], add, 0, 0, 0);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) oacc[dt][v] += mine ? add[v] : 0.f;
          }
        }
      }
    }
    buf = buf == kPBuf - 1 ? 0 : buf + 1;
  }

  // ---- out: lane = row, four consecutive dimensions at a time -------------------------------------------
  if (!live || wave_row0 + col >= n_rows) return;
  const float l = l_run + other_half(l_run);
  if (p.direct) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *o = p.o + q_tok * p.o_st + q_head * p.o_sh + hf * 4;
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const u32x2_t w = {pack_bf16(oacc[dt][q4 * 4] * inv, oacc[dt][q4 * 4 + 1] * inv),
                           pack_bf16(oacc[dt][q4 * 4 + 2] * inv, oacc[dt][q4 * 4 + 3] * inv)};
        *reinterpret_cast<u32x2_t *>(o + dt * 32 + q4 * 8) = w;
      }
    if (p.lse && hf == 0)
      p.lse[q_tok * (p.n_kv_heads * p.group) + q_head] = l == 0.f ? -INFINITY : (mb + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  } else {
    const int64_t at = part * p.part_rows + q_tok * (p.n_kv_heads * p.group) + q_head;
    float *o = p.part_o + at * D + hf * 4;
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4_t *>(o + dt * 32 + q4 * 8) = f32x4_t{oacc[dt][q4 * 4], oacc[dt][q4 * 4 + 1], oacc[dt][q4 * 4 + 2], oacc[dt][q4 * 4 + 3]};
    if (hf == 0) *reinterpret_cast<f32x2_t *>(p.part_ml + at * 2) = f32x2_t{l == 0.f ? -INFINITY : mb, l};
  }
}

// o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over a row's parts, m = max m_i.  32 lanes a row.
constexpr int kMergeThreads = 256;
template <int D, typename Groups>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedAttnParams p, Groups groups) {
  constexpr int E = D / 32;
  typedef float vec_t __attribute__((ext_vector_type(E)));
  const int64_t row = (int64_t)blockIdx.x * (kMergeThreads / 32) + threadIdx.x / 32;
  if (row >= p.part_rows) return;
  const int lane = threadIdx.x & 31, hq = p.n_kv_heads * p.group;
  const int tok = (int)(row / hq), head = (int)(row - (int64_t)tok * hq);
  const int seq = (int)fast_div((uint32_t)tok, p.nq_div);
  const int g = group_of(groups, seq);
  const int prefix = g < 0 ? 0 : groups.prefix[g];
  const int parts = (g < 0 ? 0 : groups.splits[g]) + (max(0, length_of(p, seq) - prefix) + p.chunk - 1) / p.chunk;
  float m = -INFINITY, l = 0.f;
  vec_t o;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const int64_t at = i * p.part_rows + row;
    const f32x2_t ml = *reinterpret_cast<const f32x2_t *>(p.part_ml + at * 2);
    const vec_t x = *reinterpret_cast<const vec_t *>(p.part_o + at * D + lane * E);
    if (ml[1] == 0.f) continue;  // saw nothing
    const float to = fmaxf(m, ml[0]);
    const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - to), add = __builtin_amdgcn_exp2f(ml[0] - to);
    m = to;
    l = l * keep + ml[1] * add;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * keep + x[e] * add;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint32_t w[E / 2];
#pragma unroll
  for (int e = 0; e < E / 2; ++e) w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
  uint32_t *to = reinterpret_cast<uint32_t *>(p.o + tok * p.o_st + head * p.o_sh + lane * E);
#pragma unroll
  for (int e = 0; e < E / 2; ++e) to[e] = w[e];
  if (p.lse && lane == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, typename Groups>
hipError_t launch_attn_d(const PagedAttnParams &p, const Groups &g, hipStream_t stream) {
  const int64_t items = p.prefix_items + (int64_t)p.n_seqs * p.n_kv_heads * p.own_row_tiles * p.own_splits;
  if (items < 1 || items > 0x7fffffff || p.chunk > kPagedMaxChunk) return hipErrorInvalidValue;
  const size_t lds = PGeo<D>::TABLE + (size_t)(p.chunk / p.page_rows + 2) * 4;  // (a range may begin and end inside a page)
  static_assert(PGeo<D>::TABLE + (kPagedMaxChunk + 2) * 4 <= 65536, "as much as a launch may ask for without further ado");
  paged_attn_kernel<D, Groups><<<(unsigned)items, kPThreads, lds, stream>>>(p, g);
  return hipGetLastError();
}
template <int D, typename Groups>
hipError_t launch_merge_d(const PagedAttnParams &p, const Groups &g, hipStream_t stream) {
  constexpr int kRows = kMergeThreads / 32;
  const int64_t wgs = (p.part_rows + kRows - 1) / kRows;
  if (wgs < 1 || wgs > 0x7fffffff) return hipErrorInvalidValue;
  paged_merge_kernel<D, Groups><<<(unsigned)wgs, kMergeThreads, 0, stream>>>(p, g);
  return hipGetLastError();
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

}  // namespace ba
