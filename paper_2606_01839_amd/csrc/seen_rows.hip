// Attention of rows that are not a conversation's last tokens in causal order (host/seen.hpp), for few rows: a tree of
// some guesses, a decoder's hypotheses. Split over the keys as the decode (decode.hip), but up to 64 rows (query tokens x
// query heads of the kv head) share what is read: blocks of 16 rows are the N side of the matrix products, and each K and V
// operand serves all blocks from the registers it was loaded to.
//   S^T[key][row] = K . Q^T      O^T[dim][row] += V^T . P^T      (v_mfma_f32_16x16x32_bf16)
// Weights are taken against a running maximum that is only refreshed when a lane's sum of a step's weights exceeds 2^8 (or is not
// finite, as on the first): no exchange between lanes on the common path. Scores lose the maximum before they are scaled, so
// those of any magnitude keep their largest weight at 1.
//
// Bound: HBM where the cache is long. 64 conversations of 8k-32k tokens, 32 query and 8 kv heads of 128: 682 us for trees of one
// token (6.70 TB/s, as the decode), 703 for 4, 729 for 8, 753 for 12, 796 for 16 (64 rows; as tiles 861); the matrix cores are 9%
// busy at 28 rows. What the rows add is the join of an item's waves (a block of 16 rows 1 us at the end of an item) and
// records. One tree of 16 tokens on 24.6k takes 28.0 us, of 4 19.7: start, loads in three bursts, join, merge launch 4.5.
// Over 4-bit pages 207 us for 4 tokens, 258 for 8, 393 for 16: arithmetic, two products' chains of each block.
#include <cfloat>
#include <cmath>

#include "decode_split.hpp"
#include "device_common.hpp"
#include "fp4.hpp"
#include "kernels.hpp"

namespace cs {

struct RowsArgs {
  const uint16_t* pool;
  int64_t n_pages;
  int n_kv_heads, group_log2, layer;
  const int32_t* page_table;
  int max_pages;
  const void* meta;
  uint32_t masks_off, words_off, items_off, merges_off;
  int split;          // keys per wave, a multiple of 32, at most 1024
  const uint16_t* q;
  uint16_t* out;
  float* parts;       // records [record][kv head][16 NB rows] of partial_floats(D)
  float scale_log2;
  __device__ __forceinline__ SeenItem item(int i) const {
    const auto* p = meta_at<SeenItem>(meta, items_off) + i;
    return {p->conv, p->k0};
  }
  __device__ __forceinline__ ExtendConvDesc conv(int i) const {
    const auto* p = meta_at<ExtendConvDesc>(meta, 0) + i;
    return {p->slot, p->len, p->q_len, p->q_row};
  }
  __device__ __forceinline__ SeenMask seen(int i) const {
    const auto* p = meta_at<SeenMask>(meta, masks_off) + i;
    return {p->clear, p->off, p->words, p->rec};
  }
};

constexpr int kRowWaves = kDecodeSubSplits;
constexpr float kRowSumLimit = 256.f;

// max / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quarters_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// (vectors of the compiler's own: arrays of the runtime's uint2 ended up in scratch memory)
__device__ __forceinline__ u32x4_t nt16(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4_t*>(p)); }
__device__ __forceinline__ u32x2_t nt8(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x2_t*>(p)); }
__device__ __forceinline__ bf16x8 pages_v(u32x2_t a, u32x2_t b) { return __builtin_bit_cast(bf16x8, u32x4_t{a.x, a.y, b.x, b.y}); }

// One (item, kv head) per workgroup of eight waves.
template <int D, int NB, bool FP4>
__device__ __forceinline__ void rows_body(const RowsArgs& a) {
  constexpr int KS = D / 32, DT = D / 16, R = partial_floats(D);
  constexpr bool QLDS = NB > 2;             // queries in LDS instead of registers
  constexpr int QW = FP4 ? 5 : KS;          // 16-byte words of a lane's query operand, a block
  constexpr int NX = NB > 1 ? 2 : 1;        // blocks the waves exchange at a time
  __shared__ __attribute__((aligned(16))) float xch[NX][kRowWaves][16][R];
  constexpr bool WLDS = NB > 3 && !FP4;     // words in LDS: the registers are full
  __shared__ uint32_t w_lds[WLDS ? kRowWaves : 1][WLDS ? NB : 1][16];
  __shared__ uint4 q_lds[QLDS ? NB : 1][QLDS ? QW : 1][64];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, qd = lane >> 4;
  const int g = blockIdx.x % a.n_kv_heads;
  const SeenItem it = a.item(blockIdx.x / a.n_kv_heads);
  const ExtendConvDesc cd = a.conv(it.conv);
  const SeenMask mk = a.seen(it.conv);
  const int item_keys = kRowWaves * a.split;
  const int k1 = min(cd.len, it.k0 + item_keys);
  const int wave_keys = ((k1 - it.k0 + kRowWaves - 1) / kRowWaves + 2 * kPageTokens - 1) & ~(2 * kPageTokens - 1);
  const int k_begin = it.k0 + wave * wave_keys, k_end = min(k1, k_begin + wave_keys);
  const int n_pg = k_end > k_begin ? (k_end - k_begin + kPageTokens - 1) / kPageTokens : 0;
  const int32_t* pt = a.page_table + static_cast<size_t>(cd.slot) * a.max_pages + k_begin / kPageTokens;
  const int pid = lane < n_pg ? pt[lane] : 0;

  const int n_rows = cd.q_len << a.group_log2, n_q_heads = a.n_kv_heads << a.group_log2;
  const int nb_used = NB == 1 ? 1 : (n_rows + 15) / 16;
  auto row_offset = [&](int r) {   // of row r of the kv head, elements
    return (static_cast<size_t>(cd.q_row + (r >> a.group_log2)) * n_q_heads + (g << a.group_log2) + (r & ((1 << a.group_log2) - 1))) * D;
  };
  // Query operand of block nb: row 16 nb + c, dims 32 ks + 8 qd .. (4-bit pages: (D/4) qd ..). Rows past the last are zeros.
  auto load_q = [&](int nb, uint4 (&x)[4]) {
    const int r = 16 * nb + c;
    const uint16_t* p = a.q + row_offset(r < n_rows ? r : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_uint4(0, 0, 0, 0);
    if (r < n_rows) {
#pragma unroll
      for (int i = 0; i < KS; ++i) x[i] = ld16(FP4 ? p + D / 4 * qd + 8 * i : p + 32 * i + 8 * qd);
    }
  };
  using B = Fp4Block<D>;
  constexpr int NW = B::kWords;
  const size_t block_bytes = FP4 ? B::kBytes : 4 * kPageTokens * D;
  const size_t page_stride = static_cast<size_t>(a.n_kv_heads) * block_bytes;
  const uint8_t* base = reinterpret_cast<const uint8_t*>(a.pool) + static_cast<size_t>(a.layer) * a.n_pages * page_stride +
                        static_cast<size_t>(g) * block_bytes;
  const uint32_t koff = (c * 32 + 8 * qd) * 2, voff = (kPageTokens * D + c * kPageTokens + 4 * qd) * 2;
  const uint32_t f_k = B::k_lane(lane), f_v = B::kV + lane * 4 * NW, f_ks = B::k_scale_lane(lane), f_vs = B::kVScale + 4 * qd;
  struct Page {
    u32x4_t k[FP4 ? 1 : KS];
    u32x2_t v[FP4 ? 2 : DT];
    uint32_t ks, vs;
  };
  auto load = [&](int j) {
    Page p;
    const uint8_t* blk = base + static_cast<size_t>(__builtin_amdgcn_readlane(pid, j)) * page_stride;
    p.ks = p.vs = 0;
    if constexpr (FP4) {
      // (as 32-bit offsets to a scalar base; hoisted out of the loop they would be widened to register pairs)
      uint32_t ok = f_k, ov = f_v, oks = f_ks, ovs = f_vs;
      asm volatile("" : "+v"(ok), "+v"(ov), "+v"(oks), "+v"(ovs));
      if constexpr (D == 128) {
        const u32x4_t v = nt16(blk + ov);
        p.k[0] = nt16(blk + ok);
        p.v[0] = v.lo, p.v[1] = v.hi;
      } else {
        const u32x2_t k = nt8(blk + ok);
        p.k[0] = u32x4_t{k.x, k.y, 0, 0};
        p.v[0] = nt8(blk + ov), p.v[1] = u32x2_t{0, 0};
      }
      p.ks = blk[oks];
      p.vs = *reinterpret_cast<const uint32_t*>(blk + ovs);
    } else {
#pragma unroll
      for (int i = 0; i < KS; ++i) p.k[i] = nt16(blk + koff + 1024 * i);
#pragma unroll
      for (int t = 0; t < DT; ++t) p.v[t] = nt8(blk + voff + 16 * kPageTokens * 2 * t);
    }
    return p;
  };

  struct Query {
    bf16x8 b[KS];
    Bf6Query x;
  };
  Query qop[QLDS ? 1 : NB];
  if constexpr (QLDS) {
    if (wave < nb_used) {
      uint4 x[4];
      load_q(wave, x);
      if constexpr (FP4) {
        const Bf6Query s = split_query(x);
        uint32_t w[20];
#pragma unroll
        for (int i = 0; i < 18; ++i) w[i] = s.p[i / 6][i % 6];
        w[18] = s.scale, w[19] = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) q_lds[wave][i][lane] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) q_lds[wave][i][lane] = x[i];
      }
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      uint4 x[4];
      load_q(nb, x);
      if constexpr (FP4) qop[nb].x = split_query(x);
      else
#pragma unroll
        for (int i = 0; i < KS; ++i) qop[nb].b[i] = as_bf16x8(x[i]);
    }
  }
  auto query = [&](int nb) {
    if constexpr (!QLDS) return qop[nb];
    Query r;
    if constexpr (FP4) {
      uint32_t w[20];
#pragma unroll
      for (int i = 0; i < 5; ++i) {
        const uint4 x = q_lds[nb][i][lane];
        w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
      }
#pragma unroll
      for (int i = 0; i < 18; ++i) r.x.p[i / 6][i % 6] = w[i];
      r.x.scale = w[18];
    } else {
#pragma unroll
      for (int i = 0; i < KS; ++i) r.b[i] = as_bf16x8(q_lds[nb][i][lane]);
    }
    return r;
  };

  float m_run[NB], l_run[NB];
  f32x4 o[NB][DT];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m_run[nb] = -FLT_MAX;
    l_run[nb] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[nb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool sick = false;   // values that are not finite were cleared
  const bf16x2 ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};

  // Keys k .. k + 31: pages j, j + 1 (a last single page stands in for its second, whose keys are not seen).
  auto step = [&](const Page& pa, const Page& pb, const int j) {
    const int k = k_begin + kPageTokens * j;
    const bool partly = k + 2 * kPageTokens > mk.clear;
    uint32_t seen_w[WLDS ? 1 : NB];   // of the lane's rows, for the 32 keys
    if (partly) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        uint32_t word;
        if (mk.words > 0) {
          const int w = (k >> 5) - (mk.clear >> 5), i = (16 * nb + c) >> a.group_log2;
          const uint32_t* words = (const uint32_t*)meta_at<uint32_t>(a.meta, a.words_off) + mk.off;
          word = w < mk.words ? words[static_cast<size_t>(min(i, cd.q_len - 1)) * mk.words + w] : 0u;
        } else {
          const int left = mk.clear - k;
          word = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
        }
        if constexpr (WLDS) w_lds[wave][nb][c] = word;
        else seen_w[nb] = word;
      }
    }
    auto word_of = [&](int nb) { return WLDS ? w_lds[wave][nb][c] : seen_w[WLDS ? 0 : nb]; };
    bf16x8 vop[DT];
    auto convert = [&]() {
      const uint32_t wa[4] = {pa.v[0].x, pa.v[0].y, pa.v[1].x, pa.v[1].y}, wb[4] = {pb.v[0].x, pb.v[0].y, pb.v[1].x, pb.v[1].y};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        vop[2 * w] = as_bf16x8(make_uint2(fp4_pair<0>(wa[w], 1.f), fp4_pair<1>(wa[w], 1.f)),
                               make_uint2(fp4_pair<0>(wb[w], 1.f), fp4_pair<1>(wb[w], 1.f)));
        vop[2 * w + 1] = as_bf16x8(make_uint2(fp4_pair<2>(wa[w], 1.f), fp4_pair<3>(wa[w], 1.f)),
                                   make_uint2(fp4_pair<2>(wb[w], 1.f), fp4_pair<3>(wb[w], 1.f)));
      }
    };
    if constexpr (FP4) {
      if constexpr (NB > 1) convert();   // once for all blocks (one block: where it is used, two workgroups a CU)
    } else {
#pragma unroll
      for (int t = 0; t < DT; ++t) vop[t] = pages_v(pa.v[t], pb.v[t]);
      if (partly && j + 1 >= n_pg) {
#pragma unroll
        for (int t = 0; t < DT; ++t) vop[t] = pages_v(pa.v[t], u32x2_t{0, 0});
      }
      if (partly) {
        uint32_t any = 0;
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const u32x4_t w = __builtin_bit_cast(u32x4_t, vop[t]);
          any |= not_finite(w[0]) | not_finite(w[1]) | not_finite(w[2]) | not_finite(w[3]);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(any != 0) != 0, false)) {
          // They must not meet weights of 0: cleared here, and added after the last step to the rows that see them (any weight of an
          // infinity is an infinity). No row sees those behind the last key, which a failed append may have left.
          sick = true;
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            u32x4_t w = __builtin_bit_cast(u32x4_t, vop[t]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = finite_or_zero(w[i]);
            vop[t] = __builtin_bit_cast(bf16x8, w);
          }
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (NB > 1 && nb >= nb_used) break;
      const Query qn = query(nb);
      f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
      if constexpr (FP4) {
        const uint4 kpa = __builtin_bit_cast(uint4, pa.k[0]), kpb = __builtin_bit_cast(uint4, pb.k[0]);
        sa = mx_score<0, 0>(kpa, pa.ks, qn.x, sa);
        sb = mx_score<0, 0>(kpb, pb.ks, qn.x, sb);
        sa = mx_score<1, 0>(kpa, pa.ks, qn.x, sa);
        sb = mx_score<1, 0>(kpb, pb.ks, qn.x, sb);
        sa = mx_score<2, 0>(kpa, pa.ks, qn.x, sa);
        sb = mx_score<2, 0>(kpb, pb.ks, qn.x, sb);
      } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          sa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pa.k[i]), qn.b[i], sa, 0, 0, 0);
          sb = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pb.k[i]), qn.b[i], sb, 0, 0, 0);
        }
      }
      // sa[r]: row c, key k + 4 qd + r; sb[r]: the same + 16.
      float x[8] = {sa[0], sa[1], sa[2], sa[3], sb[0], sb[1], sb[2], sb[3]}, vn[8];
      if constexpr (FP4)
#pragma unroll
        for (int r = 0; r < 8; ++r) vn[r] = fp4_scale_of(r < 4 ? pa.vs : pb.vs, r % 4);
      if (partly) {
        const uint32_t mine = word_of(nb) >> (4 * qd);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const bool in = mine >> (r < 4 ? r : 12 + r) & 1;
          x[r] = in ? x[r] : -INFINITY;
          if constexpr (FP4) vn[r] = in ? vn[r] : 0.f;   // (0 x a scale of 255 would be NaN)
        }
      }
      uint4 pw;
      float p[8];
      auto weights = [&]() {
#pragma unroll
        for (int r = 0; r < 8; ++r) p[r] = fast_exp2((x[r] - m_run[nb]) * a.scale_log2);
        pw = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
        // the denominator sums the same bf16-rounded weights the PV product uses
        float s0 = 0.f, s1 = 0.f;
        s0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw.x), ones, s0, false);
        s1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw.y), ones, s1, false);
        s0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw.z), ones, s0, false);
        s1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw.w), ones, s1, false);
        return s0 + s1;
      };
      float ps = weights();
      if (__builtin_amdgcn_ballot_w64(!(ps <= kRowSumLimit)) != 0) {
        float mx = x[0];
#pragma unroll
        for (int r = 1; r < 8; ++r) mx = fmaxf(mx, x[r]);
        const float m_new = fmaxf(m_run[nb], quarters_max(mx));
        const float alpha = fast_exp2((m_run[nb] - m_new) * a.scale_log2);
        m_run[nb] = m_new;
        l_run[nb] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[nb][t] *= alpha;
        ps = weights();
      }
      l_run[nb] += ps;
      if constexpr (FP4) {
        pw = make_uint4(pack_bf16x2(p[0] * vn[0], p[1] * vn[1]), pack_bf16x2(p[2] * vn[2], p[3] * vn[3]),
                        pack_bf16x2(p[4] * vn[4], p[5] * vn[5]), pack_bf16x2(p[6] * vn[6], p[7] * vn[7]));
      }
      const bf16x8 pop = __builtin_bit_cast(bf16x8, pw);
      if constexpr (FP4 && NB == 1) convert();
#pragma unroll
      for (int t = 0; t < DT; ++t) o[nb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop[t], pop, o[nb][t], 0, 0, 0);
    }
  };
  if constexpr (FP4) {
    if (n_pg > 0) {   // the next pages fly during a step
      Page a0 = load(0), b0 = load(min(1, n_pg - 1));
      for (int j = 0; j < n_pg; j += 2) {
        const Page pa = a0, pb = b0;
        a0 = load(min(j + 2, n_pg - 1));
        b0 = load(min(j + 3, n_pg - 1));
        step(pa, pb, j);
      }
    }
  } else {
    for (int j = 0; j < n_pg; j += 2) {
      const Page pa = load(j), pb = load(min(j + 1, n_pg - 1));
      step(pa, pb, j);
    }
  }

  if constexpr (!FP4) {
    if (__builtin_expect(sick, false)) {
      const uint32_t* words = (const uint32_t*)meta_at<uint32_t>(a.meta, a.words_off) + mk.off;
      for (int key = max(k_begin, mk.clear & ~31); key < k_end; ++key) {   // of the masked steps
        const uint16_t* v = reinterpret_cast<const uint16_t*>(base + static_cast<size_t>(__builtin_amdgcn_readlane(pid, (key - k_begin) / kPageTokens)) * page_stride) +
                            kPageTokens * D + key % kPageTokens;
        uint32_t x[DT][4];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][r] = v[(16 * t + 4 * qd + r) * kPageTokens];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int i = min((16 * nb + c) >> a.group_log2, cd.q_len - 1);
          const bool sees = key < mk.clear || (words[static_cast<size_t>(i) * mk.words + (key >> 5) - (mk.clear >> 5)] >> (key & 31) & 1);
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (sees && (x[t][r] & 0x7F80u) == 0x7F80u) o[nb][t][r] += __uint_as_float(x[t][r] << 16);
        }
      }
    }
  }

  // The eight waves' results are joined NX blocks at a time, each wave some rows, in the order of the waves. (The joining code is there
  // once: what a launch runs for the first time has to be fetched, and small launches wait for that.)
  constexpr int LPR = D / 4, RPW = 64 / LPR;   // lanes of a row, rows a wave
  const int rr = wave * RPW + lane / LPR, d4 = 4 * (lane % LPR);
#pragma unroll 1
  for (int nb0 = 0; nb0 < nb_used; nb0 += NX) {
    if (nb0 > 0) __syncthreads();   // the bytes' last readers
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb / NX * NX != nb0 || nb >= nb_used) continue;
      float (*x)[R] = xch[nb % NX][wave];
      const float l = quarters_sum(l_run[nb]);
#pragma unroll
      for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(&x[c][16 * t + 4 * qd]) = o[nb][t];
      if (qd == 0) *reinterpret_cast<f32x2*>(&x[c][D]) = f32x2{m_run[nb], l};
    }
    __syncthreads();
    if (rr >= 16) continue;
#pragma unroll 1
    for (int u = 0; u < NX; ++u) {
      const int r = 16 * (nb0 + u) + rr;
      if (r >= n_rows) break;
      f32x2 ml[kRowWaves];
      f32x4 y[kRowWaves];
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {
        ml[w] = *reinterpret_cast<const f32x2*>(&xch[u][w][rr][D]);
        y[w] = *reinterpret_cast<const f32x4*>(&xch[u][w][rr][d4]);
      }
      float M = ml[0].x;
#pragma unroll
      for (int w = 1; w < kRowWaves; ++w) M = fmaxf(M, ml[w].x);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      float den = 0.f;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {
        const float wt = fast_exp2((ml[w].x - M) * a.scale_log2);
        den = __builtin_fmaf(wt, ml[w].y, den);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(wt, y[w][i], acc[i]);
      }
      if (mk.rec < 0) {   // the item is the whole conversation
        const float inv = 1.f / den;
        st8(a.out + row_offset(r) + d4, make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)));
      } else {
        float* rec = a.parts + ((static_cast<size_t>(mk.rec + it.k0 / item_keys) * a.n_kv_heads + g) * (16 * NB) + r) * R;
        __builtin_nontemporal_store(acc, reinterpret_cast<f32x4*>(rec + d4));
        if (d4 == 0) *reinterpret_cast<f32x2*>(rec + D) = f32x2{M, den};
      }
    }
  }
}

template <int D, int NB>
__global__ __launch_bounds__(64 * kRowWaves) __attribute__((amdgpu_waves_per_eu(2))) void seen_rows_kernel(LaunchMeta, RowsArgs a) {
  rows_body<D, NB, false>(a);
}
template <int D, int NB>
__global__ __launch_bounds__(64 * kRowWaves) __attribute__((amdgpu_waves_per_eu(NB == 1 ? 4 : 2))) void seen_rows_fp4_kernel(LaunchMeta, RowsArgs a) {
  rows_body<D, NB, true>(a);
}

// The records of the rows of an entry of several items, joined in a fixed order. A workgroup's 256 threads are SG groups of D / 4
// lanes (4 dims each); `per_row` of them (a power of two, at most 4 records each where that holds all) share a row. kv heads
// fastest, as in the grid that wrote the records. (A workgroup a row: 42 us for 64 trees of 64 rows, two or three records a row.)
template <int D>
__global__ __launch_bounds__(256) void seen_rows_merge_kernel(LaunchMeta, RowsArgs a, int row_groups, int per_row, int rows16) {
  constexpr int DV = D / 4, SG = 256 / DV, R = partial_floats(D), kAhead = 4;
  __shared__ float red_m[SG], red_l[SG];
  __shared__ __attribute__((aligned(16))) float red_o[SG][D];
  const int tid = threadIdx.x, d4 = 4 * (tid % DV), sg = tid / DV, part = sg % per_row;
  const int g = blockIdx.x % a.n_kv_heads, rg = blockIdx.x / a.n_kv_heads % row_groups;
  const int conv = meta_at<int32_t>(a.meta, a.merges_off)[blockIdx.x / a.n_kv_heads / row_groups];
  const ExtendConvDesc cd = a.conv(conv);
  const int n_rows = cd.q_len << a.group_log2, r0 = rg * (SG / per_row), r = r0 + sg / per_row;
  if (r0 >= n_rows) return;
  const int item_keys = kRowWaves * a.split, n = (cd.len + item_keys - 1) / item_keys;
  const size_t stride = static_cast<size_t>(a.n_kv_heads) * rows16 * R;
  const float* base = a.parts + (static_cast<size_t>(a.seen(conv).rec) * a.n_kv_heads + g) * rows16 * R + static_cast<size_t>(min(r, n_rows - 1)) * R;
  f32x2 ml[kAhead];
  f32x4 v[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int s = part + k * per_row;
    const float* p = base + (s < n ? s : 0) * stride;
    ml[k] = *reinterpret_cast<const f32x2*>(p + D);
    v[k] = *reinterpret_cast<const f32x4*>(p + d4);
  }
  float M = ml[0].x;                 // (record 0 where the thread has none)
#pragma unroll
  for (int k = 1; k < kAhead; ++k) M = fmaxf(M, ml[k].x);
  for (int s = part + kAhead * per_row; s < n; s += per_row) M = fmaxf(M, base[s * stride + D]);
  if (per_row > 1) {
    if (d4 == 0) red_m[sg] = M;
    __syncthreads();
    for (int k = 0; k < per_row; ++k) M = fmaxf(M, red_m[sg - part + k]);
  }
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
  auto add = [&](f32x2 x, f32x4 y) {
    const float wt = fast_exp2((x.x - M) * a.scale_log2);
    acc += wt * y;
    den += wt * x.y;
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (part + k * per_row < n) add(ml[k], v[k]);
#pragma unroll 4
  for (int s = part + kAhead * per_row; s < n; s += per_row)
    add(*reinterpret_cast<const f32x2*>(base + s * stride + D), *reinterpret_cast<const f32x4*>(base + s * stride + d4));
  if (per_row > 1) {
    *reinterpret_cast<f32x4*>(&red_o[sg][d4]) = acc;
    if (d4 == 0) red_l[sg] = den;
    __syncthreads();
    if (part != 0) return;
    for (int k = 1; k < per_row; ++k) {
      acc += *reinterpret_cast<const f32x4*>(&red_o[sg + k][d4]);
      den += red_l[sg + k];
    }
  }
  if (r >= n_rows) return;
  const int n_q_heads = a.n_kv_heads << a.group_log2;
  uint16_t* row = a.out + (static_cast<size_t>(cd.q_row + (r >> a.group_log2)) * n_q_heads + (g << a.group_log2) + (r & ((1 << a.group_log2) - 1))) * D;
  const float inv = 1.f / den;
  st8(row + d4, make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)));
}

static RowsArgs make_rows_args(const PoolGeom& g, int layer, const SeenLaunch& w, const void* q, void* out, float* parts) {
  RowsArgs a;
  a.pool = static_cast<const uint16_t*>(g.pool);
  a.n_pages = g.n_pages;
  a.n_kv_heads = g.n_kv_heads;
  a.group_log2 = __builtin_ctz(static_cast<unsigned>(g.n_q_heads / g.n_kv_heads));
  a.layer = layer;
  a.page_table = g.page_table;
  a.max_pages = g.max_pages;
  a.meta = w.meta.dev;
  a.masks_off = static_cast<uint32_t>(w.masks_off);
  a.words_off = static_cast<uint32_t>(w.words_off);
  a.items_off = static_cast<uint32_t>(w.items_off);
  a.merges_off = static_cast<uint32_t>(w.merges_off);
  a.split = w.split;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.parts = parts;
  a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(g.head_dim)));
  return a;
}

hipError_t launch_seen_rows(const PoolGeom& g, int layer, const SeenLaunch& w, const void* q, void* out, float* parts,
                            hipStream_t stream) {
  if (w.n_items == 0) return hipSuccess;
  if (!w.meta.ok() || w.split < 32 || w.split % 32 || w.split > 1024 || (w.n_merges > 0 && parts == nullptr)) return hipErrorInvalidValue;
  const RowsArgs a = make_rows_args(g, layer, w, q, out, parts);
  const int64_t n_blocks = static_cast<int64_t>(w.n_items) * g.n_kv_heads;
  if (!grid_holds(n_blocks, 64 * kRowWaves)) return hipErrorInvalidConfiguration;
  LaunchMeta m;
  fill_meta(w.meta, &m);
  auto by_blocks = [&](auto d) {
    auto launch = [&](auto nb) {
      if (g.fp4) seen_rows_fp4_kernel<d(), nb()><<<static_cast<unsigned>(n_blocks), 64 * kRowWaves, 0, stream>>>(m, a);
      else seen_rows_kernel<d(), nb()><<<static_cast<unsigned>(n_blocks), 64 * kRowWaves, 0, stream>>>(m, a);
      return hipGetLastError();
    };
    if (w.blocks == 1) return launch(std::integral_constant<int, 1>{});
    if (w.blocks == 2) return launch(std::integral_constant<int, 2>{});
    if (w.blocks == 3) return launch(std::integral_constant<int, 3>{});
    if (w.blocks == 4) return launch(std::integral_constant<int, 4>{});
    return hipErrorInvalidValue;
  };
  if (g.head_dim == 128) return by_blocks(std::integral_constant<int, 128>{});
  if (g.head_dim == 64) return by_blocks(std::integral_constant<int, 64>{});
  return hipErrorInvalidValue;
}

hipError_t launch_seen_rows_merge(const PoolGeom& g, const SeenLaunch& w, void* out, float* parts, hipStream_t stream) {
  if (w.n_merges == 0) return hipSuccess;
  if (!w.meta.ok() || parts == nullptr) return hipErrorInvalidValue;
  const RowsArgs a = make_rows_args(g, 0, w, nullptr, out, parts);
  // record groups a row: as many as hold the most records of an entry, four each
  const int groups = 1024 / g.head_dim;
  int per_row = 1;
  while (per_row < groups && 4 * per_row < w.merge_items) per_row *= 2;
  const int rows = groups / per_row, row_groups = (w.merge_rows + rows - 1) / rows;
  const int64_t n_blocks = static_cast<int64_t>(w.n_merges) * row_groups * g.n_kv_heads;
  if (!grid_holds(n_blocks, 256)) return hipErrorInvalidConfiguration;
  LaunchMeta m;
  fill_meta(w.meta, &m);
  if (g.head_dim == 128) seen_rows_merge_kernel<128><<<static_cast<unsigned>(n_blocks), 256, 0, stream>>>(m, a, row_groups, per_row, 16 * w.blocks);
  else if (g.head_dim == 64) seen_rows_merge_kernel<64><<<static_cast<unsigned>(n_blocks), 256, 0, stream>>>(m, a, row_groups, per_row, 16 * w.blocks);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace cs
