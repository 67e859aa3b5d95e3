// KV movement of 4-bit pools (block layout in fp4.hpp), and appends that rotate keys: new tokens into pages,
// a conversation into and out of the transfer's wire format, a bf16 pool's conversation into a 4-bit wire,
// tokens back out of the pages of either kind. All bound by HBM bytes.
#include <algorithm>

#include "device_common.hpp"
#include "fp4.hpp"
#include "kernels.hpp"
#include "rope.hpp"

namespace cs {

// Largest x over the 4 (8, 16) lanes of an aligned group; every lane of the group gets it.
__device__ __forceinline__ uint32_t dpp_max(uint32_t x, uint32_t y) { return x > y ? x : y; }
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  x = dpp_max(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true));                          // lane ^ 1
  x = dpp_max(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true));                          // lane ^ 2
  if constexpr (LANES >= 8) x = dpp_max(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true));   // 7 - lane of 8
  if constexpr (LANES >= 16) x = dpp_max(x, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, true));  // 15 - lane of 16
  return x;
}

__device__ __forceinline__ uint32_t max_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = dpp_max(m, abs_bits(x[i]));
  return m;
}

__device__ __forceinline__ PageChunk load_chunk(ConstPtr<PageChunk> p) {
  return {p->conv, p->slot, p->lpage, p->page, p->t0, p->t1, p->src_row, p->new_page};
}

// ---------------------------------------------------------------------------------------------
// Append. One wave per (layer, kv head) and kChunks page chunks; workgroups behind those of the K and V
// rotate the same chunks' queries. The workgroup first makes the (cos, sin) of its tokens' angles in LDS,
// one pair a lane: they serve all its heads. V goes through LDS to be written key-minor.
// A chunk that starts a page (t0 = 0) writes the whole block, zeros in slots [t1, 16); one that continues a
// page writes only its slots. Two tokens of a 4-bit page share a byte of V: the wave that owns the (page,
// head) puts its codes between the others'.
// Bound by HBM: 12.5k tokens of 32 layers, 8 kv heads of 128 into 4-bit pages (2.09 GB read and written, by the
// counters too) 350 us, 5.97 TB/s; 5.3k rotated into bf16 pages (1.39 GB) 236 us, 5.90 TB/s: the rotation costs nothing.
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
  const void* meta;
  uint32_t pos_off;   // positions of the tokens in meta; 0: their slots
  int n_chunks;
  int n_layers, n_kv_heads, n_q_heads;
  int kv_blocks;   // grid rows of the K and V; the queries' follow
  int q_groups;    // grid rows a layer of the queries
  int q_heads;     // query heads a workgroup rotates
  uint4* carry_dst;
  int carry_off, carry_n16;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q;
  uint16_t* q_out;
  int64_t src_rows;
  void* pool;
  int64_t n_pages;
  int32_t* page_table;
  int max_pages;
};

constexpr int kChunks = 2;
constexpr int kQHeads = 16;   // query heads a workgroup rotates

// (cos, sin) of the angles of rows [0, rows) into tab[row][D / 2]; pos(row) < 0: none
template <int D, typename Pos>
__device__ __forceinline__ void rope_table(f32x2 (*tab)[D / 2], int rows, const RopeArgs& r, int waves, Pos&& pos) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint64_t frac = lane < r.pairs ? meta_at<RopeArgs>(nullptr, sizeof(LaunchMeta))->frac[lane] : 0;
  for (int row = wave; row < rows; row += waves) {
    const int p = pos(row);
    if (p >= 0 && lane < r.pairs) tab[row][lane] = rope_turn(frac, static_cast<uint32_t>(p), r.amplitude);
  }
  __syncthreads();
}

template <int D, bool FP4, bool ROPE>
__global__ __launch_bounds__(256) void kv_append_as_kernel(LaunchMeta, RopeArgs rope, AppendArgs a) {
  using B = Fp4Block<D>;
  constexpr int kCh = D / 8;                 // lanes (16-byte pieces) per token row
  constexpr int kRows = 64 / kCh;            // token rows per pass
  constexpr int kPasses = kPageTokens / kRows;
  constexpr int CH = kChunks;
  __shared__ f32x2 tab[ROPE ? CH * kPageTokens : 1][D / 2];
  __shared__ uint32_t vts[4][CH][kPageTokens][FP4 ? kCh + 1 : D / 2 + 4];

  const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int ch = lane % kCh, t_lane = lane / kCh;

  if (a.carry_n16 > 0 && blockIdx.x == 0 && blockIdx.y == 0) {
    const auto* src = meta_at<u32x4_t>(nullptr, a.carry_off);
    for (int i = threadIdx.x; i < a.carry_n16; i += blockDim.x) {
      const u32x4_t x = src[i];
      a.carry_dst[i] = make_uint4(x.x, x.y, x.z, x.w);
    }
  }

  const auto* chunks = meta_at<PageChunk>(a.meta, 0);
  PageChunk c[CH];
  bool have[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int idx = blockIdx.x * CH + i;
    have[i] = idx < a.n_chunks;
    c[i] = load_chunk(chunks + (have[i] ? idx : 0));
  }
  // Position of row `lane` (a trip to memory for all rows of a tree, whose positions are not their slots: 26 tokens of 4 layers
  // 14.4 us with one for each row).
  int lane_pos = -1;
  if constexpr (ROPE) {
    const int t = lane % kPageTokens;
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (lane / kPageTokens == i && have[i] && t >= c[i].t0 && t < c[i].t1)
        lane_pos = a.pos_off ? meta_at<int32_t>(a.meta, a.pos_off)[(blockIdx.x * CH + i) * kPageTokens + t] : c[i].lpage * kPageTokens + t;
  }
  auto row_pos = [&](int row) { return __builtin_amdgcn_readlane(lane_pos, row); };
  // 16 bytes of row t of a chunk: [layer][row][head][D] + 8 ch
  auto row_at = [&](int layer, int i, int t, int n_heads, int head) {
    const size_t row = static_cast<size_t>(c[i].src_row) + static_cast<size_t>(t - c[i].t0);
    return ((static_cast<size_t>(layer) * static_cast<size_t>(a.src_rows) + row) * n_heads + head) * D + ch * 8;
  };

  if (ROPE && static_cast<int>(blockIdx.y) >= a.kv_blocks) {
    rope_table<D>(tab, CH * kPageTokens, rope, waves, row_pos);
    const int y = blockIdx.y - a.kv_blocks;
    const int layer = y / a.q_groups, h0 = y % a.q_groups * a.q_heads;
    for (int h = h0 + wave; h < min(h0 + a.q_heads, a.n_q_heads); h += waves) {
      uint4 x[CH][kPasses];
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int ps = 0; ps < kPasses; ++ps) {
          const int t = t_lane + ps * kRows;
          x[i][ps] = make_uint4(0, 0, 0, 0);
          if (have[i] && t >= c[i].t0 && t < c[i].t1) x[i][ps] = ld16(a.q + row_at(layer, i, t, a.n_q_heads, h));
        }
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int ps = 0; ps < kPasses; ++ps) {
          const int t = t_lane + ps * kRows;
          float f[8];
          unpack8(x[i][ps], f);
          rope_rotate<D>(f, ch, rope, tab[i * kPageTokens + t]);
          if (have[i] && t >= c[i].t0 && t < c[i].t1) st16_nt(a.q_out + row_at(layer, i, t, a.n_q_heads, h), pack8(f));
        }
    }
    return;
  }

  const int groups = a.n_kv_heads / waves;
  const int layer = blockIdx.y / groups;
  const int head = (blockIdx.y % groups) * waves + wave;
  uint4 kv[CH][kPasses], vv[CH][kPasses];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int ps = 0; ps < kPasses; ++ps) {
      const int t = t_lane + ps * kRows;
      kv[i][ps] = vv[i][ps] = make_uint4(0, 0, 0, 0);
      if (have[i] && t >= c[i].t0 && t < c[i].t1) {
        const size_t src = row_at(layer, i, t, a.n_kv_heads, head);
        kv[i][ps] = FP4 ? ld16_nt(a.k + src) : ld16(a.k + src);
        vv[i][ps] = FP4 ? ld16_nt(a.v + src) : ld16(a.v + src);
      }
    }
  if constexpr (ROPE) rope_table<D>(tab, CH * kPageTokens, rope, waves, row_pos);

#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (!have[i]) continue;
    const bool starts = c[i].t0 == 0;
    uint16_t* blk16 = static_cast<uint16_t*>(a.pool) + block_elem<D>(layer, c[i].page, head, a.n_pages, a.n_kv_heads);
    uint8_t* blk = static_cast<uint8_t*>(a.pool) + B::at(layer, c[i].page, head, a.n_pages, a.n_kv_heads);
#pragma unroll
    for (int ps = 0; ps < kPasses; ++ps) {
      const int t = t_lane + ps * kRows;
      const bool in = t >= c[i].t0 && t < c[i].t1;
      const bool writes = in || (starts && t >= c[i].t1);
      float x[8];
      if (FP4 || ROPE) unpack8(kv[i][ps], x);
      if constexpr (ROPE) {
        rope_rotate<D>(x, ch, rope, tab[i * kPageTokens + t]);
        if (!in) {   // (rows without a token have no angles)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
        }
      }
      if constexpr (FP4) {
        const uint32_t kb = fp4_scale_byte(group_max<4>(max_bits(x)));
        const uint32_t codes = fp4_encode8(x, fp4_scale(kb));
        if (writes) {
          *reinterpret_cast<uint32_t*>(blk + B::k_word(t, ch)) = codes;
          if ((ch & 3) == 0) blk[B::k_scale(t, ch >> 2)] = static_cast<uint8_t>(in ? kb : 0);
        }
        unpack8(vv[i][ps], x);
        const uint32_t vb = fp4_scale_byte(group_max<kCh>(max_bits(x)));
        vts[wave][i][t][ch] = vb == 255 ? 0u : fp4_encode8(x, fp4_scale(vb));
        if (writes && ch == 0) blk[B::kVScale + t] = static_cast<uint8_t>(in ? vb : 0);
      } else {
        if (writes) st16(blk16 + k_elem(t, ch), ROPE ? pack8(x) : kv[i][ps]);
        st16(&vts[wave][i][t][ch * 4], vv[i][ps]);
      }
    }
    if (FP4 && starts && lane < (B::kBytes - B::kPad) / 16) st16(blk + B::kPad + 16 * lane, make_uint4(0, 0, 0, 0));
  }
  __syncthreads();

#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (!have[i]) continue;
    const auto& vt = vts[wave][i];
    if constexpr (FP4) {
      uint8_t* blk = static_cast<uint8_t*>(a.pool) + B::at(layer, c[i].page, head, a.n_pages, a.n_kv_heads);
      const int col = lane & 15, qd = lane >> 4;
      uint32_t* dst = reinterpret_cast<uint32_t*>(blk + B::kV) + lane * B::kWords;
      const uint32_t keep = c[i].t0 == 0 ? ~0u : fp4_key_bits(qd, c[i].t0, c[i].t1);
      uint32_t w[B::kWords];
#pragma unroll
      for (int j = 0; j < B::kWords; ++j) {
        w[j] = 0;
#pragma unroll
        for (int s = 0; s < 8; ++s) {   // tile 2 j + s / 4, key 4 qd + s % 4
          const uint32_t x = vt[4 * qd + s % 4][2 * (2 * j + s / 4) + (col >> 3)] >> (4 * (col & 7));
          w[j] |= (x & 15u) << (4 * s);
        }
      }
      if (keep != 0) {
        if (keep != ~0u) {
#pragma unroll
          for (int j = 0; j < B::kWords; ++j) w[j] = (dst[j] & ~keep) | (w[j] & keep);
        }
        if constexpr (D == 128) st16_nt(dst, make_uint4(w[0], w[1], w[2], w[3]));
        else st8(dst, make_uint2(w[0], w[1]));
      }
    } else {
      uint16_t* vdst = static_cast<uint16_t*>(a.pool) + block_elem<D>(layer, c[i].page, head, a.n_pages, a.n_kv_heads) +
                       kPageTokens * D;
#pragma unroll
      for (int e = lane; e < D; e += 64) {
        uint16_t* row = vdst + e * kPageTokens;
        auto at = [&](int t) { return static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(&vt[t][0])[e]); };
        if (c[i].t0 == 0) {
          uint32_t w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = at(2 * j) | at(2 * j + 1) << 16;
          st16(row, make_uint4(w[0], w[1], w[2], w[3]));
          st16(row + 8, make_uint4(w[4], w[5], w[6], w[7]));
        } else {
          for (int t = c[i].t0; t < c[i].t1; ++t) row[t] = static_cast<uint16_t>(at(t));
        }
      }
    }
    if (c[i].new_page && blockIdx.y == 0 && threadIdx.x == 0)
      a.page_table[static_cast<size_t>(c[i].slot) * a.max_pages + c[i].lpage] = c[i].page;
  }
}

// ---------------------------------------------------------------------------------------------
// Queries rotated at their positions: 16 rows and kQHeads heads per workgroup. Bound by HBM: 5.69 TB/s read and
// written over 1.4 GB of queries (a copy: 5.76). NT: streaming loads, for queries that the last-level cache (256 MB)
// cannot hold beside the output: 1.4 GB 488 us against 505 with plain loads, but 131 MB that a kernel before has just written
// 50.6 against 44.8.
// ---------------------------------------------------------------------------------------------
constexpr size_t kRopeStreamBytes = size_t(128) << 20;

template <int D, bool NT>
__global__ __launch_bounds__(256) void rope_q_kernel(LaunchMeta, RopeArgs rope, const void* meta, int n_convs, int64_t rows,
                                                     int n_q_heads, int q_groups, const uint16_t* q,
                                                     uint16_t* out) {
  constexpr int kCh = D / 8, kRows = 64 / kCh, kPasses = kPageTokens / kRows;
  __shared__ f32x2 tab[kPageTokens][D / 2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int ch = lane % kCh, t_lane = lane / kCh;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kPageTokens;
  const auto* convs = meta_at<RopeConv>(meta, 0);
  rope_table<D>(tab, kPageTokens, rope, 4, [&](int t) {
    const int64_t row = row0 + t;
    if (row >= rows) return -1;
    if (n_convs == 0) return static_cast<int>(meta_at<int32_t>(meta, 0)[row]);
    int lo = 0, hi = n_convs - 1;   // the last conversation that starts at or before the row
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (convs[mid].row <= row) lo = mid; else hi = mid - 1;
    }
    return static_cast<int>(convs[lo].pos + (row - convs[lo].row));
  });
  const int layer = blockIdx.y / q_groups, h0 = blockIdx.y % q_groups * kQHeads;
  for (int h = h0 + wave; h < min(h0 + kQHeads, n_q_heads); h += 4) {
    uint4 x[kPasses];
    auto at = [&](int t) { return ((static_cast<size_t>(layer) * rows + row0 + t) * n_q_heads + h) * D + ch * 8; };
#pragma unroll
    for (int ps = 0; ps < kPasses; ++ps) {
      const int t = t_lane + ps * kRows;
      x[ps] = make_uint4(0, 0, 0, 0);
      if (row0 + t < rows) x[ps] = NT ? ld16_nt(q + at(t)) : ld16(q + at(t));
    }
#pragma unroll
    for (int ps = 0; ps < kPasses; ++ps) {
      const int t = t_lane + ps * kRows;
      float f[8];
      unpack8(x[ps], f);
      rope_rotate<D>(f, ch, rope, tab[t]);
      if (row0 + t < rows) st16_nt(out + at(t), pack8(f));
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Read back: one wave per (chunk, layer, kv head); V through LDS into token rows. Bound by HBM: 12.5k tokens of 32
// layers, 8 kv heads of 128 out of 4-bit pages (2.09 GB read and written) 382 us, 5.47 TB/s; 5.3k out of bf16 pages (1.39 GB)
// 243 us, 5.73 TB/s (283 with the K loads behind the V part and the cached forms).
// ---------------------------------------------------------------------------------------------
template <int D, bool FP4>
__global__ __launch_bounds__(256) void kv_read_kernel(LaunchMeta, const void* meta, int n_kv_heads, const void* pool,
                                                      int64_t n_pages, uint16_t* __restrict__ k, uint16_t* __restrict__ v,
                                                      int64_t dst_rows) {
  using B = Fp4Block<D>;
  constexpr int kCh = D / 8, kRows = 64 / kCh, kPasses = kPageTokens / kRows;
  __shared__ uint32_t vts[4][kPageTokens][D / 2 + 4];
  const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int groups = n_kv_heads / waves;
  const int layer = blockIdx.y / groups, head = (blockIdx.y % groups) * waves + wave;
  const int ch = lane % kCh, t_lane = lane / kCh;
  const PageChunk c = load_chunk(meta_at<PageChunk>(meta, 0) + blockIdx.x);
  const uint16_t* blk16 = static_cast<const uint16_t*>(pool) + block_elem<D>(layer, c.page, head, n_pages, n_kv_heads);
  const uint8_t* blk = static_cast<const uint8_t*>(pool) + B::at(layer, c.page, head, n_pages, n_kv_heads);
  auto at = [&](int t) {
    return ((static_cast<size_t>(layer) * dst_rows + c.src_row + (t - c.t0)) * n_kv_heads + head) * D + ch * 8;
  };
  uint16_t* vt = reinterpret_cast<uint16_t*>(&vts[wave][0][0]);
  constexpr int kStride = D + 8;
  // all loads before the first store (a chunk's pages are whole: slots outside [t0, t1) are read too)
  uint4 kx[kPasses];
  uint32_t kw[kPasses], kb[kPasses];
#pragma unroll
  for (int ps = 0; ps < kPasses; ++ps) {
    const int t = t_lane + ps * kRows;
    if constexpr (FP4) {
      kw[ps] = *reinterpret_cast<const uint32_t*>(blk + B::k_word(t, ch));
      kb[ps] = blk[B::k_scale(t, ch >> 2)];
    } else {
      kx[ps] = ld16_nt(blk16 + k_elem(t, ch));
    }
  }
  if constexpr (FP4) {
    const int col = lane & 15, qd = lane >> 4;
    uint32_t w[B::kWords];
    if constexpr (D == 128) {
      const uint4 x = ld16(blk + B::kV + 16 * lane);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else {
      const uint2 x = ld8(blk + B::kV + 8 * lane);
      w[0] = x.x, w[1] = x.y;
    }
    const uint32_t vs = *reinterpret_cast<const uint32_t*>(blk + B::kVScale + 4 * qd);
    __builtin_amdgcn_sched_barrier(0);
    const float s[4] = {fp4_scale_of(vs, 0), fp4_scale_of(vs, 1), fp4_scale_of(vs, 2), fp4_scale_of(vs, 3)};
#pragma unroll
    for (int j = 0; j < B::kWords; ++j) {
      const uint2 lo = fp4_quad<0>(w[j], s), hi = fp4_quad<1>(w[j], s);
      const uint32_t x[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
      for (int e = 0; e < 8; ++e)   // tile 2 j + e / 4, key 4 qd + e % 4
        vt[(4 * qd + e % 4) * kStride + 16 * (2 * j + e / 4) + col] = static_cast<uint16_t>(x[e / 2] >> (16 * (e % 2)));
    }
  } else {
    uint4 r[D / 64][2];
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) r[i][h] = ld16_nt(blk16 + kPageTokens * D + (lane + 64 * i) * kPageTokens + 8 * h);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint32_t x[8] = {r[i][0].x, r[i][0].y, r[i][0].z, r[i][0].w, r[i][1].x, r[i][1].y, r[i][1].z, r[i][1].w};
#pragma unroll
      for (int t = 0; t < kPageTokens; ++t) vt[t * kStride + lane + 64 * i] = static_cast<uint16_t>(x[t / 2] >> (16 * (t % 2)));
    }
  }
#pragma unroll
  for (int ps = 0; ps < kPasses; ++ps) {
    const int t = t_lane + ps * kRows;
    if (t >= c.t0 && t < c.t1) st16_nt(k + at(t), FP4 ? fp4_word(kw[ps], fp4_scale(kb[ps])) : kx[ps]);
  }
  __syncthreads();
#pragma unroll
  for (int ps = 0; ps < kPasses; ++ps) {
    const int t = t_lane + ps * kRows;
    if (t >= c.t0 && t < c.t1) st16_nt(v + at(t), ld16(vt + t * kStride + ch * 8));
  }
}

// ---------------------------------------------------------------------------------------------
// Pack and unpack of 4-bit pages: the blocks of a page's heads lie one after the other in the pool and in
// the wire alike, so a workgroup copies one (layer, page) of all heads. Bound by HBM: 3.8k tokens of 32 layers
// unpacked (264 MB read and written) 49 us, 5.41 TB/s.
// ---------------------------------------------------------------------------------------------
// Word w of a block with the token slots >= valid zeroed.
template <int D>
__device__ __forceinline__ uint32_t fp4_mask_word(uint32_t x, int w, int valid) {
  using B = Fp4Block<D>;
  if (4 * w < B::kV) return (w / 4) % kPageTokens < valid ? x : 0u;
  if (4 * w < B::kKScale) return x & fp4_key_bits((w - B::kV / 4) / (16 * B::kWords), 0, valid);
  if (4 * w >= B::kPad) return 0u;
  // the scales of a token's K (D = 64: of two tokens'), or of four tokens' V
  const bool is_v = 4 * w >= B::kVScale;
  const int bytes = is_v ? 1 : D / 32;                                  // of a token
  const int t = is_v ? 4 * w - B::kVScale : (4 * w - B::kKScale) / bytes;   // the first token
  const int n = (valid - t) * bytes;                                    // bytes to keep
  return n >= 4 ? x : n <= 0 ? 0u : x & ((1u << (8 * n)) - 1u);
}

template <int D>
__device__ __forceinline__ void fp4_copy_page(const uint8_t* src, uint8_t* dst, int n_kv_heads, int valid) {
  constexpr int kPieces = Fp4Block<D>::kBytes / 16;
  for (int i = threadIdx.x; i < n_kv_heads * kPieces; i += blockDim.x) {
    uint4 x = ld16_nt(src + 16 * static_cast<size_t>(i));
    if (valid < kPageTokens) {
      const int w = i % kPieces * 4;
      x = make_uint4(fp4_mask_word<D>(x.x, w, valid), fp4_mask_word<D>(x.y, w + 1, valid), fp4_mask_word<D>(x.z, w + 2, valid),
                     fp4_mask_word<D>(x.w, w + 3, valid));
    }
    st16_nt(dst + 16 * static_cast<size_t>(i), x);
  }
}

__device__ __forceinline__ int valid_tokens(int64_t len, int lpage) {
  const int64_t rem = len - static_cast<int64_t>(lpage) * kPageTokens;
  return rem < kPageTokens ? static_cast<int>(rem) : kPageTokens;
}

template <int D>
__global__ __launch_bounds__(256) void kv_pack_same_fp4_kernel(const uint8_t* __restrict__ pool, int64_t n_pages, int n_kv_heads,
                                                               const int32_t* __restrict__ pt_row, int64_t len,
                                                               uint8_t* __restrict__ wire, int n_lpages, int lp0) {
  using B = Fp4Block<D>;
  const int lp = lp0 + blockIdx.x, layer = blockIdx.y;
  fp4_copy_page<D>(pool + B::at(layer, pt_row[lp], 0, n_pages, n_kv_heads), wire + B::at(layer, lp, 0, n_lpages, n_kv_heads),
                   n_kv_heads, valid_tokens(len, lp));
}

template <int D>
__global__ __launch_bounds__(256) void kv_unpack_fp4_kernel(LaunchMeta, const uint8_t* __restrict__ wire, const void* meta,
                                                            int64_t len, uint8_t* __restrict__ pool, int64_t n_pages,
                                                            int n_kv_heads, int32_t* __restrict__ pt_row, int n_lpages, int lp0) {
  using B = Fp4Block<D>;
  const int lp = lp0 + blockIdx.x, layer = blockIdx.y;
  const int page = meta_at<int32_t>(meta, 0)[blockIdx.x];
  fp4_copy_page<D>(wire + B::at(layer, lp, 0, n_lpages, n_kv_heads), pool + B::at(layer, page, 0, n_pages, n_kv_heads), n_kv_heads,
                   valid_tokens(len, lp));
  if (blockIdx.y == 0 && threadIdx.x == 0) pt_row[lp] = page;
}

// ---------------------------------------------------------------------------------------------
// Pack of a bf16 pool's conversation in 4 bits: one wave per (logical page, layer, kv head). Nothing is
// transposed: the bf16 block too has K in groups of 32 dims, token by token (lane = 4 token + a quarter of the
// group, a word of codes each), and V by dims (a lane loads the four tokens' values whose codes it holds). The scale
// of a K group needs 4 lanes, that of a V token the 16 lanes of a row. Bound by HBM: 3.8k tokens of 32 layers, 8 kv
// heads of 128 (629 MB read and written) 105 us, 5.98 TB/s.
// ---------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void kv_pack_fp4_kernel(const uint16_t* __restrict__ pool, int64_t n_pages, int n_kv_heads,
                                                          const int32_t* __restrict__ pt_row, int64_t len,
                                                          uint8_t* __restrict__ wire, int n_lpages, int lp0) {
  using B = Fp4Block<D>;
  constexpr int NW = B::kWords;
  const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, qd = lane >> 4;
  const int groups = n_kv_heads / waves;
  const int lp = lp0 + blockIdx.x, layer = blockIdx.y / groups, head = (blockIdx.y % groups) * waves + wave;
  const uint16_t* src = pool + block_elem<D>(layer, pt_row[lp], head, n_pages, n_kv_heads);
  uint8_t* dst = wire + B::at(layer, lp, head, n_lpages, n_kv_heads);
  const int valid = valid_tokens(len, lp);

  uint4 kx[NW];
  uint2 vx[2 * NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) kx[i] = ld16_nt(src + 512 * i + 8 * lane);
#pragma unroll
  for (int t = 0; t < 2 * NW; ++t) vx[t] = ld8_nt(src + kPageTokens * D + (16 * t + c) * kPageTokens + 4 * qd);

  // K: token lane / 4, dims 32 i + 8 (lane % 4) ..
  const bool k_in = lane / 4 < valid;
  uint32_t kb = 0, kw[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    float f[8];
    if (!k_in) kx[i] = make_uint4(0, 0, 0, 0);
    unpack8(kx[i], f);
    const uint32_t b = fp4_scale_byte(group_max<4>(max_bits(f)));
    kw[i] = fp4_encode8(f, fp4_scale(b));
    kb |= (k_in ? b : 0u) << (8 * i);
  }
  // V: keys 4 qd .. 4 qd + 3 of dims 16 t + c
  uint32_t vm[4] = {0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < 2 * NW; ++t) {
    vx[t].x = mask_bf16x2(vx[t].x, 4 * qd < valid, 4 * qd + 1 < valid);
    vx[t].y = mask_bf16x2(vx[t].y, 4 * qd + 2 < valid, 4 * qd + 3 < valid);
    vm[0] = dpp_max(vm[0], abs_bits(bf16_lo(vx[t].x)));
    vm[1] = dpp_max(vm[1], abs_bits(bf16_hi(vx[t].x)));
    vm[2] = dpp_max(vm[2], abs_bits(bf16_lo(vx[t].y)));
    vm[3] = dpp_max(vm[3], abs_bits(bf16_hi(vx[t].y)));
  }
  uint32_t vb = 0, held = 0;
  float inv[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t b = fp4_scale_byte(group_max<16>(vm[k]));
    vb |= (4 * qd + k < valid ? b : 0u) << (8 * k);
    held |= (b == 255 ? 0u : 0x000F000Fu) << (4 * k);
    inv[k] = fp4_scale(254 - min(b, 253u));   // exact: 1 / scale
  }
  uint32_t vw[NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    const uint2 a = vx[2 * j], b = vx[2 * j + 1];
    const float x[8] = {bf16_lo(a.x) * inv[0], bf16_hi(a.x) * inv[1], bf16_lo(a.y) * inv[2], bf16_hi(a.y) * inv[3],
                        bf16_lo(b.x) * inv[0], bf16_hi(b.x) * inv[1], bf16_lo(b.y) * inv[2], bf16_hi(b.y) * inv[3]};
    vw[j] = fp4_encode8(x, 1.f) & held;
  }
#pragma unroll
  for (int i = 0; i < NW; ++i) *reinterpret_cast<uint32_t*>(dst + B::kK + 256 * i + 4 * lane) = kw[i];
  if constexpr (D == 128) st16_nt(dst + B::kV + 16 * lane, make_uint4(vw[0], vw[1], vw[2], vw[3]));
  else st8(dst + B::kV + 8 * lane, make_uint2(vw[0], vw[1]));
  if ((lane & 3) == 0) {
    if constexpr (D == 128) *reinterpret_cast<uint32_t*>(dst + B::kKScale + lane) = kb;
    else *reinterpret_cast<uint16_t*>(dst + B::kKScale + lane / 2) = static_cast<uint16_t>(kb);
  }
  if (c == 0) *reinterpret_cast<uint32_t*>(dst + B::kVScale + 4 * qd) = vb;
  if (lane < (B::kBytes - B::kPad) / 16) st16(dst + B::kPad + 16 * lane, make_uint4(0, 0, 0, 0));
}

// ---------------------------------------------------------------------------------------------
template <typename F>
static hipError_t by_dim(int D, F&& f) {
  if (D == 64) return f(std::integral_constant<int, 64>{});
  if (D == 128) return f(std::integral_constant<int, 128>{});
  return hipErrorInvalidValue;
}

// kv heads (waves) per workgroup: 4, 2 or 1, whichever is the largest that divides n_kv_heads
static int head_waves(int n_kv_heads) { return n_kv_heads % 4 == 0 ? 4 : (n_kv_heads % 2 == 0 ? 2 : 1); }

hipError_t launch_append_as(const PoolGeom& g, const Meta& meta, int n_chunks, const AppendCarry& carry, const RopeArgs* rope,
                            const void* k, const void* v, const void* q, void* q_out, int64_t src_rows, size_t pos_off,
                            hipStream_t stream) {
  if (n_chunks == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n_chunks * sizeof(PageChunk)) return hipErrorInvalidValue;
  if (pos_off > 0 && (rope == nullptr || meta.bytes < pos_off + n_chunks * kPageTokens * sizeof(int32_t))) return hipErrorInvalidValue;
  if (carry.bytes > 0 && (meta.dev != nullptr || carry.dst == nullptr || carry.off % 16 || carry.bytes % 16 ||
                          carry.off + carry.bytes > meta.bytes))
    return hipErrorInvalidValue;
  if (rope != nullptr && (rope->pairs < 8 || rope->pairs % 8 || 2 * rope->pairs > g.head_dim)) return hipErrorInvalidValue;
  if (rope == nullptr && (q != nullptr || !g.fp4)) return hipErrorInvalidValue;
  LaunchMeta m;
  fill_meta(meta, &m);
  const int waves = head_waves(g.n_kv_heads);
  AppendArgs a{};
  a.meta = meta.dev;
  a.pos_off = static_cast<uint32_t>(pos_off);
  a.n_chunks = n_chunks;
  a.n_layers = g.n_layers;
  a.n_kv_heads = g.n_kv_heads;
  a.n_q_heads = g.n_q_heads;
  a.kv_blocks = g.n_layers * (g.n_kv_heads / waves);
  // One head a wave where that leaves CUs without work: a wave's heads come one after the other.
  const int64_t chunk_groups = (n_chunks + kChunks - 1) / kChunks;
  a.q_heads = chunk_groups * g.n_layers * ((g.n_q_heads + waves - 1) / waves) <= kCus ? waves : kQHeads;
  a.q_groups = (g.n_q_heads + a.q_heads - 1) / a.q_heads;
  a.carry_dst = static_cast<uint4*>(carry.dst);
  a.carry_off = static_cast<int>(carry.off);
  a.carry_n16 = static_cast<int>(carry.bytes / 16);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.src_rows = src_rows;
  a.pool = g.pool;
  a.n_pages = g.n_pages;
  a.page_table = g.page_table;
  a.max_pages = g.max_pages;
  const dim3 grid((n_chunks + kChunks - 1) / kChunks, a.kv_blocks + (q != nullptr ? g.n_layers * a.q_groups : 0));
  return by_dim(g.head_dim, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    const RopeArgs r = rope ? *rope : RopeArgs{};
    if (!g.fp4) kv_append_as_kernel<D, false, true><<<grid, 64 * waves, 0, stream>>>(m, r, a);
    else if (rope) kv_append_as_kernel<D, true, true><<<grid, 64 * waves, 0, stream>>>(m, r, a);
    else kv_append_as_kernel<D, true, false><<<grid, 64 * waves, 0, stream>>>(m, r, a);
    return hipGetLastError();
  });
}

int64_t append_rope_groups(const PoolGeom& g, size_t n_chunks) {
  return static_cast<int64_t>((n_chunks + kChunks - 1) / kChunks) * g.n_layers * ((g.n_q_heads + kQHeads - 1) / kQHeads);
}

int rope_q_layers(const PoolGeom& g) { return std::max(1, 65535 / ((g.n_q_heads + kQHeads - 1) / kQHeads)); }

hipError_t launch_rope_q(const PoolGeom& g, const Meta& meta, int n_convs, int64_t rows, int n_layers, const RopeArgs& rope,
                         const void* q, void* out, hipStream_t stream) {
  if (rows == 0 || n_layers == 0) return hipSuccess;
  if (n_convs < 0 || !meta.ok() || meta.bytes < (n_convs > 0 ? n_convs * sizeof(RopeConv) : rows * sizeof(int32_t)))
    return hipErrorInvalidValue;
  if (rope.pairs < 8 || rope.pairs % 8 || 2 * rope.pairs > g.head_dim) return hipErrorInvalidValue;
  LaunchMeta m;
  fill_meta(meta, &m);
  const int q_groups = (g.n_q_heads + kQHeads - 1) / kQHeads;
  const dim3 grid(static_cast<unsigned>((rows + kPageTokens - 1) / kPageTokens), n_layers * q_groups);
  return by_dim(g.head_dim, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    auto launch = [&](auto kernel) {
      kernel<<<grid, 256, 0, stream>>>(m, rope, meta.dev, n_convs, rows, g.n_q_heads, q_groups,
                                       static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out));
      return hipGetLastError();
    };
    const size_t bytes = static_cast<size_t>(rows) * n_layers * g.n_q_heads * D * 2;
    return bytes > kRopeStreamBytes ? launch(rope_q_kernel<D, true>) : launch(rope_q_kernel<D, false>);
  });
}

hipError_t launch_read(const PoolGeom& g, const Meta& meta, int n_chunks, void* k, void* v, int64_t dst_rows, hipStream_t stream) {
  if (n_chunks == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n_chunks * sizeof(PageChunk)) return hipErrorInvalidValue;
  LaunchMeta m;
  fill_meta(meta, &m);
  const int waves = head_waves(g.n_kv_heads);
  const dim3 grid(n_chunks, g.n_layers * (g.n_kv_heads / waves));
  return by_dim(g.head_dim, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    auto launch = [&](auto kernel) {
      kernel<<<grid, 64 * waves, 0, stream>>>(m, meta.dev, g.n_kv_heads, g.pool, g.n_pages, static_cast<uint16_t*>(k),
                                              static_cast<uint16_t*>(v), dst_rows);
      return hipGetLastError();
    };
    return g.fp4 ? launch(kv_read_kernel<D, true>) : launch(kv_read_kernel<D, false>);
  });
}

hipError_t launch_pack_fp4(const PoolGeom& g, int slot, int64_t len, int lp0, int n_lp, void* wire, hipStream_t stream) {
  if (n_lp == 0) return hipSuccess;
  const int n_lpages = static_cast<int>(pages_for(len));
  const int32_t* pt_row = g.page_table + static_cast<size_t>(slot) * g.max_pages;
  const int waves = head_waves(g.n_kv_heads);
  return by_dim(g.head_dim, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    if (g.fp4)
      kv_pack_same_fp4_kernel<D><<<dim3(n_lp, g.n_layers), 256, 0, stream>>>(
          static_cast<const uint8_t*>(g.pool), g.n_pages, g.n_kv_heads, pt_row, len, static_cast<uint8_t*>(wire), n_lpages, lp0);
    else
      kv_pack_fp4_kernel<D><<<dim3(n_lp, g.n_layers * (g.n_kv_heads / waves)), 64 * waves, 0, stream>>>(
          static_cast<const uint16_t*>(g.pool), g.n_pages, g.n_kv_heads, pt_row, len, static_cast<uint8_t*>(wire), n_lpages, lp0);
    return hipGetLastError();
  });
}

hipError_t launch_unpack_fp4(const PoolGeom& g, const void* wire, const Meta& meta, int slot, int64_t len, int lp0, int n_lp,
                             hipStream_t stream) {
  if (n_lp == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n_lp * sizeof(int32_t)) return hipErrorInvalidValue;
  LaunchMeta m;
  fill_meta(meta, &m);
  return by_dim(g.head_dim, [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    kv_unpack_fp4_kernel<D><<<dim3(n_lp, g.n_layers), 256, 0, stream>>>(
        m, static_cast<const uint8_t*>(wire), meta.dev, len, static_cast<uint8_t*>(g.pool), g.n_pages, g.n_kv_heads,
        g.page_table + static_cast<size_t>(slot) * g.max_pages, static_cast<int>(pages_for(len)), lp0);
    return hipGetLastError();
  });
}

}  // namespace cs
