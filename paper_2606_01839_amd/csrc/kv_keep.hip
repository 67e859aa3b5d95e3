// Keep of drafted tokens: of a conversation's last tokens the accepted ones move up to follow the cached ones, and the
// slots behind them in the last page become zeros. Pure byte movement.
//
// One wave per (conversation, layer, kv head) takes the pages that change in order. A token only ever moves to a lower
// slot, and those of a page come from that page or later ones, so a page may be written once its own tokens have been
// read, and no later page's are in it. The host gives physical pages, so what is waited for is one trip to memory for the
// sources' places and one for their bytes, a page; accepted drafts are one or two pages long.
// V lies dimension-major, 32 bytes a dim and page: whole rows of a source page are loaded and the tokens picked from registers (a
// 2-byte load for each token and dim keeps the address units busy for 41 of 85 us of 64 conversations, 32 layers, 8 kv heads). Of a page's rows
// the half of 8 slots in front of the first that changes is neither read nor written. 64 conversations, 32 layers, 8 kv heads: 44 us a
// call (104 MB read, 108 written); one conversation of 4 layers 4.5.
#include "device_common.hpp"
#include "fp4.hpp"
#include "kernels.hpp"

namespace cs {

struct KeepArgs {
  void* pool;
  int64_t n_pages;
  int n_kv_heads;
  const void* meta;
  uint32_t pages_off, src_off;
};

// Element u (wave-uniform) of the 16 that x and y hold.
__device__ __forceinline__ uint32_t pick16(uint4 x, uint4 y, int u) {
  const uint4 h = u & 8 ? y : x;
  const uint32_t a = u & 4 ? h.z : h.x, b = u & 4 ? h.w : h.y;
  return ((u & 2 ? b : a) >> (16 * (u & 1))) & 0xFFFFu;
}

template <int D, bool FP4>
__global__ __launch_bounds__(256) void kv_keep_kernel(LaunchMeta, KeepArgs a) {
  using B = Fp4Block<D>;
  constexpr int kCh = D / 8, kRows = 64 / kCh, kPasses = kPageTokens / kRows;
  const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int groups = a.n_kv_heads / waves;
  const int layer = blockIdx.y / groups, head = (blockIdx.y % groups) * waves + wave;
  const int ch = lane % kCh, t_lane = lane / kCh, col = lane & 15, qd = lane >> 4;
  const auto* pc = meta_at<KeepConv>(a.meta, 0) + blockIdx.x;
  const KeepConv c = {pc->page0, pc->n, pc->first, pc->len, pc->from, pc->src};
  const auto* pages = meta_at<int32_t>(a.meta, a.pages_off) + c.page0;
  const auto* src = meta_at<int64_t>(a.meta, a.src_off) + c.src;
  auto block16 = [&](int page) { return static_cast<uint16_t*>(a.pool) + block_elem<D>(layer, page, head, a.n_pages, a.n_kv_heads); };
  auto block4 = [&](int page) { return static_cast<uint8_t*>(a.pool) + B::at(layer, page, head, a.n_pages, a.n_kv_heads); };
  for (int lp = 0; lp < c.n; ++lp) {
    const int page = pages[lp], s0 = lp * kPageTokens;
    // lane t: the source of slot t of the page, page and slot; slots in front of `from` and behind the end have none
    int f_page = -1, f_t = 0;
    if (lane < kPageTokens && s0 + lane >= c.from && s0 + lane < c.len) {
      const int64_t f = src[s0 + lane - c.from];
      f_page = static_cast<int>(f / kPageTokens);
      f_t = static_cast<int>(f % kPageTokens);
    }
    auto page_of = [&](int t) { return __builtin_amdgcn_ds_bpermute(t << 2, f_page); };   // of a slot that differs by lane
    auto slot_of = [&](int t) { return __builtin_amdgcn_ds_bpermute(t << 2, f_t); };
    if constexpr (FP4) {
      uint8_t* dst = block4(page);
      uint32_t k[kPasses], ks[kPasses], vs[kPasses];
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows, fp = page_of(t), ft = slot_of(t);
        k[ps] = ks[ps] = vs[ps] = 0;
        if (fp >= 0 && s0 + t >= c.first) {
          const uint8_t* b = block4(fp);
          k[ps] = *reinterpret_cast<const uint32_t*>(b + B::k_word(ft, ch));
          ks[ps] = b[B::k_scale(ft, ch >> 2)];
          vs[ps] = b[B::kVScale + ft];
        }
      }
      // V: tokens 4 qd + i of the dims 16 t + col; those in front of `first` stay (they may lie in front of `from`)
      uint32_t* v = reinterpret_cast<uint32_t*>(dst + B::kV) + lane * B::kWords;
      const uint32_t stays = fp4_key_bits(qd, 0, c.first - s0);
      uint32_t w[B::kWords];
#pragma unroll
      for (int j = 0; j < B::kWords; ++j) w[j] = stays ? v[j] & stays : 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = 4 * qd + i, fp = page_of(t), ft = slot_of(t);
        if (fp < 0 || s0 + t < c.first) continue;
        const uint32_t* x = reinterpret_cast<const uint32_t*>(block4(fp) + B::kV) + ((ft / 4) * 16 + col) * B::kWords;
#pragma unroll
        for (int j = 0; j < B::kWords; ++j) w[j] |= ((x[j] >> (4 * (ft % 4))) & 0x000F000Fu) << (4 * i);
      }
      __builtin_amdgcn_sched_barrier(0);   // all of the page's loads before its stores
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows;
        if (s0 + t < c.first) continue;
        *reinterpret_cast<uint32_t*>(dst + B::k_word(t, ch)) = k[ps];
        if ((ch & 3) == 0) dst[B::k_scale(t, ch >> 2)] = static_cast<uint8_t>(ks[ps]);
        if (ch == 0) dst[B::kVScale + t] = static_cast<uint8_t>(vs[ps]);
      }
      if (~stays) {
        if constexpr (D == 128) st16(v, make_uint4(w[0], w[1], w[2], w[3]));
        else st8(v, make_uint2(w[0], w[1]));
      }
    } else {
      uint16_t* dst = block16(page);
      uint4 k[kPasses];
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows, fp = page_of(t), ft = slot_of(t);
        k[ps] = make_uint4(0, 0, 0, 0);
        if (fp >= 0 && s0 + t >= c.first) k[ps] = ld16(block16(fp) + k_elem(ft, ch));
      }
      uint32_t w[D / 64][8];
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = 0;
      // source pages one after the other, each of its slots' tokens picked
      int prev = -1;
      for (int t0 = max(c.from - s0, 0); t0 < min(c.len - s0, kPageTokens); ++t0) {
        const int sp = __builtin_amdgcn_readlane(f_page, t0);
        if (sp == prev) continue;
        prev = sp;
        const uint16_t* b = block16(sp) + kPageTokens * D;
        uint4 x[D / 64][2];
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) x[j][h] = ld16(b + (lane + 64 * j) * kPageTokens + 8 * h);
#pragma unroll
        for (int t = 0; t < kPageTokens; ++t) {
          if (__builtin_amdgcn_readlane(f_page, t) != sp) continue;
          const int u = __builtin_amdgcn_readlane(f_t, t);
#pragma unroll
          for (int j = 0; j < D / 64; ++j) w[j][t / 2] |= pick16(x[j][0], x[j][1], u) << (16 * (t % 2));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows;
        if (s0 + t >= c.first) st16(dst + k_elem(t, ch), k[ps]);
      }
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint16_t* row = dst + kPageTokens * D + (lane + 64 * j) * kPageTokens;
        if (s0 >= c.from) st16(row, make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]));
        st16(row + 8, make_uint4(w[j][4], w[j][5], w[j][6], w[j][7]));
      }
    }
  }
}

hipError_t launch_keep(const PoolGeom& g, const Meta& meta, size_t pages_off, size_t src_off, int n_convs, hipStream_t stream) {
  if (n_convs == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n_convs * sizeof(KeepConv) || meta.bytes < pages_off || meta.bytes < src_off) return hipErrorInvalidValue;
  KeepArgs a;
  a.pool = g.pool;
  a.n_pages = g.n_pages;
  a.n_kv_heads = g.n_kv_heads;
  a.meta = meta.dev;
  a.pages_off = static_cast<uint32_t>(pages_off);
  a.src_off = static_cast<uint32_t>(src_off);
  LaunchMeta m;
  fill_meta(meta, &m);
  const int waves = g.n_kv_heads % 4 == 0 ? 4 : (g.n_kv_heads % 2 == 0 ? 2 : 1);
  const dim3 grid(n_convs, g.n_layers * (g.n_kv_heads / waves));
  if (!grid_holds(static_cast<int64_t>(grid.x), 64 * waves)) return hipErrorInvalidConfiguration;
  if (g.head_dim == 128 && g.fp4) kv_keep_kernel<128, true><<<grid, 64 * waves, 0, stream>>>(m, a);
  else if (g.head_dim == 64 && g.fp4) kv_keep_kernel<64, true><<<grid, 64 * waves, 0, stream>>>(m, a);
  else if (g.head_dim == 128) kv_keep_kernel<128, false><<<grid, 64 * waves, 0, stream>>>(m, a);
  else if (g.head_dim == 64) kv_keep_kernel<64, false><<<grid, 64 * waves, 0, stream>>>(m, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace cs
