// Keep of drafted tokens: of a conversation's last tokens the accepted ones move up to follow the cached ones, and the
// slots behind them in the last page become zeros. Pure byte movement.
//
// One wave per (conversation, layer, kv head) takes the pages that change in order. A token only ever moves to a lower
// slot, and those of a page come from that page or later ones, so a page may be written once its own tokens have been
// read, and no later page's are in it. What bounds it is that chain, one trip to memory for the sources' pages and one
// for the tokens a page: accepted drafts are one or two pages long.
#include "device_common.hpp"
#include "fp4.hpp"
#include "kernels.hpp"

namespace cs {

struct KeepArgs {
  void* pool;
  int64_t n_pages;
  int n_kv_heads;
  const int32_t* page_table;
  int max_pages;
  const void* meta;
  uint32_t src_off;
};

template <int D, bool FP4>
__global__ __launch_bounds__(256) void kv_keep_kernel(LaunchMeta, KeepArgs a) {
  using B = Fp4Block<D>;
  constexpr int kCh = D / 8, kRows = 64 / kCh, kPasses = kPageTokens / kRows;
  const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int groups = a.n_kv_heads / waves;
  const int layer = blockIdx.y / groups, head = (blockIdx.y % groups) * waves + wave;
  const int ch = lane % kCh, t_lane = lane / kCh, col = lane & 15, qd = lane >> 4;
  const auto* pc = meta_at<KeepConv>(a.meta, 0) + blockIdx.x;
  const KeepConv c = {pc->slot, pc->lp0, pc->n_lp, pc->first, pc->len, pc->src};
  const auto* src = meta_at<int32_t>(a.meta, a.src_off) + c.src;
  const int32_t* pt = a.page_table + static_cast<size_t>(c.slot) * a.max_pages;
  auto block16 = [&](int page) { return static_cast<uint16_t*>(a.pool) + block_elem<D>(layer, page, head, a.n_pages, a.n_kv_heads); };
  auto block4 = [&](int page) { return static_cast<uint8_t*>(a.pool) + B::at(layer, page, head, a.n_pages, a.n_kv_heads); };
  for (int lp = c.lp0; lp < c.lp0 + c.n_lp; ++lp) {
    const int page = pt[lp], s0 = lp * kPageTokens;
    // slot -> its source (slots [first, len)), or itself
    auto from = [&](int s) { return s >= c.first && s < c.len ? src[s - c.first] : s; };
    auto writes = [&](int s) { return s >= c.first; };
    if constexpr (FP4) {
      uint8_t* dst = block4(page);
      uint32_t k[kPasses], ks[kPasses], vs[kPasses];
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int s = s0 + t_lane + ps * kRows, f = from(s), t = f % kPageTokens;
        const uint8_t* b = block4(pt[f / kPageTokens]);
        k[ps] = ks[ps] = vs[ps] = 0;
        if (s < c.len) {
          k[ps] = *reinterpret_cast<const uint32_t*>(b + B::k_word(t, ch));
          ks[ps] = b[B::k_scale(t, ch >> 2)];
          vs[ps] = b[B::kVScale + t];
        }
      }
      uint32_t w[B::kWords] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // tokens 4 qd + i of the dims 16 t + col
        const int s = s0 + 4 * qd + i, f = from(s), t = f % kPageTokens;
        const uint32_t* x = reinterpret_cast<const uint32_t*>(block4(pt[f / kPageTokens]) + B::kV) + ((t / 4) * 16 + col) * B::kWords;
        if (s < c.len)
#pragma unroll
          for (int j = 0; j < B::kWords; ++j) w[j] |= ((x[j] >> (4 * (t % 4))) & 0x000F000Fu) << (4 * i);
      }
      __builtin_amdgcn_sched_barrier(0);   // all of the page's loads before its stores
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows;
        if (!writes(s0 + t)) continue;
        *reinterpret_cast<uint32_t*>(dst + B::k_word(t, ch)) = k[ps];
        if ((ch & 3) == 0) dst[B::k_scale(t, ch >> 2)] = static_cast<uint8_t>(ks[ps]);
        if (ch == 0) dst[B::kVScale + t] = static_cast<uint8_t>(vs[ps]);
      }
      uint32_t* v = reinterpret_cast<uint32_t*>(dst + B::kV) + lane * B::kWords;
      if constexpr (D == 128) st16(v, make_uint4(w[0], w[1], w[2], w[3]));
      else st8(v, make_uint2(w[0], w[1]));
    } else {
      uint16_t* dst = block16(page);
      uint4 k[kPasses];
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int s = s0 + t_lane + ps * kRows, f = from(s);
        k[ps] = make_uint4(0, 0, 0, 0);
        if (s >= c.first && s < c.len) k[ps] = ld16(block16(pt[f / kPageTokens]) + k_elem(f % kPageTokens, ch));
      }
      uint32_t v[D / 64][kPageTokens];
#pragma unroll
      for (int t = 0; t < kPageTokens; ++t) {
        const int s = s0 + t, f = from(s);
        const uint16_t* b = block16(pt[f / kPageTokens]) + kPageTokens * D + f % kPageTokens;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) v[j][t] = s < c.len ? b[(lane + 64 * j) * kPageTokens] : 0u;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ps = 0; ps < kPasses; ++ps) {
        const int t = t_lane + ps * kRows;
        if (writes(s0 + t)) st16(dst + k_elem(t, ch), k[ps]);
      }
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint16_t* row = dst + kPageTokens * D + (lane + 64 * j) * kPageTokens;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = v[j][2 * i] | v[j][2 * i + 1] << 16;
        st16(row, make_uint4(w[0], w[1], w[2], w[3]));
        st16(row + 8, make_uint4(w[4], w[5], w[6], w[7]));
      }
    }
  }
}

hipError_t launch_keep(const PoolGeom& g, const Meta& meta, size_t src_off, int n_convs, hipStream_t stream) {
  if (n_convs == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n_convs * sizeof(KeepConv) || meta.bytes < src_off) return hipErrorInvalidValue;
  KeepArgs a;
  a.pool = g.pool;
  a.n_pages = g.n_pages;
  a.n_kv_heads = g.n_kv_heads;
  a.page_table = g.page_table;
  a.max_pages = g.max_pages;
  a.meta = meta.dev;
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
