// Attention of rows that are not a conversation's last tokens in causal order (host/seen.hpp), for many rows: the tiles of
// attn_tile.hpp with words in place of the causal mask. Bound by the matrix cores as those: 62% busy in texts of 100-3500 rows on
// 600-9000 states (264 GFLOP, 251 us), 65% in trees of 130-250 tokens on 8k-40k (483 GFLOP, 496 us, an eighth of the tiles'
// rows empty); by HBM where a tile's rows are few (64 trees of 32 tokens on 8k-32k 865 us, 5.3 TB/s).
#include "attn_tile.hpp"

namespace cs {

template <int D, int G, bool FP4>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void seen_tile_kernel(LaunchMeta, SeenTileArgs a) {
  attn_fwd_block<D, G, true, false, FP4, true>(a, blockIdx.x, 0);
}

hipError_t launch_seen_tiles(const PoolGeom& g, int layer, const ExtendLaunch& e, const void* q, void* out, float* parts,
                             hipStream_t stream) {
  if (e.n_tiles == 0) return hipSuccess;
  if (!e.meta.ok() || e.chained || (e.n_parts > 0 && (parts == nullptr || e.piece < 1))) return hipErrorInvalidValue;
  SeenTileArgs a;
  static_cast<ExtendArgs&>(a) = make_extend_args(g, layer, e, q, out, parts);
  a.masks_off = static_cast<uint32_t>(e.masks_off);
  a.words_off = static_cast<uint32_t>(e.words_off);
  LaunchMeta m;
  fill_meta(e.meta, &m);
  const int64_t blocks = static_cast<int64_t>(e.n_tiles) * g.n_kv_heads;
  if (!grid_holds(blocks, 512)) return hipErrorInvalidConfiguration;
  return by_shape(g, [&](auto d, auto grp) {
    if (g.fp4) seen_tile_kernel<d(), grp(), true><<<static_cast<unsigned>(blocks), 512, 0, stream>>>(m, a);
    else seen_tile_kernel<d(), grp(), false><<<static_cast<unsigned>(blocks), 512, 0, stream>>>(m, a);
    return hipGetLastError();
  });
}

// One workgroup an entry.
__global__ __launch_bounds__(256) void seen_empty_kernel(LaunchMeta, const void* meta, uint16_t* out, int64_t row_elems) {
  const auto* e = meta_at<SeenEmpty>(meta, 0) + blockIdx.x;
  uint16_t* dst = out + e->row * row_elems;
  for (int64_t i = 8 * threadIdx.x; i < e->n * row_elems; i += 8 * blockDim.x) st16(dst + i, make_uint4(0, 0, 0, 0));
}

hipError_t launch_seen_empty(const PoolGeom& g, const Meta& meta, int n, void* out, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  if (!meta.ok() || meta.bytes < n * sizeof(SeenEmpty)) return hipErrorInvalidValue;
  LaunchMeta m;
  fill_meta(meta, &m);
  seen_empty_kernel<<<n, 256, 0, stream>>>(m, meta.dev, static_cast<uint16_t*>(out), static_cast<int64_t>(g.n_q_heads) * g.head_dim);
  return hipGetLastError();
}

}  // namespace cs
