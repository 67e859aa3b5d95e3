// Turn-1 prefill and turn-N extend-prefill attention over paged KV (flash-attention forward).
//
// A workgroup owns one (conversation, query block, kv head) tile; its waves cover the G query
// heads of that kv head (the GQA group), so every K/V tile in LDS serves all the query rows of
// the group (256 rows at head_dim 128).
// Each wave computes the transposed score tile on the matrix cores (v_mfma_f32_32x32x16_bf16):
//   S^T[key][query] = K[key][:] . Q[query][:]       A = K rows from LDS, B = Q kept in registers
//   O^T[dim][query] += V^T[dim][key] . P^T[key][query]   A = V^T rows from LDS, B = P registers
// With the transposed formulation every lane owns one query row (32 rows of a 32x32 tile, the two
// 32-lane halves holding different keys), so the online-softmax max/sum are in-lane except for
// one exchange between the halves, and the P accumulator registers are directly the B operand of
// the PV product: the key order of K or V^T in LDS is arranged so the two contractions agree.
//
// Eight waves, G query heads x 8/G blocks of 32 queries (a 64-query tile at G = 4, 128 queries at
// G = 2), two waves per SIMD.
// K/V tiles of 64 keys (4 pages) are copied from HBM straight into a four-deep LDS ring with
// global_load_lds_dwordx4 (no staging registers, no LDS store instructions), three tiles ahead;
// the K operands of tile j+1 are read into registers while the PV product of tile j runs.
// Diagonal tiles apply the causal mask and fully visible tiles skip it.
//
// A workgroup sweeps its tile's keys one after another, so a launch with fewer tiles than the chip
// has CUs takes as long as its longest tile. The host then cuts the tiles' keys into pieces
// (split_extend in host_state.cpp): each piece is a workgroup that writes its unnormalised output, row
// maximum and row sum, and extend_merge_kernel combines the pieces of a tile in their order. Where other
// work fills the CUs (a mixed step's decode, many layers in one launch) one workgroup takes a tile's
// pieces one after the other instead and combines them itself, with the same result bit for bit.
// A 301-token chunk on 41k tokens (40 workgroups, 646 key tiles each) 802 -> 200 us, a 1437-token prompt
// 39.4 -> 25.7 us.
//
// Bound: large launches by the matrix cores at the part's power limit (1.24-1.29 PFLOP/s at head dim
// 128; a library product of 8192^3 reaches 1.37). Small ones by a workgroup's start-up, 9 us at head dim
// 128 of which 0.5 is the plan, 1.5 pages, queries and first copies, 1.0 their arrival, 2.5 the first
// tile (mask, weights taken twice) and 2.0-3.7 were 8-byte output stores into 32 rows at a time.
// Over 4-bit pages (fp4.hpp) a launch is bound by the same, with 3/4 of the score product's matrix time and the conversion
// of V beside it: eight conversations' 128-2048 tokens on 8k-40k 1451-1550 us (1.18-1.26 PFLOP/s; in turn with bf16 pages
// 1472 against 1626), 301 tokens on 41k 175-182 (178 against 189). At head dim 64 the softmax leaves little difference (109
// us against 111): vector units busy 63% of the time, matrix cores 31%, hardly at a time.
// Head dim 64 against a kernel that staged tiles through registers, one wave per SIMD: six prompts of
// 300-9000 tokens 361 -> 229 us.
#include "attn_tile.hpp"

namespace cs {

// blockIdx.y: layer (consecutive layers of one launch share the plan)
template <int D, int G, bool PRE, bool CHAIN>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(PRE ? 2 : 4)))
void attn_fwd_kernel(LaunchMeta, ExtendArgs a) {
  attn_fwd_block<D, G, PRE, CHAIN>(a, blockIdx.x, blockIdx.y);
}

// the same over 4-bit pages
template <int D, int G, bool PRE, bool CHAIN>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(PRE ? 2 : 4)))
void attn_fp4_kernel(LaunchMeta, ExtendArgs a) {
  attn_fwd_block<D, G, PRE, CHAIN, true>(a, blockIdx.x, blockIdx.y);
}

template <int D, int G>
__global__ __launch_bounds__(256) void extend_merge_kernel(LaunchMeta, ExtendArgs a) {
  extend_merge_body<D, G>(a, blockIdx.x, blockIdx.y, threadIdx.x);
}

// One layer of a mixed step in one launch: extend tiles (or pieces) and work items of the decode split
// (8 waves, as in the split kernel), one workgroup each. Every workgroup gets the attention kernel's LDS
// ring and register budget, one workgroup (two waves per SIMD) a CU; at head dim 128 the decode split has no
// more by itself. At 64 it has three workgroups a CU by itself: 16 conversations of 10k tokens and a 20-token
// chunk take 64 us a layer here, 61 with the decode in its own launch.
// Units of n_kv_heads workgroups are taken in an order that spreads the extend units evenly over the
// first n_mix units, so that at any time some CUs use the matrix cores while others read HBM; n_mix =
// their number puts them all in front (tiles longer than everything else).
template <int D, int G, bool CHAIN, bool FP4>
__device__ __forceinline__ void mixed_layer_block(const ExtendArgs& ea, int n_ext, int n_mix, const DecodeArgs& da, float* xch) {
  static_assert(kDecodeItemThreads == 512, "a decode work item fills one attention workgroup");
  const int unit = blockIdx.x / ea.n_kv_heads, head = blockIdx.x % ea.n_kv_heads;
  const int before = unit < n_mix ? static_cast<int>(static_cast<int64_t>(unit) * n_ext / n_mix) : n_ext;
  const int after = unit < n_mix ? static_cast<int>(static_cast<int64_t>(unit + 1) * n_ext / n_mix) : n_ext;
  if (after > before) {
    attn_fwd_block<D, G, true, CHAIN, FP4>(ea, before * ea.n_kv_heads + head, 0);
    return;
  }
  split_body<D, FP4>(da, (unit - before) * ea.n_kv_heads + head, 0, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), xch);
}

template <int D, int G, bool CHAIN>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2)))
void mixed_layer_kernel(ExtendArgs ea, int n_ext, int n_mix, DecodeArgs da) {
  __shared__ float xch[split_exchange_floats<D>()];
  mixed_layer_block<D, G, CHAIN, false>(ea, n_ext, n_mix, da, xch);
}

// the same over 4-bit pages
template <int D, int G, bool CHAIN>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2)))
void mixed_fp4_kernel(ExtendArgs ea, int n_ext, int n_mix, DecodeArgs da) {
  __shared__ float xch[split_exchange_floats<D>()];
  mixed_layer_block<D, G, CHAIN, true>(ea, n_ext, n_mix, da, xch);
}

// What is left of that layer: the first n_ext workgroups merge its cut extend tiles, the others its
// decode records (n_dec of them, 256 threads each).
template <int D, int G>
__global__ __launch_bounds__(256) void mixed_merge_kernel(ExtendArgs ea, int n_ext, DecodeArgs da) {
  __shared__ MergeLds<D> lds;
  const int blk = blockIdx.x;
  if (blk < n_ext) {
    extend_merge_body<D, G>(ea, blk, 0, threadIdx.x);
    return;
  }
  merge_body<D>(da, blk - n_ext, 0, threadIdx.x, lds);
}

int extend_query_tile(int group) { return kExtendTileRows / group; }

hipError_t launch_extend(const PoolGeom& g, int layer, int n_layers, const ExtendLaunch& e, const void* q, void* out,
                         float* parts, hipStream_t stream) {
  if (e.n_tiles == 0 || n_layers == 0) return hipSuccess;
  if (!e.meta.ok() || (e.n_parts > 0 && (parts == nullptr || e.piece < 1))) return hipErrorInvalidValue;
  const ExtendArgs a = make_extend_args(g, layer, e, q, out, parts);
  LaunchMeta m;
  fill_meta(e.meta, &m);
  const int64_t blocks = static_cast<int64_t>(e.n_tiles) * g.n_kv_heads;
  if (!grid_holds(blocks, 512)) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks), n_layers);
  // At head_dim 64 a launch of more than 2.5 workgroups per CU runs two at a time on each: one prompt of
  // 9000 tokens (1128 workgroups) 352 -> 339 us, 6000 (752) 168 -> 163; below, one at a time that reads
  // its operands ahead is the faster form: 4500 (568) 98 against 106 us, 2500 (320) 41 against 45. A
  // head_dim 128 workgroup fills its CU's LDS.
  const bool two_per_cu = static_cast<int64_t>(grid.x) * grid.y > 5 * kCus / 2;
  auto launch = [&](auto kernel) {
    kernel<<<grid, 512, 0, stream>>>(m, a);
    return hipGetLastError();
  };
  return by_shape(g, [&](auto d, auto grp) {
    if (g.fp4) {
      if constexpr (d() == 64) {
        if (two_per_cu)
          return e.chained ? launch(attn_fp4_kernel<d(), grp(), false, true>) : launch(attn_fp4_kernel<d(), grp(), false, false>);
      }
      return e.chained ? launch(attn_fp4_kernel<d(), grp(), true, true>) : launch(attn_fp4_kernel<d(), grp(), true, false>);
    }
    if constexpr (d() == 64) {
      if (two_per_cu)
        return e.chained ? launch(attn_fwd_kernel<d(), grp(), false, true>) : launch(attn_fwd_kernel<d(), grp(), false, false>);
    }
    return e.chained ? launch(attn_fwd_kernel<d(), grp(), true, true>) : launch(attn_fwd_kernel<d(), grp(), true, false>);
  });
}

hipError_t launch_extend_merge(const PoolGeom& g, int n_layers, const ExtendLaunch& e, void* out, float* parts,
                               hipStream_t stream) {
  if (e.n_merges == 0 || n_layers == 0) return hipSuccess;
  if (!e.meta.ok() || parts == nullptr) return hipErrorInvalidValue;
  const ExtendArgs a = make_extend_args(g, 0, e, nullptr, out, parts);
  LaunchMeta m;
  fill_meta(e.meta, &m);
  return by_shape(g, [&](auto d, auto grp) {
    extend_merge_kernel<d(), grp()><<<dim3(e.n_merges * g.n_kv_heads * 8, n_layers), 256, 0, stream>>>(m, a);
    return hipGetLastError();
  });
}

hipError_t launch_mixed_layer(const PoolGeom& g, int layer, const ExtendLaunch& e, const void* q_ext,
                              void* out_ext, float* parts, const DecodeLaunch& w, const void* q_dec,
                              float* partials, void* direct_out, hipStream_t stream) {
  if (e.n_tiles == 0 || w.n_convs == 0) return hipErrorInvalidValue;
  if (e.meta.dev == nullptr || w.meta.dev == nullptr || w.n_items < w.n_convs) return hipErrorInvalidValue;
  if (direct_out != nullptr && w.n_items != w.n_convs) return hipErrorInvalidValue;
  if (e.n_parts > 0 && (parts == nullptr || e.piece < 1)) return hipErrorInvalidValue;
  const ExtendArgs ea = make_extend_args(g, layer, e, q_ext, out_ext, parts);
  DecodeArgs da = make_decode_args(g, layer, w, q_dec, direct_out, partials);
  da.direct = direct_out != nullptr;
  // Pieces of cut tiles (all short) are spread over the first 60% of the decode items; whole and chained
  // tiles go in front of them. Layers of 16 conversations (2k-12k tokens, a 513-token chunk): 4.20-4.33 ms per 32-layer
  // step with the pieces in front, 4.06 spread over 40%, 4.05 over 70%, 4.72 over all; 16 x 4k tokens and
  // a 300-token chunk 3.19, 2.88, 2.70, 2.92.
  // (Over 4-bit pages all in front: an item there takes its CU's time rather than HBM's, so extend units among them only
  // end later. 64 conversations of 1k-9k beside chunks of 700 on 8k and 64 on 3k, 32 layers: 10.3 -> 5.9 ms, seven other
  // steps 1-9% faster or the same within 2%.)
  const int n_mix = e.n_tiles + (e.n_merges > 0 && !g.fp4 ? w.n_items * 6 / 10 : 0);
  const int64_t n_blocks = (static_cast<int64_t>(e.n_tiles) + w.n_items) * g.n_kv_heads;
  if (!grid_holds(n_blocks, 512)) return hipErrorInvalidConfiguration;
  const int blocks = static_cast<int>(n_blocks);
  return by_shape(g, [&](auto d, auto grp) {
    if (g.fp4 && e.chained) mixed_fp4_kernel<d(), grp(), true><<<blocks, 512, 0, stream>>>(ea, e.n_tiles, n_mix, da);
    else if (g.fp4) mixed_fp4_kernel<d(), grp(), false><<<blocks, 512, 0, stream>>>(ea, e.n_tiles, n_mix, da);
    else if (e.chained) mixed_layer_kernel<d(), grp(), true><<<blocks, 512, 0, stream>>>(ea, e.n_tiles, n_mix, da);
    else mixed_layer_kernel<d(), grp(), false><<<blocks, 512, 0, stream>>>(ea, e.n_tiles, n_mix, da);
    return hipGetLastError();
  });
}

hipError_t launch_mixed_merge(const PoolGeom& g, const ExtendLaunch& e, void* out_ext, float* parts,
                              const DecodeLaunch& w, const float* partials, void* out_dec, hipStream_t stream) {
  // out_dec == nullptr: the split wrote the decode outputs
  const int n_ext = e.n_merges * g.n_kv_heads * 8;
  const int64_t n_blocks = n_ext + (out_dec != nullptr ? static_cast<int64_t>(w.n_convs) * g.n_q_heads : 0);
  if (n_blocks == 0) return hipSuccess;
  if (!grid_holds(n_blocks, 256)) return hipErrorInvalidConfiguration;
  const int blocks = static_cast<int>(n_blocks);
  if (e.meta.dev == nullptr || w.meta.dev == nullptr || (n_ext > 0 && parts == nullptr)) return hipErrorInvalidValue;
  const ExtendArgs ea = make_extend_args(g, 0, e, nullptr, out_ext, parts);
  const DecodeArgs da = make_decode_args(g, 0, w, nullptr, out_dec, partials);
  return by_shape(g, [&](auto d, auto grp) {
    mixed_merge_kernel<d(), grp()><<<blocks, 256, 0, stream>>>(ea, n_ext, da);
    return hipGetLastError();
  });
}

}  // namespace cs
