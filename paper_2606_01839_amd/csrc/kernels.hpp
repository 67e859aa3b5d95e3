// Host-callable launchers of the gfx950 kernels (defined in the .hip files).
#pragma once

#include <hip/hip_runtime.h>

#include <cstring>

#include "host/host_state.hpp"
#include "host/seen.hpp"

namespace cs {

struct PoolGeom {
  void* pool;          // device base of the KV pool
  int64_t n_pages;
  int n_layers;
  int n_kv_heads;
  int n_q_heads;
  int head_dim;
  int32_t* page_table;  // device mirror [max_convs][max_pages]
  int max_pages;
  bool fp4;             // blocks of 4-bit codes and scales (fp4.hpp) instead of bf16
};

// Whether a grid holds that many workgroups in x: fewer than 2^32 threads (a launch of more runs some of them and reports
// no error). Launches whose count grows with a batch return hipErrorInvalidConfiguration where it does not.
inline bool grid_holds(int64_t workgroups, int threads) { return workgroups * threads < (int64_t(1) << 32); }

// Metadata of one launch (descriptors, work lists, page ids): `bytes` bytes laid out on the host at
// `host`, or already on the device at `dev` (a stream-ordered upload; `host` is then unused). A plan
// of at most kMetaBytes travels in the launch's own kernel arguments (dev = nullptr): an upload is a
// copy kernel of 2-5 us that the launch waits for (~8 us apart when nothing else is queued). Decode of
// 16 conversations of 1k-9k tokens 29.4 -> 25.6 us, one of 24k 25.6 -> 23.3, prefill of 1.4k tokens
// 39.4 -> 37.3; the larger argument block costs a launch of 690 us nothing measurable. Larger plans
// are uploaded: they belong to launches of many tiles. 3 KiB keeps every kernel's arguments inside
// the 4 KiB a launch may pass.
constexpr size_t kMetaBytes = 3072;
struct LaunchMeta {
  alignas(16) uint32_t w[kMetaBytes / 4];
};
struct Meta {
  const void* host = nullptr;
  const void* dev = nullptr;
  size_t bytes = 0;
  // false: neither uploaded nor small enough to travel with the launch
  bool ok() const { return dev != nullptr || (host != nullptr && bytes <= kMetaBytes); }
};

// The argument block of a launch whose plan is not on the device: the plan's bytes. (The rest of the
// block is not read.)
inline void fill_meta(const Meta& m, LaunchMeta* out) {
  if (m.dev == nullptr) std::memcpy(out->w, m.host, m.bytes);
}

// Metadata to device memory (16-byte aligned, room up to a multiple of 16) in the arguments of launches,
// kMetaBytes each: what a captured graph keeps, unlike a copy's source.
hipError_t launch_store_meta(const void* host, size_t bytes, void* dst, hipStream_t stream);

// KV append: write chunks (meta: PageChunk[n_chunks]) of k,v [n_layers][src_rows][Hkv][D]. With
// carry_bytes > 0 the metadata travels in the kernel arguments and its bytes [carry_off, carry_off +
// carry_bytes) (multiples of 16) are also stored to carry_dst, for the launches that follow.
struct AppendCarry {
  void* dst = nullptr;
  size_t off = 0, bytes = 0;
};
hipError_t launch_append(const PoolGeom& g, const Meta& meta, int n_chunks, const AppendCarry& carry,
                         const void* k, const void* v, int64_t src_rows, hipStream_t stream);

// Rotation of the first 2 pairs dims of a head (rope.hpp): per pair the 64-bit fraction of a turn a
// position makes.
struct RopeArgs {
  uint64_t frac[64];
  float amplitude;
  int pairs;        // a multiple of 8, at most head_dim / 2
  int interleaved;  // pair i = dims 2 i, 2 i + 1; else dims i, i + pairs
};

// The append of 4-bit pools, and of both kinds with rotated keys (rope != nullptr). With q != nullptr the
// launch also writes the rotated q [n_layers][src_rows][Hq][D] to q_out (may be q itself). pos_off > 0: the positions that
// tokens turn by are int32[n_chunks][16] there in meta, by token slot of the chunk's page; else they are the slots.
hipError_t launch_append_as(const PoolGeom& g, const Meta& meta, int n_chunks, const AppendCarry& carry, const RopeArgs* rope,
                            const void* k, const void* v, const void* q, void* q_out, int64_t src_rows, size_t pos_off,
                            hipStream_t stream);

// Rotation of query rows q [n_layers][rows][Hq][D] into out (may be q): meta = RopeConv[n_convs], or with n_convs = 0
// every row's position, int32[rows].
struct RopeConv {
  int32_t row;   // first row of the conversation
  int32_t pos;   // its position
};
hipError_t launch_rope_q(const PoolGeom& g, const Meta& meta, int n_convs, int64_t rows, int n_layers, const RopeArgs& rope,
                         const void* q, void* out, hipStream_t stream);

// Keep of drafted tokens: meta = KeepConv[n_convs], at pages_off int32 physical pages, at src_off int64 sources (16 x physical page
// + token slot).
struct KeepConv {
  int32_t page0, n;    // the pages that are rewritten: entries page0 .. page0 + n - 1, in order
  int32_t first, len;  // token slots, counted from the first of those pages': [first, len) receive tokens, those behind them zeros
  int32_t from, src;   // source of slot from + i (from: first rounded down to 8; a slot before `first` is its own): entry src + i
};
hipError_t launch_keep(const PoolGeom& g, const Meta& meta, size_t pages_off, size_t src_off, int n_convs, hipStream_t stream);

// Workgroups that the queries of an append of n_chunks add to its launch.
int64_t append_rope_groups(const PoolGeom& g, size_t n_chunks);
// Layers one launch_rope_q may take (a grid dimension).
int rope_q_layers(const PoolGeom& g);

// Read back: chunks (meta: PageChunk[n_chunks]) of the pool to k, v [n_layers][dst_rows][Hkv][D] in bf16.
hipError_t launch_read(const PoolGeom& g, const Meta& meta, int n_chunks, void* k, void* v, int64_t dst_rows, hipStream_t stream);

// Pack of logical pages [lp0, lp0 + n_lp) of a conversation (of a pool of either kind) into the wire of a 4-bit
// pool, and that pool's unpack. A launch takes at most kMaxPackPages (256 threads a page).
constexpr int kMaxPackPages = (1 << 24) - 1;
hipError_t launch_pack_fp4(const PoolGeom& g, int slot, int64_t len, int lp0, int n_lp, void* wire, hipStream_t stream);
hipError_t launch_unpack_fp4(const PoolGeom& g, const void* wire, const Meta& meta, int slot, int64_t len, int lp0, int n_lp,
                             hipStream_t stream);

// Pack: conversation pages (page-table row `slot`) -> wire [layer][lpage][head] blocks.
hipError_t launch_pack(const PoolGeom& g, int slot, int64_t len, void* wire, hipStream_t stream);

// Unpack: wire logical pages [lp0, lp0 + n_lp) -> physical pages (meta: int32[n_lp]) of the
// conversation in page-table row `slot` (length len).
hipError_t launch_unpack(const PoolGeom& g, const void* wire, const Meta& meta, int slot,
                         int64_t len, int lp0, int n_lp, hipStream_t stream);

// Decode partial record of one (work item, query head): o[d], running max m, sum l, two unused
// floats, so records stay 16-byte aligned.
constexpr int partial_floats(int head_dim) { return head_dim + 4; }

// A decode plan as the kernels read it: meta = DecodeConvDesc[n_convs], then (16-byte aligned, at
// order_off) the launch order of its n_items items (a permutation).
struct DecodeLaunch {
  Meta meta;
  size_t order_off = 0;
  int n_convs = 0, n_items = 0, split = 0;
};

// Decode of n_layers consecutive layers from `layer` on in one launch: split kernel over plan items
// (partials: n_layers x n_items x n_q_heads records), then the merge kernel (output). q and out:
// [n_layers][n_convs][n_q_heads][head_dim].
// direct_out != nullptr (only when every conversation is one item, n_items == n_convs): the split
// writes the final output there and no merge follows.
hipError_t launch_decode_split(const PoolGeom& g, int layer, int n_layers, const DecodeLaunch& w, const void* q,
                               float* partials, void* direct_out, hipStream_t stream);
hipError_t launch_decode_merge(const PoolGeom& g, int n_layers, const DecodeLaunch& w, const float* partials,
                               void* out, hipStream_t stream);

// Streaming-read probe: read `bytes` (a multiple of 16) of device memory once with non-temporal
// 16-byte loads on 8 workgroups per CU; `sink` is 4 bytes of device memory (almost never written).
hipError_t launch_stream_read_probe(const void* src, size_t bytes, uint32_t* sink, int n_cus,
                                    hipStream_t stream);

// Capacity of the static decode scratch (floats): 16 MiB on each GPU.
constexpr size_t kStaticScratchFloats = size_t(4) << 20;
// Device address of the static decode scratch on the current device (looked up once per device
// with hipGetSymbolAddress and cached; allocates nothing).
hipError_t static_decode_scratch(float** out);

// Query rows (query tokens x query heads of the kv head) of an extend tile.
constexpr int kExtendTileRows = 256;
// Record of one piece of a cut extend tile and one kv head: o[256 rows][d] in accumulator order, then
// (maximum, sum) for each of the 8 x 64 lanes.
constexpr int extend_part_floats(int head_dim) { return kExtendTileRows * head_dim + 2 * 512; }

// An extend plan as the kernels read it: meta = ExtendConvDesc[..], then (16-byte aligned, at
// tiles_off) ExtendTile[n_tiles] and (at merges_off) ExtendMerge[n_merges].
struct ExtendLaunch {
  Meta meta;
  size_t tiles_off = 0, merges_off = 0;
  int n_tiles = 0, n_merges = 0;
  int piece = 0, n_parts = 0;
  bool chained = false;  // some tiles hold their pieces (ExtendTile::k0 < 0)
  int64_t q_rows = 0;  // query rows of a layer
  size_t masks_off = 0, words_off = 0;   // launch_seen_tiles: SeenMask[..] of the conversations, and their words
};

// One layer of a mixed step in one launch: the extend tiles of the layer and its decode split
// (partials); launch_mixed_merge then combines the pieces of cut extend tiles and (out_dec !=
// nullptr) the decode records in one launch. Both plans uploaded.
hipError_t launch_mixed_layer(const PoolGeom& g, int layer, const ExtendLaunch& e, const void* q_ext,
                              void* out_ext, float* parts, const DecodeLaunch& w, const void* q_dec,
                              float* partials, void* direct_out, hipStream_t stream);
hipError_t launch_mixed_merge(const PoolGeom& g, const ExtendLaunch& e, void* out_ext, float* parts,
                              const DecodeLaunch& w, const float* partials, void* out_dec, hipStream_t stream);

// Query tokens per extend/prefill work tile for this GQA group (the host plan must match).
int extend_query_tile(int group);

// Extend / prefill of n_layers consecutive layers from `layer` on: one workgroup per (tile or piece, kv
// head, layer); then, where tiles are cut (n_merges > 0), the merge of their pieces. q and out:
// [n_layers][q_rows][n_q_heads][head_dim]; parts: n_layers x n_parts x n_kv_heads records.
hipError_t launch_extend(const PoolGeom& g, int layer, int n_layers, const ExtendLaunch& e, const void* q, void* out,
                         float* parts, hipStream_t stream);
hipError_t launch_extend_merge(const PoolGeom& g, int n_layers, const ExtendLaunch& e, void* out, float* parts,
                               hipStream_t stream);

// Attention of rows that see what their words say (host/seen.hpp), at most kSeenRows rows (query tokens x query heads of a kv head) an entry: meta = ExtendConvDesc[..], and SeenMask[..],
// the words, SeenItem[n_items] in launch order and int32[n_merges] (entries of several items) at their offsets. Records of
// the items of entries with several: SeenMask::rec + item, [kv head][16 blocks rows] of partial_floats each.
constexpr int kSeenRows = 64;
struct SeenLaunch {
  Meta meta;
  size_t masks_off = 0, words_off = 0, items_off = 0, merges_off = 0;
  int n_items = 0, n_merges = 0;
  int merge_rows = 0, merge_items = 0;   // the most rows, and items, of an entry of several items
  int blocks = 1;       // blocks of 16 rows: 1 to 4
  int split = 0;        // keys per wave
};
hipError_t launch_seen_rows(const PoolGeom& g, int layer, const SeenLaunch& w, const void* q, void* out, float* parts,
                            hipStream_t stream);
hipError_t launch_seen_rows_merge(const PoolGeom& g, const SeenLaunch& w, void* out, float* parts, hipStream_t stream);

// The same for any number of rows, in tiles as launch_extend's; pieces are joined by
// launch_extend_merge.
hipError_t launch_seen_tiles(const PoolGeom& g, int layer, const ExtendLaunch& e, const void* q, void* out, float* parts,
                             hipStream_t stream);

// Rows of zeros: those of conversations without a key. meta: SeenEmpty[n].
struct SeenEmpty {
  int64_t row;   // first row
  int64_t n;
};
hipError_t launch_seen_empty(const PoolGeom& g, const Meta& meta, int n, void* out, hipStream_t stream);

}  // namespace cs
