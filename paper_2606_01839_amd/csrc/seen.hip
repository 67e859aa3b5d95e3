// Attention whose rows are not a conversation's last tokens in causal order: a tree of drafted tokens over the
// cache that holds them (a token sees the cached ones, its ancestors and itself), and rows that see every token
// (an encoder's states). o = softmax(q K^T / sqrt(d)) V over the keys a row sees (host/seen.hpp).
//
// One workgroup per (row, query head); its waves take the pages in turn, fp32 throughout, and join at the end.
#include <cfloat>
#include <cmath>

#include "device_common.hpp"
#include "fp4.hpp"
#include "kernels.hpp"

namespace cs {

struct SeenArgs {
  const void* pool;
  int64_t n_pages;
  int n_kv_heads, group, layer;
  const int32_t* page_table;
  int max_pages;
  const void* meta;
  uint32_t masks_off, words_off;
  int n_convs;
  const uint16_t* q;
  uint16_t* out;
  float scale_log2;
};

template <int D, bool FP4>
__global__ __launch_bounds__(256) void seen_row_kernel(LaunchMeta, SeenArgs a) {
  constexpr int DL = D / 4;                  // dims of a score's part
  __shared__ float xo[4][D], xm[4], xl[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n_q_heads = a.n_kv_heads * a.group;
  const int row = blockIdx.x / n_q_heads, h = blockIdx.x % n_q_heads, g = h / a.group;
  const auto* convs = meta_at<ExtendConvDesc>(a.meta, 0);
  int lo = 0, hi = a.n_convs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (convs[mid].q_row <= row) lo = mid; else hi = mid - 1;
  }
  const int len = convs[lo].len, slot = convs[lo].slot, i = row - convs[lo].q_row;
  const auto* mk = meta_at<SeenMask>(a.meta, a.masks_off) + lo;
  const int clear = mk->clear, words = mk->words, w0 = clear / 32;
  const auto* my = meta_at<uint32_t>(a.meta, a.words_off) + mk->off + static_cast<size_t>(i) * words;
  const int32_t* pt = a.page_table + static_cast<size_t>(slot) * a.max_pages;
  const int key = lane & 15, part = lane >> 4;
  float qf[DL];
  const uint16_t* qrow = a.q + (static_cast<size_t>(row) * n_q_heads + h) * D;
  for (int e = 0; e < DL; ++e) qf[e] = __uint_as_float(static_cast<uint32_t>(qrow[DL * part + e]) << 16);
  float m = -FLT_MAX, l = 0.f, o[D / 64] = {};
  for (int p = wave; p * kPageTokens < len; p += 4) {
    const size_t block = (static_cast<size_t>(a.layer) * a.n_pages + pt[p]) * a.n_kv_heads + g;
    const uint16_t* b16 = static_cast<const uint16_t*>(a.pool) + block * (2 * kPageTokens * D);
    const uint8_t* b4 = static_cast<const uint8_t*>(a.pool) + block * Fp4Block<D>::kBytes;
    const int k = p * kPageTokens + key;
    auto code = [](uint32_t c) {
      const float t[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
      return c & 8 ? -t[c & 7] : t[c & 7];
    };
    auto scale = [](uint32_t b) { return b == 255 ? __builtin_nanf("") : fp4_scale(b); };
    float s = 0.f;
    for (int e = 0; e < DL; ++e) {
      const int d = DL * part + e;
      float x;
      if constexpr (FP4) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(b4 + Fp4Block<D>::k_word(key, d / 8));
        x = code(w >> (4 * (d % 8)) & 15) * scale(b4[Fp4Block<D>::k_scale(key, d / 32)]);
      } else {
        x = __uint_as_float(static_cast<uint32_t>(b16[k_elem(key, d / 8) + d % 8]) << 16);
      }
      s = __builtin_fmaf(qf[e], x, s);
    }
    s += xor_shfl(s, 16);
    s += xor_shfl(s, 32);
    const bool sees = k < clear || (k < len && (my[k / 32 - w0] >> (k % 32) & 1));
    if (!sees) s = -INFINITY;
    float mx = s;
    for (int off = 1; off < 16; off <<= 1) mx = fmaxf(mx, xor_shfl(mx, off));
    const float m_new = fmaxf(m, mx), alpha = fast_exp2((m - m_new) * a.scale_log2);
    const float w = fast_exp2((s - m_new) * a.scale_log2);
    m = m_new;
    l *= alpha;
    for (int t = 0; t < D / 64; ++t) o[t] *= alpha;
    for (int t = 0; t < kPageTokens; ++t) {
      const float wt = __shfl(w, t);
      if (!__shfl(sees, t)) continue;
      l += wt;
      for (int j = 0; j < D / 64; ++j) {
        const int d = lane + 64 * j;
        float x;
        if constexpr (FP4) {
          const uint32_t v = *reinterpret_cast<const uint32_t*>(b4 + Fp4Block<D>::kV + (((t / 4) * 16 + d % 16) * Fp4Block<D>::kWords + d / 32) * 4);
          x = code(v >> (16 * (d / 16 % 2) + 4 * (t % 4)) & 15) * scale(b4[Fp4Block<D>::kVScale + t]);
        } else {
          x = __uint_as_float(static_cast<uint32_t>(b16[kPageTokens * D + d * kPageTokens + t]) << 16);
        }
        o[j] = __builtin_fmaf(wt, x, o[j]);
      }
    }
  }
  for (int j = 0; j < D / 64; ++j) xo[wave][lane + 64 * j] = o[j];
  if (lane == 0) xm[wave] = m, xl[wave] = l;
  __syncthreads();
  if (threadIdx.x < D) {
    const float M = fmaxf(fmaxf(xm[0], xm[1]), fmaxf(xm[2], xm[3]));
    float num = 0.f, den = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float wt = fast_exp2((xm[w] - M) * a.scale_log2);
      num = __builtin_fmaf(wt, xo[w][threadIdx.x], num);
      den = __builtin_fmaf(wt, xl[w], den);
    }
    // no key at all: zeros
    a.out[(static_cast<size_t>(row) * n_q_heads + h) * D + threadIdx.x] =
        static_cast<uint16_t>(pack_bf16x2(len > 0 ? num / den : 0.f, 0.f) & 0xFFFFu);
  }
}

hipError_t launch_seen_rows(const PoolGeom& g, int layer, const SeenLaunch& w, const void* q, void* out, hipStream_t stream) {
  if (!w.meta.ok()) return hipErrorInvalidValue;
  SeenArgs a;
  a.pool = g.pool;
  a.n_pages = g.n_pages;
  a.n_kv_heads = g.n_kv_heads;
  a.group = g.n_q_heads / g.n_kv_heads;
  a.layer = layer;
  a.page_table = g.page_table;
  a.max_pages = g.max_pages;
  a.meta = w.meta.dev;
  a.masks_off = static_cast<uint32_t>(w.masks_off);
  a.words_off = static_cast<uint32_t>(w.words_off);
  a.n_convs = w.n_convs;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(g.head_dim)));
  const int64_t blocks = w.rows * g.n_q_heads;
  if (!grid_holds(blocks, 256)) return hipErrorInvalidConfiguration;
  LaunchMeta m;
  fill_meta(w.meta, &m);
  const unsigned n = static_cast<unsigned>(blocks);
  if (g.head_dim == 128 && g.fp4) seen_row_kernel<128, true><<<n, 256, 0, stream>>>(m, a);
  else if (g.head_dim == 64 && g.fp4) seen_row_kernel<64, true><<<n, 256, 0, stream>>>(m, a);
  else if (g.head_dim == 128) seen_row_kernel<128, false><<<n, 256, 0, stream>>>(m, a);
  else if (g.head_dim == 64) seen_row_kernel<64, false><<<n, 256, 0, stream>>>(m, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace cs
