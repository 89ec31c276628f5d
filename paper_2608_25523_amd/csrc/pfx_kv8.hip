// The 8-bit KV pool on the device: quantising appends, whole pages between the
// bf16 and the 8-bit format, and attention over e4m3 keys and values.
//
// A block (one page of one KV head, K or V) holds 16 D e4m3 bytes in the order
// in which the attention kernels' lanes take them, so that a wave's 16-byte
// loads of a block are consecutive and need no transposition:
//   K: [D / 16][16 tokens][16 dims]: lane (token, g) reads dims 16 g .. of its
//     token with one load (and 64 + 16 g .. with a second, D = 128);
//   V: [D / 64][4 token groups][16 r][4 i][4 tokens]: lane (r, g) reads, with
//     one load per 64 dims, dims 64 f + 16 i + r of tokens 4 g .. 4 g + 3: the
//     A operand's rows of four 16-dim blocks in the key order of the scores.
// The products run on the bf16 matrix unit.  e4m3 fits into bf16, and
// v_cvt_scalef32_pk_bf16_fp8 applies the block's power of two as it converts,
// two values an instruction (1.8 ns a wave's instruction, as an fma), so the
// dequantised values are exact and no product or sum carries a scale.
#include <type_traits>
#include <vector>

#include "pfx_device.h"

namespace pfx {

typedef float f32x2v __attribute__((ext_vector_type(2)));

// 2^(e - 127) of a scale byte.
__device__ __forceinline__ float scale_of(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Two e4m3 bytes of w (low or high half) as packed bf16, times a power of two.
template <bool HI>
__device__ __forceinline__ uint32_t bf16_of(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

// ---------------------------------------------------------------------------
// Blocks in the quantised format
//
// Quantising and reading back work on a block per wave: lane (t, g) holds
// token t's dims 16 (g + 4 f) .. + 15 for the D / 64 halves f.  For K that is
// the block's order.  For V the four lanes of a quad hold four tokens of the
// same dims, and a 4 x 4 byte transpose inside the quad gives each lane the
// words [4 tokens] of dims 4 j + q (q: its place in the quad).
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t quad_lane(uint32_t x, int k) {
  switch (k) {
    case 0: return __builtin_amdgcn_mov_dpp(int(x), 0x00, 0xF, 0xF, true);
    case 1: return __builtin_amdgcn_mov_dpp(int(x), 0x55, 0xF, 0xF, true);
    case 2: return __builtin_amdgcn_mov_dpp(int(x), 0xAA, 0xF, 0xF, true);
    default: return __builtin_amdgcn_mov_dpp(int(x), 0xFF, 0xF, 0xF, true);
  }
}

// Byte q of each of the quad's four words, q the lane's place in the quad.  Its
// own inverse over the quad.
__device__ __forceinline__ uint32_t quad_transpose(uint32_t w, int q) {
  const uint32_t sel = uint32_t(q) | uint32_t(4 + q) << 8;
  const uint32_t lo = __builtin_amdgcn_perm(quad_lane(w, 1), quad_lane(w, 0), sel);
  const uint32_t hi = __builtin_amdgcn_perm(quad_lane(w, 3), quad_lane(w, 2), sel);
  return (lo & 0xFFFFu) | hi << 16;
}

// Byte offset, in a V block, of the word [4 tokens] of dim 64 f + 16 g + 4 j + q
// of lane (t, g)'s token group.
__device__ __forceinline__ int v_word(int f, int j, int lane) {
  const int t = lane & 15, g = lane >> 4;
  return 1024 * f + 256 * (t >> 2) + 16 * (4 * j + (t & 3)) + 4 * g;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = max(x, uint32_t(__shfl_xor(int(x), m)));
  return x;
}

// Four fp32 values times a power of two as e4m3 (nearest, ties to even; past
// the largest number, and for a NaN, a NaN byte).
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// A bf16 (its bits in the upper half of x) as fp32; NaN for what the format does
// not hold: infinities, NaN, magnitudes of 2^127 and more.
__device__ __forceinline__ float storable(uint32_t x) {
  return __builtin_bit_cast(float, (x & 0x7FFFFFFFu) >= 0x7F000000u ? 0x7FC00000u : x);
}

// The bits that count for a block's maximum, of two packed bf16.
__device__ __forceinline__ uint32_t magnitude(uint32_t w) {
  const uint32_t lo = w & 0x7FFFu, hi = w >> 16 & 0x7FFFu;
  return max(lo < 0x7F00u ? lo : 0u, hi < 0x7F00u ? hi : 0u);
}

// e4m3 bytes of w at another exponent: their values times f.
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float f) {
  const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  return e4m3x4(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}

// One wave writes one block: slots [slot0, slot0 + count) from `count` bf16 rows
// at `rows`, `stride` elements apart; the slots before them keep their values,
// those behind them become zero.  A block is written whole (2 KiB, D = 128):
// its scale covers every token of it.
template <int D>
__device__ __forceinline__ void quantize_block(const uint16_t* rows, size_t stride, int slot0, int count,
                                               unsigned char* block, uint8_t* scale, bool is_v, int lane) {
  constexpr int F = D / 64;
  const int t = lane & 15, g = lane >> 4;
  const bool fresh = t >= slot0 && t < slot0 + count;
  u32x4 x[F][2], old[F];
  uint32_t old_e = 0;
#pragma unroll
  for (int f = 0; f < F; ++f) {
    x[f][0] = x[f][1] = old[f] = u32x4{0u, 0u, 0u, 0u};
    if (fresh) {
      const uint16_t* src = rows + size_t(t - slot0) * stride + 16 * (g + 4 * f);
      x[f][0] = *reinterpret_cast<const u32x4*>(src);
      x[f][1] = *reinterpret_cast<const u32x4*>(src + 8);
    }
  }
  if (slot0 > 0) {
    old_e = *scale;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      if (is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) old[f][j] = *reinterpret_cast<const uint32_t*>(block + v_word(f, j, lane));
      } else {
        old[f] = *reinterpret_cast<const u32x4*>(block + 1024 * f + 16 * lane);
      }
    }
  }
  uint32_t most = 0;
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) most = max(most, magnitude(x[f][h][j]));
  most = wave_max(most);
  // The least exponent that holds it: 448 = 1.75 * 2^8.
  int e = int(most >> 7) - 8 + ((most & 0x7Fu) > 0x60u);
  e = max(e, 1);
  if (slot0 > 0) e = min(max(e, int(old_e)), 253);
  const float inv = scale_of(uint32_t(254 - e));
  const int drop = 127 + int(old_e) - e;  // 2^(old_e - e), which may underflow to 0
  const float f_old = scale_of(uint32_t(max(drop, 0)));
#pragma unroll
  for (int f = 0; f < F; ++f) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = x[f][j >> 1][2 * (j & 1)], b = x[f][j >> 1][2 * (j & 1) + 1];
      w[j] = e4m3x4(storable(a << 16) * inv, storable(a & 0xFFFF0000u) * inv, storable(b << 16) * inv,
                    storable(b & 0xFFFF0000u) * inv);
    }
    if (slot0 > 0 && e != int(old_e)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) old[f][j] = rescaled(old[f][j], f_old);
    }
    if (is_v) {
      // Bytes of tokens before slot0 in the lane's token group.
      const int keep = min(max(slot0 - 4 * (t >> 2), 0), 4);
      const uint32_t mask = keep == 4 ? 0xFFFFFFFFu : (1u << 8 * keep) - 1u;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint32_t*>(block + v_word(f, j, lane)) =
            (quad_transpose(w[j], t & 3) & ~mask) | (old[f][j] & mask);
    } else {
      *reinterpret_cast<u32x4*>(block + 1024 * f + 16 * lane) = t < slot0 ? old[f] : w;
    }
  }
  if (lane == 0) *scale = uint8_t(e);
}

// The touched pages of an append: one wave per (page, KV head, K or V).  Bound
// by the chain record -> rows and old block -> store for a decode batch (64
// tokens, 8 KV heads, D = 128: 4.5 us), by HBM for prompts (36864 tokens: 49-57 us,
// 4.0-4.6 TB/s of rows read and blocks written).
template <int D>
__global__ __launch_bounds__(256) void append8_kernel(const PageWrite* writes, size_t units, const uint16_t* k_new,
                                                      const uint16_t* v_new, unsigned char* k8, unsigned char* v8,
                                                      uint8_t* scales, int hkv) {
  const size_t u = size_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= units) return;
  const bool is_v = u & 1;
  const int h = int(u / 2 % hkv);
  const PageWrite w = writes[u / 2 / hkv];
  const size_t blk = size_t(w.page) * hkv + h;
  quantize_block<D>((is_v ? v_new : k_new) + (size_t(w.row0) * hkv + h) * D, size_t(hkv) * D, w.slot0, w.count,
                    (is_v ? v8 : k8) + blk * (16 * D), scales + 2 * blk + is_v, is_v, threadIdx.x & 63);
}

// Page lists of the whole-page calls, in the launch's arguments or in device
// memory.  Pools of up to 65536 pages list them in 16 bits: twice as many fit
// into 3.6 KB of arguments, and a longer list takes half the launches to stage
// (us a call, 16 bits against 32: 401 pages of 8 KV heads read back 10.3, 14.9;
// 1200 pages 25.0, 27.0; 4800 pages 120, 133).
struct PagesHere16 {
  static constexpr int kMax = 800;
  uint32_t pair[kMax], count[kMax / 8];  // source << 16 | destination; tokens - 1, 4 bits each
  void set(int i, int32_t dst, int32_t src, int32_t tokens) {
    pair[i] = uint32_t(src) << 16 | uint32_t(dst);
    count[i / 8] = (i % 8 ? count[i / 8] : 0) | uint32_t(tokens - 1) << (4 * (i % 8));
  }
  __device__ __forceinline__ int32_t dst(size_t i) const { return pair[i] & 0xFFFFu; }
  __device__ __forceinline__ int32_t src(size_t i) const { return pair[i] >> 16; }
  __device__ __forceinline__ int32_t tokens(size_t i) const { return int32_t(count[i / 8] >> (4 * (i % 8)) & 15) + 1; }
};
struct PagesHere32 {
  static constexpr int kMax = 400;
  int32_t pair[2 * kMax];
  uint8_t count[kMax];
  void set(int i, int32_t dst, int32_t src, int32_t tokens) {
    pair[2 * i] = dst;
    pair[2 * i + 1] = src;
    count[i] = uint8_t(tokens);
  }
  __device__ __forceinline__ int32_t dst(size_t i) const { return pair[2 * i]; }
  __device__ __forceinline__ int32_t src(size_t i) const { return pair[2 * i + 1]; }
  __device__ __forceinline__ int32_t tokens(size_t i) const { return count[i]; }
};
struct PagesAt {
  const int32_t* at;  // triples
  __device__ __forceinline__ int32_t dst(size_t i) const { return at[3 * i]; }
  __device__ __forceinline__ int32_t src(size_t i) const { return at[3 * i + 1]; }
  __device__ __forceinline__ int32_t tokens(size_t i) const { return at[3 * i + 2]; }
};

// Put a slice of a long list into device memory.
template <typename List>
__global__ __launch_bounds__(List::kMax) void stage_pages_kernel(List list, int32_t* at, int n) {
  const int i = threadIdx.x;
  if (i >= n) return;
  at[3 * i] = list.dst(i);
  at[3 * i + 1] = list.src(i);
  at[3 * i + 2] = list.tokens(i);
}

// Whole pages into the 8-bit format: one wave per block, as the append (256 pages
// of 8 KV heads, D = 128: 25 MB in 7.9 us; launch and ramp are half of it).
template <int D, typename List>
__global__ __launch_bounds__(256) void page_quantize_kernel(List list, size_t units, const uint16_t* src_k,
                                                            const uint16_t* src_v, unsigned char* k8,
                                                            unsigned char* v8, uint8_t* scales, int hkv) {
  const size_t u = size_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= units) return;
  const bool is_v = u & 1;
  const int h = int(u / 2 % hkv);
  const size_t i = u / 2 / hkv;
  const size_t dst = size_t(list.dst(i)) * hkv + h, src = size_t(list.src(i)) * hkv + h;
  quantize_block<D>((is_v ? src_v : src_k) + src * (16 * D), D, 0, list.tokens(i), (is_v ? v8 : k8) + dst * (16 * D),
                    scales + 2 * dst + is_v, is_v, threadIdx.x & 63);
}

// Two e4m3 bytes as packed bf16 at any scale (subnormal results included, which
// the scaled conversion flushes).
__device__ __forceinline__ u32x2 exact_bf16x4(uint32_t w, float scale) {
  const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  return u32x2{pack_bf16(a[0] * scale, a[1] * scale), pack_bf16(b[0] * scale, b[1] * scale)};
}

// And back: one wave per block, 32 bytes a lane and half out (256 pages 8.3 us;
// 2396 pages, 235 MB, 41.8 us: 5.6 TB/s, what was just written still in the
// caches).
template <int D, typename List>
__global__ __launch_bounds__(256) void page_dequantize_kernel(List list, size_t units, const unsigned char* k8,
                                                              const unsigned char* v8, const uint8_t* scales,
                                                              uint16_t* dst_k, uint16_t* dst_v, int hkv) {
  constexpr int F = D / 64;
  const size_t u = size_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= units) return;
  const int lane = threadIdx.x & 63, t = lane & 15, g = lane >> 4;
  const bool is_v = u & 1;
  const int h = int(u / 2 % hkv);
  const size_t i = u / 2 / hkv;
  const size_t dst = size_t(list.dst(i)) * hkv + h, src = size_t(list.src(i)) * hkv + h;
  const unsigned char* block = (is_v ? v8 : k8) + src * (16 * D);
  const float scale = scale_of(scales[2 * src + is_v]);
  uint16_t* out = (is_v ? dst_v : dst_k) + dst * (16 * D) + t * D + 16 * g;
  u32x4 w[F];
#pragma unroll
  for (int f = 0; f < F; ++f) {
    if (is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[f][j] = *reinterpret_cast<const uint32_t*>(block + v_word(f, j, lane));
    } else {
      w[f] = *reinterpret_cast<const u32x4*>(block + 1024 * f + 16 * lane);
    }
  }
#pragma unroll
  for (int f = 0; f < F; ++f) {
    if (is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[f][j] = quad_transpose(w[f][j], t & 3);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const u32x2 a = exact_bf16x4(w[f][2 * p], scale), b = exact_bf16x4(w[f][2 * p + 1], scale);
      *reinterpret_cast<u32x4*>(out + 64 * f + 8 * p) = u32x4{a[0], a[1], b[0], b[1]};
    }
  }
}

// Pages and their scales as they are: a workgroup per (page, K or V), or from
// host memory 64 that take them in turn: those keep the link busy, and more only
// queue on it beside attention (as in the copy of bf16 pages).
constexpr int kLinkWorkgroups8 = 64;
template <typename List>
__global__ __launch_bounds__(256) void page_copy8_kernel(List list, size_t units, const u32x4* src_k, const u32x4* src_v,
                                                         const uint8_t* src_s, u32x4* dst_k, u32x4* dst_v,
                                                         uint8_t* dst_s, int page_vecs, int hkv) {
  for (size_t u = blockIdx.x; u < units; u += gridDim.x) {
    const bool is_v = u & 1;
    const size_t dst = size_t(list.dst(u >> 1)), src = size_t(list.src(u >> 1));
    const u32x4* from = (is_v ? src_v : src_k) + src * page_vecs;
    u32x4* to = (is_v ? dst_v : dst_k) + dst * page_vecs;
    for (int v = threadIdx.x; v < page_vecs; v += 256) to[v] = from[v];
    for (int h = threadIdx.x; h < hkv; h += 256) dst_s[2 * (dst * hkv + h) + is_v] = src_s[2 * (src * hkv + h) + is_v];
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
struct Attn8Args {
  AttnArgs a;
  const unsigned char* k8;
  const unsigned char* v8;
  const uint8_t* scales;
};

// A 32-key step's operands as a lane holds them: its 16-byte vectors of the two
// pages' blocks.
template <int D>
struct Tile8 {
  static constexpr int F = D / 64;
  u32x4 k[2][F], v[2][F];
};

// A wave's state over NB blocks of 16 query columns: lane (col, grp) holds dims
// 16 blk + 4 grp + i of its column.  l: the lane's own keys' share of the
// softmax sum, of probabilities that are not rounded.
template <int D, int NB>
struct State8 {
  f32x4 acc[NB][D / 16];
  float m[NB], l[NB];
};

template <int D, int NB>
__device__ __forceinline__ void reset8(State8<D, NB>& s) {
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    s.m[b] = kNegBig;
    s.l[b] = 0.f;
#pragma unroll
    for (int blk = 0; blk < D / 16; ++blk) s.acc[b][blk] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

// The lane's part of a query row in the order of the K blocks: product s of a
// page takes dims 64 (s / 2) + 16 grp + 8 (s % 2) .. + 7.
template <int D>
__device__ __forceinline__ void load_q8(bf16x8 (&qf)[D / 32], const uint16_t* row, int grp) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
    qf[s] = *reinterpret_cast<const bf16x8*>(row + 64 * (s >> 1) + 16 * grp + 8 * (s & 1));
}

// S^T of one page: keys 4 grp + i against the wave's columns.
template <int D, int NB>
__device__ __forceinline__ void scores8(f32x4 (&sc)[NB], const u32x4 (&k)[D / 64], float scale,
                                        const bf16x8 (&qf)[NB][D / 32]) {
  constexpr int KS = D / 32;
  bf16x8 kf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const uint32_t w0 = k[s >> 1][2 * (s & 1)], w1 = k[s >> 1][2 * (s & 1) + 1];
    kf[s] = __builtin_bit_cast(bf16x8, u32x4{bf16_of<false>(w0, scale), bf16_of<true>(w0, scale),
                                             bf16_of<false>(w1, scale), bf16_of<true>(w1, scale)});
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[s], qf[b][s], acc, 0, 0, 0);
    sc[b] = acc;
  }
}

// O^T += V^T P^T of one step: block blk of V^T is word blk % 4 of vector blk / 4
// of each page.
template <int D, int NB>
__device__ __forceinline__ void values8(State8<D, NB>& st, const u32x4 (&v)[2][D / 64], float s0, float s1,
                                        const bf16x8 (&pb)[NB]) {
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk) {
    const uint32_t w0 = v[0][blk >> 2][blk & 3], w1 = v[1][blk >> 2][blk & 3];
    const bf16x8 vop = __builtin_bit_cast(bf16x8, u32x4{bf16_of<false>(w0, s0), bf16_of<true>(w0, s0),
                                                        bf16_of<false>(w1, s1), bf16_of<true>(w1, s1)});
#pragma unroll
    for (int b = 0; b < NB; ++b)
      st.acc[b][blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, pb[b], st.acc[b][blk], 0, 0, 0);
  }
}

// x, or NaN where hit (0 or a positive count) is not 0.
__device__ __forceinline__ float nan_if(float hit, float x) {
  const uint32_t any = min(__builtin_bit_cast(uint32_t, hit), 1u);
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) | any * 0x7FC00000u);
}

// The lane's V bytes of a step whose keys are not all visible to every column.
// Slots at or past kend may hold anything: their bytes become zero (0 * NaN is
// NaN).  A NaN among the visible keys must reach the columns that see it and no
// other: the bytes become zero for the product, and a second product, of ones
// where they stood against ones where a column sees the key, makes NaN of what
// it reaches.
template <int D, int NB>
__device__ __forceinline__ void masked_values8(State8<D, NB>& st, u32x4 (&v)[2][D / 64], int k0, int kend,
                                               const int (&lim)[NB], int grp) {
  constexpr int F = D / 64;
  uint32_t bad = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int live = min(max(kend - (k0 + 16 * t + 4 * grp), 0), 4);
    const uint32_t mask = live == 4 ? 0xFFFFFFFFu : (1u << 8 * live) - 1u;
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[t][f][j] &= mask;
        bad |= (v[t][f][j] & 0x7F7F7F7Fu) + 0x01010101u;  // bit 7 of a byte that is 0x7F
      }
  }
  if (!__any(bad & 0x80808080u)) return;
  PFX_KEEP_BRANCH();
  bf16x8 sees[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    u32x4 w;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int key = k0 + 16 * (p >> 1) + 4 * grp + 2 * (p & 1);
      w[p] = (uint32_t(~((lim[b] - key) >> 31)) & 0x3F80u) | (uint32_t(~((lim[b] - key - 1) >> 31)) & 0x3F800000u);
    }
    sees[b] = __builtin_bit_cast(bf16x8, w);
  }
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk) {
    uint32_t ones[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t w = v[t][blk >> 2][blk & 3];
      const uint32_t nan = (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;  // 1 in each NaN byte
      ones[t] = nan * 0x38u;                                                       // 1.0
      v[t][blk >> 2][blk & 3] = w & ~(nan * 0xFFu);
    }
    const bf16x8 vop = __builtin_bit_cast(bf16x8, u32x4{bf16_of<false>(ones[0], 1.f), bf16_of<true>(ones[0], 1.f),
                                                        bf16_of<false>(ones[1], 1.f), bf16_of<true>(ones[1], 1.f)});
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const f32x4 hit =
          __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, sees[b], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[b][blk][i] = nan_if(hit[i], st.acc[b][blk][i]);
    }
  }
}

// Maximum and sum over lanes l and l ^ 32 (a column of a 32 x 32 product).
__device__ __forceinline__ float pair_max(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  row_swap32(a, b);
  return __builtin_elementwise_maximum(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float pair_sum(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  row_swap32(a, b);
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// Raise the running maxima of columns that pass them by more than the slack.
template <int D, int NB>
__device__ __forceinline__ void raise8(State8<D, NB>& st, const float (&mx)[NB], float scale_log2) {
  bool pass = false;
#pragma unroll
  for (int b = 0; b < NB; ++b) pass = pass || mx[b] * scale_log2 > st.m[b] + kRescaleSlack;
  if (!__any(pass)) return;
  PFX_KEEP_BRANCH();
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const float cm = column_max(mx[b]) * scale_log2;
    const float mnew = cm > st.m[b] + kRescaleSlack ? cm : st.m[b];
    const float alpha = fast_exp2(st.m[b] - mnew);
    st.l[b] *= alpha;
#pragma unroll
    for (int blk = 0; blk < D / 16; ++blk) st.acc[b][blk] *= alpha;
    st.m[b] = mnew;
  }
}

// P of one step as the B operand, its sum added to l.  The probabilities are
// rounded to bf16 for the product (each by at most 2^-8 of itself, as the output
// is; their errors average out over the keys, and a second term would double the
// matrix work); l sums them as they are, so lse does not see the rounding.
__device__ __forceinline__ bf16x8 probabilities8(const f32x4& s0, const f32x4& s1, float scale_log2, float m,
                                                 float& l) {
  float p[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = fast_exp2(fmaf(s0[i], scale_log2, -m));
    p[4 + i] = fast_exp2(fmaf(s1[i], scale_log2, -m));
  }
  l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
  return __builtin_bit_cast(bf16x8, u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]),
                                          pack_bf16(p[6], p[7])});
}

__device__ __forceinline__ float max8(const f32x4& a, const f32x4& b) {
  // IEEE maximum: no NaN canonicalisation of the matrix unit's results.
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_elementwise_maximum(a[i], b[i]);
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x[0], x[1]),
                                       __builtin_elementwise_maximum(x[2], x[3]));
}

// One 32-key step in registers against the wave's columns.  sc: the pages'
// scale bytes, K in bits 0-7, V in bits 8-15.  MASK: some column may not see all
// of its keys.
template <int D, int NB, bool MASK>
__device__ __forceinline__ void step8(State8<D, NB>& st, Tile8<D>& tile, uint32_t sc0, uint32_t sc1,
                                      const bf16x8 (&qf)[NB][D / 32], const int (&lim)[NB], int k0, int kend,
                                      bool causal, int grp, float scale_log2) {
  f32x4 s[2][NB];
  scores8<D, NB>(s[0], tile.k[0], scale_of(sc0 & 0xFFu), qf);
  if (NB == 2 && D == 128) __builtin_amdgcn_sched_barrier(0);  // one page's converted keys at a time: registers
  scores8<D, NB>(s[1], tile.k[1], scale_of(sc1 & 0xFFu), qf);
  if (MASK && (causal || k0 + kStepKeys > kend)) {
    PFX_KEEP_BRANCH();
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = k0 + 16 * t + 4 * grp + i;
          if (key >= kend || key > lim[b]) s[t][b][i] = -INFINITY;
        }
    masked_values8<D, NB>(st, tile.v, k0, kend, lim, grp);
  }
  float mx[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) mx[b] = max8(s[0][b], s[1][b]);
  raise8<D, NB>(st, mx, scale_log2);
  bf16x8 pb[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) pb[b] = probabilities8(s[0][b], s[1][b], scale_log2, st.m[b], st.l[b]);
  values8<D, NB>(st, tile.v, scale_of(sc0 >> 8), scale_of(sc1 >> 8), pb);
}

// ---------------------------------------------------------------------------
// Decode pieces: one workgroup each.  The waves split the piece's keys, every
// wave taking every W-th step for all of its columns, so that each byte of the
// cache is read and converted by one wave and nothing waits for a barrier until
// the waves' states meet in LDS at the end.  (A suffix piece has G columns, one
// block of the matrix unit: with columns split over the waves instead, three of
// four would idle.)  Pieces of more than 32 columns go to two pairs of waves,
// 32 columns each, which split the keys in two: more columns a wave would not
// fit the registers of two workgroups on a compute unit (64 columns as one block
// of each of four waves: 19.8 us against 16.3 with 64 requests on 4 prefixes of
// 2048 tokens, 32 query and 8 KV heads, D = 128).  Two steps' loads, 64 (D = 128)
// or 32 bytes a lane each, are in flight while a third is multiplied.
//
// Bound by HBM: that batch's 56 MB take 15.2-16.5 us (3.4-3.7 TB/s; few enough bytes
// that the record -> block ids -> first loads chain and the joins show), 16 agents
// with uneven requests, 398 MB, 85.6 us (4.65 TB/s, of 4.9 that a large copy
// reaches); calls over pools in turn, with nothing of them left in the last-level
// cache, 23.4 and 98 us with the merge instead of 18.4 and 91.  The joins' results go to merge8_kernel in fp32.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void load_tile8(Tile8<D>& t, const Attn8Args& x, int b0, int b1, int lane) {
  const size_t o0 = size_t(uint32_t(b0)) * (16 * D), o1 = size_t(uint32_t(b1)) * (16 * D);
#pragma unroll
  for (int f = 0; f < D / 64; ++f) {
    t.k[0][f] = *reinterpret_cast<const u32x4*>(x.k8 + o0 + 1024 * f + 16 * lane);
    t.k[1][f] = *reinterpret_cast<const u32x4*>(x.k8 + o1 + 1024 * f + 16 * lane);
    t.v[0][f] = *reinterpret_cast<const u32x4*>(x.v8 + o0 + 1024 * f + 16 * lane);
    t.v[1][f] = *reinterpret_cast<const u32x4*>(x.v8 + o1 + 1024 * f + 16 * lane);
  }
}

constexpr int kDecode8Lds(int D) { return 4 * 2 * (D / 16) * 64 * 16 + 4 * 2 * 16 * 8; }

// NB column blocks a wave, KS waves on the keys (and 4 / KS on the columns).
template <int D, int NB, int KS>
__device__ __forceinline__ void decode8_piece(const Attn8Args& x, const SegHead& h, const int32_t* tok,
                                              const int32_t* out, const int32_t* steps, unsigned char* smem) {
  constexpr int CH = D / 16;
  const AttnArgs& a = x.a;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int key_wave = wave % KS, col0 = wave / KS * (16 * NB);
  const int G = a.group;

  // Lane 32 p + i holds the block id and the scales of page p of the wave's i-th
  // step (at most 32).
  const int mine = key_wave + KS * (lane & 31);
  int blk = 0;
  uint32_t sc = 0;
  if (mine < h.nsteps) {
    blk = steps[2 * mine + (lane >> 5)];
    sc = *reinterpret_cast<const uint16_t*>(x.scales + 2 * size_t(uint32_t(blk)));
  }
  auto at = [&](uint32_t r, int i, int page) { return __builtin_amdgcn_readlane(int(r), i + 32 * page); };
  bf16x8 qf[NB][D / 32];
  int lim[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int c = col0 + 16 * b + col;
    const int j = c < h.ncols ? c >> a.group_shift : 0;
    lim[b] = h.causal ? tok[j] + h.causal_base : 0x7fffffff;
    load_q8<D>(qf[b], a.q + (size_t(tok[j]) * a.hq + h.kv_head * G + (c & (G - 1))) * D, grp);
  }
  State8<D, NB> st;
  reset8(st);
  const int n = h.nsteps > key_wave ? (h.nsteps - key_wave + KS - 1) / KS : 0;
  // The wave's steps from the last to the first: those with a mask (the end of
  // the item, and in a request of several rows the up to 16 keys before it, two
  // steps at most) come first, apart from the loop.  Two steps are in flight
  // while one is multiplied.
  auto load = [&](Tile8<D>& t, int i) __attribute__((always_inline)) {
    if (i < n) load_tile8<D>(t, x, at(blk, n - 1 - i, 0), at(blk, n - 1 - i, 1), lane);
  };
  auto run = [&](auto mask, Tile8<D>& t, int i) __attribute__((always_inline)) {
    const int j = n - 1 - i;
    step8<D, NB, mask.value>(st, t, uint32_t(at(sc, j, 0)), uint32_t(at(sc, j, 1)), qf, lim,
                             h.k0 + kStepKeys * (key_wave + KS * j), h.kend, h.causal != 0, grp, a.scale_log2);
  };
  Tile8<D> t0, t1, t2;
  load(t0, 0);
  load(t1, 1);
  if (n > 0) {
    load(t2, 2);
    run(std::true_type(), t0, 0);
  }
  if (n > 1) {
    load(t0, 3);
    run(std::true_type(), t1, 1);
  }
  for (int i = 2; i < n; i += 3) {
    load(t1, i + 2);
    run(std::false_type(), t2, i);
    if (i + 1 >= n) break;
    load(t2, i + 3);
    run(std::false_type(), t0, i + 1);
    if (i + 2 >= n) break;
    load(t0, i + 4);
    run(std::false_type(), t1, i + 2);
  }

  // The waves' states meet: (m, l) of every column, then the accumulators scaled
  // to the common maximum, of which each wave of the group adds up its share.
  f32x2* ml = reinterpret_cast<f32x2*>(smem + 4 * NB * CH * 64 * 16);
  f32x4* accs = reinterpret_cast<f32x4*>(smem);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const float l = column_sum(st.l[b]);
    if (grp == 0) ml[(wave * NB + b) * 16 + col] = f32x2{st.m[b], l};
  }
  __syncthreads();
  float mt[NB], lt[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    f32x2 p[KS];
    mt[b] = kNegBig;
    lt[b] = 0.f;
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      p[w] = ml[((wave / KS * KS + w) * NB + b) * 16 + col];
      mt[b] = fmaxf(mt[b], p[w][0]);
    }
#pragma unroll
    for (int w = 0; w < KS; ++w) lt[b] += fast_exp2(p[w][0] - mt[b]) * p[w][1];
    const float f = fast_exp2(st.m[b] - mt[b]);
#pragma unroll
    for (int k = 0; k < CH; ++k) accs[((wave * NB + b) * CH + k) * 64 + lane] = st.acc[b][k] * f;
  }
  __syncthreads();
  float* o_part = reinterpret_cast<float*>(a.plan.o_part);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    int late = threadIdx.x;
    asm("" : "+v"(late));  // the column anew: kept through the loop, it takes a register that is missing there
    const int c = col0 + 16 * b + (late & 15);
    if (c >= h.ncols) continue;
    const size_t row = size_t(out[c >> a.group_shift] + (c & (G - 1)));
#pragma unroll
    for (int k = 0; k < CH / KS; ++k) {
      const int ch = key_wave * (CH / KS) + k;
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KS; ++w) s += accs[(((wave / KS * KS + w) * NB + b) * CH + ch) * 64 + lane];
      *reinterpret_cast<f32x4*>(o_part + row * D + 16 * ch + 4 * grp) = s;
    }
    if (key_wave == 0 && grp == 0) *reinterpret_cast<f32x2*>(a.plan.l_part + 2 * row) = f32x2{mt[b], lt[b]};
  }
}

template <int D>
__global__ __launch_bounds__(256, 2) void decode8_kernel(Attn8Args x) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[kDecode8Lds(D)];
  const SegShape shape = x.a.plan.seg_shape;
  const int32_t* rec = reinterpret_cast<const int32_t*>(x.a.plan.segs) + size_t(blockIdx.x) * (shape.vecs() * 4);
  const SegHead h = *reinterpret_cast<const SegHead*>(rec);
  const int32_t* tok = rec + SegShape::kHeadVecs * 4;
  const int32_t* out = tok + 4 * shape.row_vecs;
  const int32_t* steps = out + 4 * shape.row_vecs;
  if (h.ncols <= 16) decode8_piece<D, 1, 4>(x, h, tok, out, steps, smem);
  else if (h.ncols <= 32) decode8_piece<D, 1, 2>(x, h, tok, out, steps, smem);
  else decode8_piece<D, 2, 2>(x, h, tok, out, steps, smem);
}

// Merged states of one row's parts: four dims of unnormalised values, with
// (m, l) of each part.  kMerge8Batch parts are requested before any is used.
constexpr int kMerge8Batch = 8;
struct Merged8 {
  float mx = kNegBig, z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
};

__device__ __forceinline__ Merged8 merge8(const float* op, size_t o_stride, const f32x2* lp, size_t l_stride, int parts) {
  Merged8 s;
  for (int k0 = 0; k0 < parts; k0 += kMerge8Batch) {
    f32x2 ml[kMerge8Batch];
    f32x4 ov[kMerge8Batch];
#pragma unroll
    for (int i = 0; i < kMerge8Batch; ++i) {
      if (k0 + i < parts) {
        ml[i] = lp[size_t(k0 + i) * l_stride];
        ov[i] = *reinterpret_cast<const f32x4*>(op + size_t(k0 + i) * o_stride);
      } else {
        ml[i] = f32x2{kNegBig, 0.f};
        ov[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    float m2 = s.mx;
#pragma unroll
    for (int i = 0; i < kMerge8Batch; ++i) m2 = fmaxf(m2, ml[i][0]);
    const float f = fast_exp2(s.mx - m2);
    s.mx = m2;
    s.z *= f;
    s.acc *= f;
#pragma unroll
    for (int i = 0; i < kMerge8Batch; ++i) {
      const float w = fast_exp2(ml[i][0] - s.mx);
      s.z += w * ml[i][1];
      s.acc += w * ov[i];
    }
  }
  return s;
}

// Four dims of a final row.  A row sees its own token: z > 0, or NaN.
__device__ __forceinline__ void write_merged8(const AttnArgs& a, size_t orow, int D, int dim, const Merged8& s) {
  const float inv = 1.0f / s.z;
  *reinterpret_cast<u32x2*>(a.o + orow * D + dim) =
      u32x2{pack_bf16(s.acc[0] * inv, s.acc[1] * inv), pack_bf16(s.acc[2] * inv, s.acc[3] * inv)};
  if (a.lse && dim == 0) a.lse[orow] = (s.mx + log2f(s.z)) * kLn2;
}

// Decode rows from their pieces' states: one thread per four dims of a row.
// Bound by latency: head -> states -> store, 4.9 us for 64 rows of 32 heads, 5.4
// for the uneven batch above.
template <int D>
__global__ __launch_bounds__(256) void merge8_kernel(AttnArgs a, int n_tok) {
  constexpr int SL = D / 4;
  const size_t t = size_t(blockIdx.x) * 256 + threadIdx.x;
  if (t >= size_t(n_tok) * a.hq * SL) return;
  const int sl = int(t % SL), qh = int(t / SL % a.hq), m = int(t / SL / a.hq);
  const size_t unit = size_t(m) * a.hkv + (qh >> a.group_shift);
  MergeHead mh = {int32_t(unit) * a.merge_parts, a.merge_parts};
  if (!a.merge_parts) mh = a.plan.merge_head[unit];
  const size_t row0 = size_t(mh.base) * a.group + (qh & (a.group - 1));
  const int tok = a.plan.merge_tok[m];
  write_merged8(a, size_t(tok) * a.hq + qh, D, 4 * sl,
                merge8(reinterpret_cast<const float*>(a.plan.o_part) + row0 * D + 4 * sl, size_t(a.group) * D,
                       reinterpret_cast<const f32x2*>(a.plan.l_part) + row0, a.group, mh.nparts));
}

// ---------------------------------------------------------------------------
// Extend blocks: one workgroup per block of up to 128 query columns (or per
// piece of a cut block), 32 columns a wave, the keys through an LDS ring of
// four 32-key stages that all waves read.  A wave copies one quarter of a stage
// (a page's K or V block) and its scale.
//
// The products are 32 x 32 x 16: 32 keys, or 32 dims, against the wave's 32
// columns.  A step has 144 vector ALU instructions beside its products (half of
// them convert the bytes), and a 32 x 32 x 16 product leaves the vector ALU more
// slots than the two 16 x 16 x 32 of the same work (with 10 instructions beside
// it 22.1 ns against 26.9).
//
// Bound by the matrix unit's sustained rate, which falls with the card's power:
// 36864 rows of 32 requests on 3 prefixes of 4096 tokens, 2.98 TFLOP, take
// 2.93-3.34 ms from card to card (0.9-1.0 PFLOP/s at 1.9-2.2 GHz; the library's
// 8192^3 bf16 product reaches 1.135).  With 16 x 16 x 32 products the loop took 6 %
// more cycles and the same time, at 2.26 GHz instead of 2.08.  Converting K and V once a workgroup into bf16 stages
// instead of in every wave cost more in LDS than it saved (3.3-3.6 ms).
//   S^T: rows are keys (page 0's, page 1's), lane (r, g) takes dims 16 (2 m + g)
//     .. + 15 of key r with its m-th load: products 2 m and 2 m + 1.  It then
//     holds keys 8 q + 4 g + i of column lane % 32 in register 4 q + i.
//   O^T: product (b, page) takes tokens 4 g .. + 3 and 8 + 4 g .. + 3 of the page,
//     which are the lane's own probabilities 8 page .. + 7, and rows r = 16 f + r'
//     are dims D / 2 f + 16 b + r': of V's vectors of token groups g and g + 2,
//     word b (D = 128, half f), or word 2 f + b (D = 64).
// ---------------------------------------------------------------------------
constexpr int kStages8 = 4;
template <int D>
constexpr int kTile8Bytes = 16 * D;
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Copy a block into LDS at lds_addr as it lies.
template <int D>
__device__ __forceinline__ void copy_tile8(const unsigned char* base, uint32_t lds_addr, int lane) {
#pragma unroll
  for (int f = 0; f < D / 64; ++f) copy16_to_lds(base + 1024 * f + 16 * lane, lds_addr + 1024 * f);
}

// A wave's state: lane (col, g) holds rows 8 q + 4 g + i of each 32-dim block of
// its column in register 4 q + i; l: its own keys' share of the softmax sum.
template <int D>
struct State32 {
  f32x16 acc[D / 32];
  float m, l;
};

// First of the four dims in registers 4 q .. 4 q + 3 of block b.
template <int D>
__device__ __forceinline__ int quad_dim(int b, int q, int g) { return D / 2 * (q >> 1) + 16 * b + 8 * (q & 1) + 4 * g; }

// The lane's V words of one page: of block b, tokens 4 g .. and 8 + 4 g ...
template <int D>
struct Words8 {
  uint32_t lo[D / 32], hi[D / 32];
};

template <int D>
__device__ __forceinline__ void read_v8(Words8<D>& w, const unsigned char* tile, int lane) {
  const int f = lane >> 4 & 1, at = 256 * (lane >> 5) + 16 * (lane & 15);
  if constexpr (D == 128) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + 1024 * f + at);
    const u32x4 y = *reinterpret_cast<const u32x4*>(tile + 1024 * f + at + 512);
#pragma unroll
    for (int b = 0; b < 4; ++b) w.lo[b] = x[b], w.hi[b] = y[b];
  } else {
    const u32x2 x = *reinterpret_cast<const u32x2*>(tile + 8 * f + at);
    const u32x2 y = *reinterpret_cast<const u32x2*>(tile + 8 * f + at + 512);
#pragma unroll
    for (int b = 0; b < 2; ++b) w.lo[b] = x[b], w.hi[b] = y[b];
  }
}

__device__ __forceinline__ bf16x8 operand8(uint32_t w0, uint32_t w1, float scale) {
  return __builtin_bit_cast(bf16x8, u32x4{bf16_of<false>(w0, scale), bf16_of<true>(w0, scale),
                                          bf16_of<false>(w1, scale), bf16_of<true>(w1, scale)});
}

// masked_values8 on the words of a step's two pages.
template <int D>
__device__ __forceinline__ void masked_words8(State32<D>& st, Words8<D> (&v)[2], int k0, int kend, int lim, int g) {
  auto keep = [](int n) { return n >= 4 ? 0xFFFFFFFFu : (1u << 8 * max(n, 0)) - 1u; };
  uint32_t bad = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int live = kend - (k0 + 16 * t + 4 * g);
    const uint32_t m0 = keep(live), m1 = keep(live - 8);
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
      v[t].lo[b] &= m0;
      v[t].hi[b] &= m1;
      bad |= ((v[t].lo[b] & 0x7F7F7F7Fu) + 0x01010101u) | ((v[t].hi[b] & 0x7F7F7F7Fu) + 0x01010101u);
    }
  }
  if (!__any(bad & 0x80808080u)) return;
  PFX_KEEP_BRANCH();
  bf16x8 sees[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    u32x4 w;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int key = k0 + 16 * t + 8 * (p >> 1) + 4 * g + 2 * (p & 1);
      w[p] = (uint32_t(~((lim - key) >> 31)) & 0x3F80u) | (uint32_t(~((lim - key - 1) >> 31)) & 0x3F800000u);
    }
    sees[t] = __builtin_bit_cast(bf16x8, w);
  }
  // The NaN bytes of w become zero; returns ones (as bytes) in their places.
  auto take = [](uint32_t& w) {
    const uint32_t nan = (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
    w &= ~(nan * 0xFFu);
    return nan * 0x38u;
  };
#pragma unroll
  for (int b = 0; b < D / 32; ++b) {
    f32x16 hit = {};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t lo = v[t].lo[b], hi = v[t].hi[b];
      const uint32_t o0 = take(lo), o1 = take(hi);
      v[t].lo[b] = lo;
      v[t].hi[b] = hi;
      hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand8(o0, o1, 1.f), sees[t], hit, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) st.acc[b][i] = nan_if(hit[i], st.acc[b][i]);
  }
}

// Two steps (two: the second exists) against the wave's columns.  sc0, sc1: the
// steps' scale bytes in LDS (K of pages 0 and 1, V of pages 0 and 1).  MASK: some
// column may not see some of their keys.
template <int D, bool MASK>
__device__ __forceinline__ void pair8(State32<D>& st, const unsigned char* st0, const unsigned char* st1,
                                      const uint32_t* sc0, const uint32_t* sc1, const bf16x8 (&qf)[D / 16], int lim,
                                      const Item& it, int s, bool two, const StepMarks& mk, int lane,
                                      float scale_log2) {
  constexpr int TB = kTile8Bytes<D>;
  const int g = lane >> 5;
  f32x16 sc[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const unsigned char* k = (u ? st1 : st0) + (lane >> 4 & 1) * TB + 256 * g + 16 * (lane & 15);
    const float scale = scale_of((u ? sc1 : sc0)[lane >> 4 & 1]);
    f32x16 x = {};
#pragma unroll
    for (int m = 0; m < D / 32; ++m) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(k + 512 * m);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand8(w[0], w[1], scale), qf[2 * m], x, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand8(w[2], w[3], scale), qf[2 * m + 1], x, 0, 0, 0);
    }
    sc[u] = x;
  }
  auto where = [&](int u) {
    StepPos p = step_pos(it, s, mk.s0_steps);
    if (u) p = two ? step_pos(it, s + 1, mk.s0_steps) : StepPos{p.list_off, p.kend, p.kend, p.seg};
    return p;
  };
  if constexpr (MASK) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const StepPos p = where(u);
      const int last = p.seg == 1 ? min(lim, p.kend - 1) : p.kend - 1;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (p.k0 + 8 * (i >> 2) + 4 * g + (i & 3) > last) sc[u][i] = -INFINITY;
    }
  }
  // IEEE maximum: no NaN canonicalisation of the matrix unit's results.
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = __builtin_elementwise_maximum(sc[0][i], sc[1][i]);
#pragma unroll
  for (int w = 8; w >= 1; w /= 2)
#pragma unroll
    for (int i = 0; i < w; ++i) x[i] = __builtin_elementwise_maximum(x[i], x[i + w]);
  if (__any(x[0] * scale_log2 > st.m + kRescaleSlack)) {
    PFX_KEEP_BRANCH();
    const float cm = pair_max(x[0]) * scale_log2;
    const float mnew = cm > st.m + kRescaleSlack ? cm : st.m;
    const float alpha = fast_exp2(st.m - mnew);
    st.l *= alpha;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) st.acc[b] *= alpha;
    st.m = mnew;
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const unsigned char* stage = u ? st1 : st0;
    const uint32_t* scale = u ? sc1 : sc0;
    if (u) asm volatile("" ::: "memory");  // the second step's V reads stay after the first step's products
    Words8<D> v[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) read_v8<D>(v[t], stage + (2 + t) * TB, lane);
    if constexpr (MASK) {
      const StepPos p = where(u);
      masked_words8<D>(st, v, p.k0, p.kend, p.seg == 1 ? lim : 0x7fffffff, g);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // Rounded to bf16 for the product, summed as they are (as probabilities8).
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = fast_exp2(fmaf(sc[u][8 * t + i], scale_log2, -st.m));
      st.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]),
                                                         pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])});
      const float vs = scale_of(uint32_t(__builtin_amdgcn_readfirstlane(int(scale[2 + t]))));
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
        st.acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand8(v[t].lo[b], v[t].hi[b], vs), pb, st.acc[b], 0, 0, 0);
    }
  }
}

template <int D>
constexpr int kExtend8Lds = kStages8 * 4 * kTile8Bytes<D> + kStages8 * 16;

// C: a piece of a cut block (*ckp), its state left in the piece's slot.
template <int D, bool C>
__device__ __forceinline__ void extend8_block(const Attn8Args& x, const Item* itp, unsigned char* smem,
                                              const Chunk* ckp) {
  constexpr int NS = kStages8, TB = kTile8Bytes<D>;
  const AttnArgs& a = x.a;
  auto ring = reinterpret_cast<unsigned char (*)[4 * TB]>(smem);
  auto scale = reinterpret_cast<uint32_t (*)[4]>(smem + NS * 4 * TB);  // K page 0, K page 1, V page 0, V page 1
  // Issued before the block's scalar load.
  const int lead = C ? ckp->pages[threadIdx.x & 3] : itp->first_pages[threadIdx.x & (kItemPages - 1)];
  const Item it = *itp;
  const int first = C ? ckp->st0 : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const int h = it.kv_head, G = a.group;

  const int p0b = it.s0_kbeg >> 4;
  const int p0n = it.s0_kend > it.s0_kbeg ? ((it.s0_kend + 15) >> 4) - p0b : 0;
  const int p1b = it.s1_kbeg >> 4;
  const int p1n = it.s1_kend > it.s1_kbeg ? ((it.s1_kend + 15) >> 4) - p1b : 0;
  PageWindow pw;
  pw.list = a.plan.page_list;
  pw.s0_at = it.s0_page_off + p0b;
  pw.s1_at = it.s1_page_off + p1b;
  pw.p0n = p0n;
  pw.ntab = p0n + p1n;
  pw.w0 = 0;
  if constexpr (C) {
    // The window of step first + 2, the first one that is looked up.
    const int s0_steps = (it.s0_kend - it.s0_kbeg + kStepKeys - 1) / kStepKeys;
    pw.w0 = (2 * (first + 2) + (first + 2 >= s0_steps ? p0n - 2 * s0_steps : 0)) & ~63;
  }
  pw.cur = window_entry(pw, pw.w0 + lane);
  pw.next = window_entry(pw, pw.w0 + 64 + lane);

  const int c = 32 * wave + (lane & 31);
  const bool any = 32 * wave < it.row_count * G, valid = c < it.row_count * G;
  // Padding columns repeat the item's first row.
  const int tok = it.tok0 + (valid ? c >> a.group_shift : 0);
  const int lim = tok + it.causal_base, orow = tok * a.hq + h * G + (c & (G - 1));
  bf16x8 qf[D / 16];
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
    qf[k] = *reinterpret_cast<const bf16x8*>(a.q + size_t(orow) * D + 16 * (2 * (k >> 1) + g) + 8 * (k & 1));
  State32<D> st;
  st.m = kNegBig;
  st.l = 0.f;
#pragma unroll
  for (int b = 0; b < D / 32; ++b) st.acc[b] = f32x16{};
  // Lane 0's column holds the wave's lowest token.
  const int lim_lo = __builtin_amdgcn_readfirstlane(lim);
  const StepMarks mk = step_marks(it, p0n, lim_lo);
  const int nsteps = C ? ckp->st1 : mk.nsteps;
  uint32_t sreg[2];  // the scales of this wave's tiles of the pair in flight
  auto issue = [&](int stage, int u, int page) __attribute__((always_inline)) {
    const size_t blk = size_t(page) * a.hkv + h;
    sreg[u] = x.scales[2 * blk + (wave >> 1)];
    copy_tile8<D>(((wave >> 1) ? x.v8 : x.k8) + blk * TB, lds_address(ring[stage]) + wave * TB, lane);
  };
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    sreg[u] = 127;  // of a step that does not exist: its zeros stay zeros
    if (first + u < nsteps)
      issue(u, u, __builtin_amdgcn_readfirstlane(
                      __builtin_amdgcn_readlane(lead, C ? 2 * u + (wave & 1) : step_entry(mk, u, wave))));
  }
  // Two steps per barrier: wait for the pair's copies, publish its scales, meet
  // (the other pair of stages is free then), refill that, run the pair.
  auto pair = [&](auto mask, int s) __attribute__((always_inline)) {
    const int stage = (s - first) & 2;
    wait_vmcnt(0);
    if (lane == 0) {
      scale[stage][wave] = sreg[0];
      scale[stage + 1][wave] = sreg[1];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sreg[u] = 127;
      if (s + 2 + u < nsteps) issue((stage ^ 2) + u, u, window_page(pw, step_entry(mk, s + 2 + u, wave), lane));
    }
    if (any)
      pair8<D, mask.value>(st, ring[stage], ring[stage + 1], scale[stage], scale[stage + 1], qf, lim, it, s,
                           s + 1 < nsteps, mk, lane, a.scale_log2);
  };
  // Pairs with keys that some column does not see (an odd last step pairs with an
  // empty one) run in a loop of their own, so that the others' stays short and
  // keeps its registers.
  auto masked = [&](int s) {
    return s + 1 >= nsteps || s + 1 >= mk.diag || s == mk.tail0 || s + 1 == mk.tail0 || s == mk.tail1 || s + 1 == mk.tail1;
  };
  for (int s = first; s < nsteps;) {
    for (; s < nsteps && !masked(s); s += 2) pair(std::false_type(), s);
    for (; s < nsteps && masked(s); s += 2) pair(std::true_type(), s);
  }
  const float l = pair_sum(st.l);
  if constexpr (C) {
    const int slot = ckp->slot;
    if (slot >= 0) {
      // The piece's state as the lanes hold it: [wave][block][q][lane] f32x4.
      if (!any) return;
      float* out = a.plan.xo_part + size_t(slot) * (kExtendTileCols * D) + wave * (32 * D) + 4 * lane;
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          __builtin_nontemporal_store(
              f32x4{st.acc[b][4 * q], st.acc[b][4 * q + 1], st.acc[b][4 * q + 2], st.acc[b][4 * q + 3]},
              reinterpret_cast<f32x4*>(out + 256 * (4 * b + q)));
      if (g == 0) reinterpret_cast<f32x2*>(a.plan.xl_part)[size_t(slot) * kExtendTileCols + c] = f32x2{st.m, l};
      return;
    }
  }
  if (!valid) return;
  const float inv = 1.0f / l;  // a row sees its own token: l > 0, or NaN
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<u32x2*>(a.o + size_t(orow) * D + quad_dim<D>(b, q, g)) =
          u32x2{pack_bf16(st.acc[b][4 * q] * inv, st.acc[b][4 * q + 1] * inv),
                pack_bf16(st.acc[b][4 * q + 2] * inv, st.acc[b][4 * q + 3] * inv)};
  if (a.lse && g == 0) a.lse[orow] = (st.m + log2f(l)) * kLn2;
}

template <int D, bool C>
__global__ __launch_bounds__(256, 2) void extend8_kernel(Attn8Args x) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kExtend8Lds<D>];
  if constexpr (C) {
    const Chunk* ck = x.a.plan.chunks + blockIdx.x;
    extend8_block<D, true>(x, x.a.plan.items + ck->item, smem, ck);
  } else {
    extend8_block<D, false>(x, x.a.plan.items + blockIdx.x, smem, nullptr);
  }
}

// The cut extend blocks' rows from their pieces' states.  A workgroup takes all
// dims of 1024 / D columns: a thread merges four of them (two lanes' places in
// the pieces' states, 128 bytes or more in a row), and the rows go out through
// LDS, 8 bytes a thread, consecutive (8-byte stores from the merging threads, 16
// bytes apart by row, took 1 us more for 80 blocks).
template <int D>
__global__ __launch_bounds__(256) void chunk_merge8_kernel(AttnArgs a) {
  constexpr int CW = 1024 / D;                             // columns of a workgroup
  constexpr int kPerItem = kExtendTileCols / CW;           // workgroups per block
  __shared__ u32x2 rows[CW][D / 4];
  __shared__ float lses[CW];
  const ChunkMerge cm = a.plan.chunk_merge[blockIdx.x / kPerItem];
  const int c0 = int(blockIdx.x) % kPerItem * CW;
  const Item* it = a.plan.items + cm.item;
  {
    const int quad = threadIdx.x / (2 * CW), g = threadIdx.x / CW % 2, col = threadIdx.x % CW, c = c0 + col;
    if ((c >> a.group_shift) < it->row_count) {
      const size_t at = size_t(c / 32) * (32 * D) + 256 * quad + 4 * (32 * g + c % 32);
      const Merged8 s = merge8(a.plan.xo_part + size_t(cm.base) * (kExtendTileCols * D) + at, kExtendTileCols * D,
                               reinterpret_cast<const f32x2*>(a.plan.xl_part) + size_t(cm.base) * kExtendTileCols + c,
                               kExtendTileCols, cm.nparts);
      const float inv = 1.0f / s.z;
      const int dim = quad_dim<D>(quad >> 2, quad & 3, g);
      rows[col][dim / 4] = u32x2{pack_bf16(s.acc[0] * inv, s.acc[1] * inv), pack_bf16(s.acc[2] * inv, s.acc[3] * inv)};
      if (dim == 0) lses[col] = (s.mx + log2f(s.z)) * kLn2;
    }
  }
  __syncthreads();
  const int col = threadIdx.x / (D / 4), dim = threadIdx.x % (D / 4) * 4, c = c0 + col;
  const int j = c >> a.group_shift;
  if (j >= it->row_count) return;
  const size_t orow = size_t(it->tok0 + j) * a.hq + it->kv_head * a.group + (c & (a.group - 1));
  *reinterpret_cast<u32x2*>(a.o + orow * D + dim) = rows[col][dim / 4];
  if (a.lse && dim == 0) a.lse[orow] = lses[col];
}

template <int D>
static void launch_attention8(Attn8Args x, const pfx_plan* p, hipStream_t s) {
  const int chunks = x.a.plan.num_chunks;
  if (chunks) hipLaunchKernelGGL((extend8_kernel<D, true>), dim3(chunks), dim3(256), 0, s, x);
  else if (p->num_items) hipLaunchKernelGGL((extend8_kernel<D, false>), dim3(p->num_items), dim3(256), 0, s, x);
  if (p->num_segs) hipLaunchKernelGGL(decode8_kernel<D>, dim3(p->num_segs), dim3(256), 0, s, x);
  if (x.a.plan.num_chunk_merges)
    hipLaunchKernelGGL(chunk_merge8_kernel<D>, dim3(x.a.plan.num_chunk_merges * (kExtendTileCols * D / 1024)), dim3(256),
                       0, s, x.a);
  const int n_tok = static_cast<int>(p->merge_tok.size());
  if (n_tok) {
    const size_t units = size_t(n_tok) * p->hq * (D / 4);
    hipLaunchKernelGGL(merge8_kernel<D>, dim3((units + 255) / 256), dim3(256), 0, s, x.a, n_tok);
  }
}

// ---------------------------------------------------------------------------
// Entry points
// ---------------------------------------------------------------------------
static bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

static int check_pool8(const pfx_pool8* pool, const pfx_plan* p, const char* who) {
  if (!pool) return fail(PFX_EINVAL, "%s: pool is NULL", who);
  if (!p) return fail(PFX_EINVAL, "%s: plan is NULL", who);
  if (p->kv_format != PFX_KV_E4M3) return fail(PFX_EINVAL, "%s: the plan is not for an 8-bit pool", who);
  if (pool->page_size != PFX_PAGE_SIZE || pool->num_kv_heads != p->hkv || pool->head_dim != p->d ||
      pool->num_pages != p->num_pages)
    return fail(PFX_EINVAL, "%s: pool shape differs from the one the plan was built for", who);
  if (!pool->k_pages || !pool->v_pages || !pool->scales) return fail(PFX_EINVAL, "%s: pool pointers are NULL", who);
  if (!aligned16(pool->k_pages) || !aligned16(pool->v_pages) || reinterpret_cast<uintptr_t>(pool->scales) % 2)
    return fail(PFX_EINVAL, "%s: pages must be 16-byte aligned, scales 2-byte aligned", who);
  if (!p->dev_ws) return fail(PFX_EINVAL, "%s: plan has not been uploaded", who);
  return PFX_OK;
}

static int check_rows(const char* who, const char* names, const void* a, const void* b) {
  if (!a || !b) return fail(PFX_EINVAL, "%s: %s is NULL", who, names);
  if (!aligned16(a) || !aligned16(b)) return fail(PFX_EINVAL, "%s: %s must be 16-byte aligned", who, names);
  return PFX_OK;
}

static bool attends(const pfx_plan* p) { return p->num_items > 0 || p->num_segs > 0; }

static int launch_append8(const pfx_pool8* pool, const pfx_plan* p, const void* k_new, const void* v_new,
                          hipStream_t s, const char* who) {
  const DevPlan dp = dev_plan(p);
  const size_t units = p->writes.size() * size_t(p->hkv) * 2;
  auto kernel = p->d == 128 ? append8_kernel<128> : append8_kernel<64>;
  hipLaunchKernelGGL(kernel, dim3((units + 3) / 4), dim3(256), 0, s, dp.writes, units,
                     static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new),
                     static_cast<unsigned char*>(pool->k_pages), static_cast<unsigned char*>(pool->v_pages), pool->scales,
                     p->hkv);
  return check_launch(who);
}

static int attention8(const pfx_pool8* pool, const pfx_plan* p, const void* q, void* o, float* lse, float sm_scale,
                      hipStream_t s, const char* who) {
  if (!(sm_scale > 0.f)) sm_scale = 1.0f / sqrtf(float(p->d));
  Attn8Args x{};
  x.a.q = static_cast<const uint16_t*>(q);
  x.a.o = static_cast<uint16_t*>(o);
  x.a.lse = lse;
  x.a.plan = dev_plan(p);
  x.a.hq = p->hq;
  x.a.hkv = p->hkv;
  x.a.group = p->group;
  x.a.group_shift = __builtin_ctz(static_cast<unsigned>(p->group));
  x.a.scale_log2 = sm_scale * kLog2e;
  x.a.merge_parts = p->merge_parts;
  x.k8 = static_cast<const unsigned char*>(pool->k_pages);
  x.v8 = static_cast<const unsigned char*>(pool->v_pages);
  x.scales = pool->scales;
  if (p->d == 128) launch_attention8<128>(x, p, s); else launch_attention8<64>(x, p, s);
  return check_launch(who);
}

}  // namespace pfx

using namespace pfx;

extern "C" int pfx_append_kv8(const pfx_pool8* pool, const pfx_plan* p, const void* k_new, const void* v_new,
                              void* stream) {
  int rc = check_pool8(pool, p, "pfx_append_kv8");
  if (rc || p->num_tokens == 0) return rc;
  if ((rc = check_rows("pfx_append_kv8", "k_new or v_new", k_new, v_new))) return rc;
  return launch_append8(pool, p, k_new, v_new, static_cast<hipStream_t>(stream), "pfx_append_kv8");
}

extern "C" int pfx_attention8(const pfx_pool8* pool, const pfx_plan* p, const void* q, void* o, float* lse,
                              float sm_scale, void* stream) {
  int rc = check_pool8(pool, p, "pfx_attention8");
  if (rc || !attends(p)) return rc;
  if ((rc = check_rows("pfx_attention8", "q or o", q, o))) return rc;
  return attention8(pool, p, q, o, lse, sm_scale, static_cast<hipStream_t>(stream), "pfx_attention8");
}

extern "C" int pfx_step8(const pfx_pool8* pool, const pfx_plan* p, const void* k_new, const void* v_new,
                         const void* q, void* o, float* lse, float sm_scale, void* stream) {
  int rc = check_pool8(pool, p, "pfx_step8");
  if (rc) return rc;
  if (p->num_tokens > 0 && (rc = check_rows("pfx_step8", "k_new or v_new", k_new, v_new))) return rc;
  if (attends(p) && (rc = check_rows("pfx_step8", "q or o", q, o))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->num_tokens > 0 && (rc = launch_append8(pool, p, k_new, v_new, s, "pfx_step8"))) return rc;
  return attends(p) ? attention8(pool, p, q, o, lse, sm_scale, s, "pfx_step8") : PFX_OK;
}

extern "C" size_t pfx_page_quantize_workspace_bytes(int32_t n) {
  return n <= 0 ? 256 : (size_t(n) * 12 + 255) & ~size_t(255);
}

namespace {

// The two sides of a whole-page call, whichever format each has.
struct PageSide {
  int32_t num_pages, page_size, hkv, d;
  const void *k, *v, *scales;  // scales: of an 8-bit side
  bool is8;
};
PageSide side(const pfx_pool* p) {
  return {p->num_pages, p->page_size, p->num_kv_heads, p->head_dim, p->k_pages, p->v_pages, nullptr, false};
}
PageSide side(const pfx_pool8* p) {
  return {p->num_pages, p->page_size, p->num_kv_heads, p->head_dim, p->k_pages, p->v_pages, p->scales, true};
}

// Checks both sides and the lists, then calls launch(list, count) with the list in
// the arguments, or in the workspace.  A long list gets there in the arguments of
// small launches: a copy from the host would wait for the work before it and hold
// up what follows (2396 pages dequantised after their append: 118 us with a copy,
// 107 this way), and a graph that captured it would read the list when it is
// gone.  Nothing escapes as an exception.
template <typename Launch>
int with_pages(const char* who, const PageSide& dst, const PageSide& src, const int32_t* dst_pages,
               const int32_t* src_pages, const int32_t* tokens, int32_t n, void* ws, size_t ws_bytes, hipStream_t s,
               Launch launch) try {
  if (n < 0) return fail(PFX_ERANGE, "%s: n %d < 0", who, n);
  if (n == 0) return PFX_OK;
  if (!dst_pages || !src_pages || !ws) return fail(PFX_EINVAL, "%s: NULL argument", who);
  if (dst.page_size != PFX_PAGE_SIZE || src.page_size != PFX_PAGE_SIZE)
    return fail(PFX_EUNSUPPORTED, "%s: page_size must be %d", who, PFX_PAGE_SIZE);
  if (dst.d != 64 && dst.d != 128) return fail(PFX_EUNSUPPORTED, "%s: head_dim %d (64 or 128 supported)", who, dst.d);
  if (dst.hkv != src.hkv || dst.d != src.d || dst.hkv < 1)
    return fail(PFX_EINVAL, "%s: source and destination page shapes differ", who);
  if (dst.num_pages < 0 || src.num_pages < 0) return fail(PFX_ERANGE, "%s: num_pages < 0", who);
  for (const PageSide* x : {&dst, &src}) {
    if (!x->k || !x->v || (x->is8 && !x->scales)) return fail(PFX_EINVAL, "%s: page pointers are NULL", who);
    if (!aligned16(x->k) || !aligned16(x->v)) return fail(PFX_EINVAL, "%s: pages must be 16-byte aligned", who);
  }
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(PFX_EINVAL, "%s: workspace not 256-byte aligned", who);
  if (ws_bytes < pfx_page_quantize_workspace_bytes(n))
    return fail(PFX_ENOMEM, "%s: workspace has %zu bytes, needs %zu", who, ws_bytes, pfx_page_quantize_workspace_bytes(n));
  std::vector<uint8_t> seen(dst.num_pages, 0);
  for (int32_t i = 0; i < n; ++i) {
    if (dst_pages[i] < 0 || dst_pages[i] >= dst.num_pages)
      return fail(PFX_ERANGE, "%s: dst_pages[%d] = %d outside [0, %d)", who, i, dst_pages[i], dst.num_pages);
    if (src_pages[i] < 0 || src_pages[i] >= src.num_pages)
      return fail(PFX_ERANGE, "%s: src_pages[%d] = %d outside [0, %d)", who, i, src_pages[i], src.num_pages);
    if (seen[dst_pages[i]]) return fail(PFX_EINVAL, "%s: destination page %d repeated", who, dst_pages[i]);
    if (tokens && (tokens[i] < 1 || tokens[i] > PFX_PAGE_SIZE))
      return fail(PFX_ERANGE, "%s: tokens[%d] = %d outside [1, %d]", who, i, tokens[i], PFX_PAGE_SIZE);
    seen[dst_pages[i]] = 1;
  }
  // Within one pool no page may be read and written at once.
  if (dst.is8 == src.is8 && (dst.k == src.k || dst.v == src.v))
    for (int32_t i = 0; i < n; ++i)
      if (src_pages[i] != dst_pages[i] && src_pages[i] < dst.num_pages && seen[src_pages[i]])
        return fail(PFX_EINVAL, "%s: page %d is a source and a destination", who, src_pages[i]);
  // Every array must be device memory or pinned host memory (the kernel would
  // fault on pageable host memory).
  for (const PageSide* x : {&dst, &src})
    for (const void* ptr : {x->k, x->v, x->scales})
      if (ptr && gpu_memory(ptr) == hipMemoryTypeUnregistered)
        return fail(PFX_EINVAL, "%s: a page pointer is neither device nor pinned host memory", who);
  auto run = [&](auto list) {
    using List = decltype(list);
    auto slice = [&](int32_t at) {
      for (int32_t i = 0; i < std::min(n - at, List::kMax); ++i)
        list.set(i, dst_pages[at + i], src_pages[at + i], tokens ? tokens[at + i] : PFX_PAGE_SIZE);
      return list;
    };
    if (n <= List::kMax) return launch(slice(0), n);
    int32_t* staged = static_cast<int32_t*>(ws);
    for (int32_t at = 0; at < n; at += List::kMax)
      hipLaunchKernelGGL(stage_pages_kernel<List>, dim3(1), dim3(List::kMax), 0, s, slice(at), staged + 3 * size_t(at),
                         std::min(n - at, List::kMax));
    launch(PagesAt{staged}, n);
  };
  if (std::max(dst.num_pages, src.num_pages) <= 65536) run(PagesHere16{}); else run(PagesHere32{});
  return check_launch(who);
} catch (...) {
  return fail_exception(who);
}

}  // namespace

extern "C" int pfx_page_quantize(const pfx_pool8* dst, const pfx_pool* src, const int32_t* dst_pages,
                                 const int32_t* src_pages, const int32_t* tokens, int32_t n, void* ws, size_t ws_bytes,
                                 void* stream) {
  if (!dst || !src) return fail(PFX_EINVAL, "pfx_page_quantize: pool descriptor is NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_pages("pfx_page_quantize", side(dst), side(src), dst_pages, src_pages, tokens, n, ws, ws_bytes, s,
                    [&](const auto& list, int32_t cnt) {
    typedef std::decay_t<decltype(list)> List;
    const size_t units = size_t(cnt) * dst->num_kv_heads * 2;
    auto kernel = dst->head_dim == 128 ? page_quantize_kernel<128, List> : page_quantize_kernel<64, List>;
    hipLaunchKernelGGL(kernel, dim3((units + 3) / 4), dim3(256), 0, s, list, units,
                       static_cast<const uint16_t*>(src->k_pages), static_cast<const uint16_t*>(src->v_pages),
                       static_cast<unsigned char*>(dst->k_pages), static_cast<unsigned char*>(dst->v_pages), dst->scales,
                       dst->num_kv_heads);
  });
}

extern "C" int pfx_page_dequantize(const pfx_pool* dst, const pfx_pool8* src, const int32_t* dst_pages,
                                   const int32_t* src_pages, int32_t n, void* ws, size_t ws_bytes, void* stream) {
  if (!dst || !src) return fail(PFX_EINVAL, "pfx_page_dequantize: pool descriptor is NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_pages("pfx_page_dequantize", side(dst), side(src), dst_pages, src_pages, nullptr, n, ws, ws_bytes, s,
                    [&](const auto& list, int32_t cnt) {
    typedef std::decay_t<decltype(list)> List;
    const size_t units = size_t(cnt) * dst->num_kv_heads * 2;
    auto kernel = dst->head_dim == 128 ? page_dequantize_kernel<128, List> : page_dequantize_kernel<64, List>;
    hipLaunchKernelGGL(kernel, dim3((units + 3) / 4), dim3(256), 0, s, list, units,
                       static_cast<const unsigned char*>(src->k_pages), static_cast<const unsigned char*>(src->v_pages),
                       src->scales, static_cast<uint16_t*>(dst->k_pages), static_cast<uint16_t*>(dst->v_pages),
                       dst->num_kv_heads);
  });
}

extern "C" int pfx_page_copy8(const pfx_pool8* dst, const pfx_pool8* src, const int32_t* dst_pages,
                              const int32_t* src_pages, int32_t n, void* ws, size_t ws_bytes, void* stream) {
  if (!dst || !src) return fail(PFX_EINVAL, "pfx_page_copy8: pool descriptor is NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_pages("pfx_page_copy8", side(dst), side(src), dst_pages, src_pages, nullptr, n, ws, ws_bytes, s,
                    [&](const auto& list, int32_t cnt) {
    typedef std::decay_t<decltype(list)> List;
    const size_t units = 2 * size_t(cnt);
    const bool from_host = gpu_memory(src->k_pages) == hipMemoryTypeHost;
    hipLaunchKernelGGL(page_copy8_kernel<List>, dim3(from_host ? std::min<size_t>(units, kLinkWorkgroups8) : units),
                       dim3(256), 0, s, list, units,
                       static_cast<const u32x4*>(src->k_pages), static_cast<const u32x4*>(src->v_pages), src->scales,
                       static_cast<u32x4*>(dst->k_pages), static_cast<u32x4*>(dst->v_pages), dst->scales,
                       dst->num_kv_heads * dst->head_dim, dst->num_kv_heads);
  });
}
