// Per-head RMS norms of queries and keys with the position rotation, one pass.
//
//   x <- x / sqrt(mean(x^2) + eps) * w;  (x_a, x_b) <- the pair turned by
//   position * inv_freq.
// Every value is read once and written once: the pass is bound by HBM (36864
// tokens of 32 + 8 heads, D = 128, 755 MB: 135-139 us, 5.4-5.6 TB/s, over buffers of
// 4.5 GB in turn too; copies of 377 MB in turn reach 5.3, one of 4 GiB 4.95), for few
// tokens by the chain position -> angle -> rotation (one token 3.4 us, 64 4.4; 1999
// with D = 64 6.3-6.9).  D / 16 lanes hold a head,
// 16 values each, as two 16-byte vectors that lie half a rotation apart, so a
// lane owns its pairs.  The workgroup computes each token's rotary_dim / 2
// angles once, in LDS, for all of its heads.
#include "pfx_device.h"

namespace pfx {

struct RopeArgs {
  const uint16_t *q, *k;
  uint16_t *q_out, *k_out;
  const int32_t* pos;
  const double* inv_freq;
  const uint16_t *q_weight, *k_weight;
  int64_t qs[2], ks[2], qos[2], kos[2];  // strides in elements: token, head
  int32_t hq, heads;                     // heads: hq + hkv
  int32_t rotary, interleaved;
  float eps;
};

// Sum over the 4 or 8 consecutive lanes that hold a head.
template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
  auto add = [&](int moved) { x += __builtin_bit_cast(float, moved); };
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
  if constexpr (LANES == 8) add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x141, 0xF, 0xF, true));  // 7 - i
  return x;
}

__device__ __forceinline__ void unpack8(float (&x)[8], const u32x4& w) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 y = unpack_bf16x4(w[2 * i], w[2 * i + 1]);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
  }
}

// Heads whose squares fp32 does not hold, all values below or some above its
// range, are brought to another scale, which the division takes out.  eps goes
// with them.  Called with an eps below kPlainEps only: beside a larger one the
// small squares do not count, and it costs a second chain of exchanges (us at 64
// and 36864 tokens of 32 + 8 heads, D = 128: 3.6 and 135 without, 4.0 and 156).
constexpr float kPlainEps = 0x1p-90f;
template <int LANES>
__device__ __forceinline__ float into_range(float (&x)[8], float (&y)[8], float eps) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(fabsf(x[e]), fabsf(y[e])));
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
  const float s = most >= 0x1p55f ? 0x1p-80f : most < 0x1p-44f ? 0x1p80f : 1.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] *= s;
    y[e] *= s;
  }
  return eps * s * s;
}

// One token a workgroup: few tokens go to as many compute units as there are.
// ANY: see into_range.
template <int D, bool ANY>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeArgs a) {
  constexpr int LANES = D / 16, UNITS = 256 / LANES;
  __shared__ __attribute__((aligned(16))) float cs[2][D / 2];
  const int64_t tok = blockIdx.x;
  if (int(threadIdx.x) < a.rotary / 2) {
    const int f = threadIdx.x;
    // Turns, reduced in fp64: at position 10^6 an fp32 angle would be off by 0.06.
    const double turns = double(a.pos[tok]) * a.inv_freq[f] * 0.15915494309189535;
    float s, c;
    sincospif(float(2.0 * (turns - rint(turns))), &s, &c);
    cs[0][f] = c;
    cs[1][f] = s;
  }
  __syncthreads();
  const int lane = threadIdx.x % LANES;
  // The lane's two vectors of a head, and whether it turns them.
  const int pairs = a.rotary / 16;
  const bool turns = lane < pairs;
  const int va = turns ? lane : 2 * lane, vb = turns ? lane + pairs : 2 * lane + 1;
  for (int hh = threadIdx.x / LANES; hh < a.heads; hh += UNITS) {
    const bool is_k = hh >= a.hq;
    const int h = is_k ? hh - a.hq : hh;
    const int64_t* is = is_k ? a.ks : a.qs;
    const int64_t* os = is_k ? a.kos : a.qos;
    const uint16_t* in = (is_k ? a.k : a.q) + tok * is[0] + h * is[1];
    uint16_t* out = (is_k ? a.k_out : a.q_out) + tok * os[0] + h * os[1];
    const uint16_t* wt = is_k ? a.k_weight : a.q_weight;
    float x[8], y[8];
    unpack8(x, *reinterpret_cast<const u32x4*>(in + 8 * va));
    unpack8(y, *reinterpret_cast<const u32x4*>(in + 8 * vb));
    if (wt) {
      float ss = 0.f, eps = a.eps;
      if constexpr (ANY) eps = into_range<LANES>(x, y, eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += x[e] * x[e] + y[e] * y[e];
      const float r = 1.0f / sqrtf(head_sum<LANES>(ss) * (1.0f / D) + eps);
      float wx[8], wy[8];
      unpack8(wx, *reinterpret_cast<const u32x4*>(wt + 8 * va));
      unpack8(wy, *reinterpret_cast<const u32x4*>(wt + 8 * vb));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= r * wx[e];
        y[e] *= r * wy[e];
      }
    }
    if (turns) {
      if (a.interleaved) {
        const f32x4 ca = *reinterpret_cast<const f32x4*>(&cs[0][4 * va]), sa = *reinterpret_cast<const f32x4*>(&cs[1][4 * va]);
        const f32x4 cb = *reinterpret_cast<const f32x4*>(&cs[0][4 * vb]), sb = *reinterpret_cast<const f32x4*>(&cs[1][4 * vb]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
          x[2 * e] = x0 * ca[e] - x1 * sa[e];
          x[2 * e + 1] = x0 * sa[e] + x1 * ca[e];
          y[2 * e] = y0 * cb[e] - y1 * sb[e];
          y[2 * e + 1] = y0 * sb[e] + y1 * cb[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float c = cs[0][8 * lane + e], s = cs[1][8 * lane + e];
          const float x0 = x[e], y0 = y[e];
          x[e] = x0 * c - y0 * s;
          y[e] = x0 * s + y0 * c;
        }
      }
    }
    *reinterpret_cast<u32x4*>(out + 8 * va) =
        u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    *reinterpret_cast<u32x4*>(out + 8 * vb) =
        u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
  }
}

}  // namespace pfx

using namespace pfx;

// One side's tensors: there if it has heads, aligned, its output rows apart.
static int check_side(const char* name, int32_t heads, int32_t tokens, int32_t d, const void* in, const void* out,
                      const void* weight, const int64_t* is, const int64_t* os) {
  const char* who = "pfx_qk_norm_rope";
  if (heads == 0) return PFX_OK;
  if (!in || !out) return fail(PFX_EINVAL, "%s: %s or %s_out is NULL", who, name, name);
  for (const void* p : {in, out, weight})
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(PFX_EINVAL, "%s: a tensor of %s is not 16-byte aligned", who, name);
  for (int i = 0; i < 2; ++i) {
    if ((i ? heads : tokens) == 1) continue;  // the stride of a single element says nothing
    if (is[i] % 8 || os[i] % 8) return fail(PFX_EINVAL, "%s: strides of %s must be multiples of 8 elements", who, name);
    if (is[i] < 0 || os[i] < 0 || is[i] > (int64_t(1) << 40) || os[i] > (int64_t(1) << 40))
      return fail(PFX_ERANGE, "%s: a stride of %s is out of range", who, name);
  }
  const bool token_major = (heads == 1 || os[1] >= d) && (tokens == 1 || os[0] >= (heads - 1) * os[1] + d);
  const bool head_major = (tokens == 1 || os[0] >= d) && (heads == 1 || os[1] >= (tokens - 1) * os[0] + d);
  if (!token_major && !head_major) return fail(PFX_EINVAL, "%s: rows of %s_out overlap", who, name);
  if (in == out && ((tokens > 1 && is[0] != os[0]) || (heads > 1 && is[1] != os[1])))
    return fail(PFX_EINVAL, "%s: %s_out is %s with other strides", who, name, name);
  return PFX_OK;
}

extern "C" int pfx_qk_norm_rope(const pfx_rope* r, int32_t tokens, const void* q, const void* k,
                                const int32_t* positions, const double* inv_freq, const void* q_weight,
                                const void* k_weight, void* q_out, void* k_out, void* stream) {
  const char* who = "pfx_qk_norm_rope";
  if (!r) return fail(PFX_EINVAL, "%s: rope is NULL", who);
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(PFX_EUNSUPPORTED, "%s: head_dim %d (64 or 128 supported)", who, r->head_dim);
  if (r->num_q_heads < 0 || r->num_kv_heads < 0 || r->num_q_heads > 65536 || r->num_kv_heads > 65536)
    return fail(PFX_ERANGE, "%s: %d query heads, %d KV heads", who, r->num_q_heads, r->num_kv_heads);
  if (r->rotary_dim < 0 || r->rotary_dim > r->head_dim || r->rotary_dim % 16)
    return fail(PFX_EUNSUPPORTED, "%s: rotary_dim %d (multiples of 16 up to head_dim)", who, r->rotary_dim);
  if (r->interleaved != 0 && r->interleaved != 1) return fail(PFX_EINVAL, "%s: interleaved %d", who, r->interleaved);
  if (!(r->eps >= 0.f) || std::isinf(r->eps)) return fail(PFX_EINVAL, "%s: eps is negative or not finite", who);
  if (tokens < 0 || tokens >= (1 << 24)) return fail(PFX_ERANGE, "%s: num_tokens %d", who, tokens);  // a launch: 2^32 threads
  const int32_t heads = r->num_q_heads + r->num_kv_heads;
  if (tokens == 0 || heads == 0) return PFX_OK;
  int rc = check_side("q", r->num_q_heads, tokens, r->head_dim, q, q_out, q_weight, r->q_stride, r->q_out_stride);
  if (!rc) rc = check_side("k", r->num_kv_heads, tokens, r->head_dim, k, k_out, k_weight, r->k_stride, r->k_out_stride);
  if (rc) return rc;
  if (r->rotary_dim > 0 && (!positions || !inv_freq)) return fail(PFX_EINVAL, "%s: positions or inv_freq is NULL", who);
  if (reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(inv_freq) % 8)
    return fail(PFX_EINVAL, "%s: positions or inv_freq is misaligned", who);
  RopeArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_out = static_cast<uint16_t*>(k_out);
  a.pos = positions;
  a.inv_freq = inv_freq;
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  for (int i = 0; i < 2; ++i) {
    const bool one_q = (i ? r->num_q_heads : tokens) == 1, one_k = (i ? r->num_kv_heads : tokens) == 1;
    a.qs[i] = one_q ? 0 : r->q_stride[i];
    a.ks[i] = one_k ? 0 : r->k_stride[i];
    a.qos[i] = one_q ? 0 : r->q_out_stride[i];
    a.kos[i] = one_k ? 0 : r->k_out_stride[i];
  }
  a.hq = r->num_q_heads;
  a.heads = heads;
  a.rotary = r->rotary_dim;
  a.interleaved = r->interleaved;
  a.eps = r->eps;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool any = (q_weight || k_weight) && r->eps < kPlainEps;
  auto kernel = r->head_dim == 128 ? any ? qk_norm_rope_kernel<128, true> : qk_norm_rope_kernel<128, false>
                                   : any ? qk_norm_rope_kernel<64, true> : qk_norm_rope_kernel<64, false>;
  hipLaunchKernelGGL(kernel, dim3(tokens), dim3(256), 0, s, a);
  return check_launch(who);
}
