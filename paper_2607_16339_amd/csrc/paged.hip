// Paged key/value cache: rotation and append of new tokens, and their
// attention over the cache.
#include "device.h"
#include "launch.h"

namespace lacache {
namespace {

// Rotation and append. A group of D/8 lanes holds one head's vector of one
// token, 8 dims per lane; lane c of the rotated part meets its partner (c +- r/16)
// by loading that chunk as well (its line is in the cache already).
template <int D, bool kFp8>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppend a) {
  constexpr int L = D / 8, G = 256 / L;
  const int c = threadIdx.x % L;
  const int64_t t = blockIdx.x;
  const int seq = a.seq_ids[t], pos = a.positions[t];
  if (seq < 0 || seq >= a.S || pos < 0 || pos >= a.max_pos) return;
  const int page = a.table[static_cast<int64_t>(seq) * a.max_pages + (pos >> a.page_log2)];
  if (page < 0 || page >= a.num_pages) return;
  const int slot = pos & ((1 << a.page_log2) - 1);
  const int hc = a.rope_dim >> 4;  // chunks of half the rotated part
  const bool rot = c < 2 * hc, low = c < hc;
  float cs[8], sn[8];
  if (rot) {
    const int64_t o = static_cast<int64_t>(pos) * (8 * hc) + 8 * (low ? c : c - hc);
    const v4f* pc = reinterpret_cast<const v4f*>(a.cs + o);
    const v4f* ps = reinterpret_cast<const v4f*>(a.sn + o);
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = pc[e >> 2][e & 3], sn[e] = ps[e >> 2][e & 3];
  }
  const int HT = a.heads + 2 * a.kv_heads;
  const uint4* src = reinterpret_cast<const uint4*>(a.qkv + t * HT * D);
  for (int hs = blockIdx.y * G + threadIdx.x / L; hs < HT; hs += gridDim.y * G) {
    const uint4 x = src[hs * L + c];
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[2 * e] = bf16lo(xw[e]), y[2 * e + 1] = bf16hi(xw[e]);
    const bool turn = rot && hs < a.heads + a.kv_heads;
    if (turn) {
      const uint4 p = src[hs * L + (low ? c + hc : c - hc)];
      const uint32_t pw[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float o = e & 1 ? bf16hi(pw[e >> 1]) : bf16lo(pw[e >> 1]);
        const float u = y[e] * cs[e], w = o * sn[e];
        y[e] = low ? u - w : u + w;
      }
    }
    const bool to_cache = hs >= a.heads;
    const bool is_v = hs >= a.heads + a.kv_heads;
    const int h = is_v ? hs - a.heads - a.kv_heads : hs - a.heads;
    const int64_t row = ((static_cast<int64_t>(page) * a.kv_heads + h) << a.page_log2) + slot;
    if (kFp8 && to_cache) {
      // the largest magnitude by its bits, so that infinities and NaNs win
      uint32_t top = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7FFFFFFFu);
#pragma unroll
      for (int o = L / 2; o >= 1; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, 64)));
      const float s = __uint_as_float(top) / kE4M3Max;
      uint32_t lo = 0x7F7F7F7Fu, hi = 0x7F7F7F7Fu;  // a vector that is not finite reads as NaN
      if (top < 0x7F800000u) quant8(y, s, lo, hi);
      reinterpret_cast<uint2*>(is_v ? a.v_cache : a.k_cache)[row * L + c] = make_uint2(lo, hi);
      if (c == 0) (is_v ? a.v_scale : a.k_scale)[row] = s;
      continue;
    }
    const uint4 o = turn ? make_uint4(cvt_pk_bf16(y[0], y[1]), cvt_pk_bf16(y[2], y[3]), cvt_pk_bf16(y[4], y[5]),
                                      cvt_pk_bf16(y[6], y[7]))
                         : x;
    if (to_cache)
      reinterpret_cast<uint4*>(is_v ? a.v_cache : a.k_cache)[row * L + c] = o;
    else
      reinterpret_cast<uint4*>(a.q)[(t * a.heads + hs) * L + c] = o;
  }
}

// The value of an e4m3 code.
__device__ __forceinline__ float e4m3_value(uint32_t code) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(code), 0);
}

// Attention, plainly: a wavefront per query row; lane j takes key j of 64 for
// the scores and dims j, j + 64 of the values.
template <int D, bool kFp8>
__global__ __launch_bounds__(64) void paged_attention_simple_kernel(PagedAttn a) {
  __shared__ float sp[64];
  __shared__ float sq[D];
  const int lane = threadIdx.x;
  const int h = blockIdx.x % a.heads, t = (blockIdx.x / a.heads) % a.nq;
  const int64_t s = blockIdx.x / (a.heads * a.nq), row = blockIdx.x;
  const int kvh = h / (a.heads / a.kv_heads);
  int len = a.seq_lens[s];
  len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
  const int end = a.causal ? len - a.nq + t + 1 : len;
  for (int i = lane; i < D; i += 64) sq[i] = bf16lo(a.q[row * D + i]);
  __syncthreads();
  float m = -__builtin_inff(), l = 0.0f, o[D / 64] = {};
  for (int k0 = 0; k0 < end; k0 += 64) {
    const int key = k0 + lane;
    float x = -__builtin_inff();
    int64_t kr = -1;
    if (key < end) {
      const int page = a.table[s * a.max_pages + (key >> a.page_log2)];
      if (page >= 0 && page < a.num_pages) {
        kr = ((static_cast<int64_t>(page) * a.kv_heads + kvh) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
        float dot = 0.0f;
        for (int i = 0; i < D; ++i) {
          const float kvv = kFp8 ? e4m3_value(static_cast<const uint8_t*>(a.k_cache)[kr * D + i])
                                 : bf16lo(static_cast<const uint16_t*>(a.k_cache)[kr * D + i]);
          dot += sq[i] * kvv;
        }
        if (kFp8) dot *= a.k_scale[kr];
        x = dot * a.scale_log2;
      }
    }
    const float mn = __builtin_fmaxf(m, max_xor<64>(x));
    const float ms = mn == -__builtin_inff() ? 0.0f : mn;
    const float alpha = __builtin_amdgcn_exp2f(m - ms), p = __builtin_amdgcn_exp2f(x - ms);
    m = mn;
    l = l * alpha + p;
    for (int e = 0; e < D / 64; ++e) o[e] *= alpha;
    __syncthreads();
    sp[lane] = kFp8 && kr >= 0 ? p * a.v_scale[kr] : p;
    __syncthreads();
    for (int j = 0; j < 64; ++j) {
      const int64_t r = __shfl(kr, j, 64);
      if (r < 0) continue;
      for (int e = 0; e < D / 64; ++e) {
        const int64_t i = r * D + 64 * e + lane;
        const float vv = kFp8 ? e4m3_value(static_cast<const uint8_t*>(a.v_cache)[i])
                              : bf16lo(static_cast<const uint16_t*>(a.v_cache)[i]);
        o[e] += sp[j] * vv;
      }
    }
  }
  for (int x = 32; x >= 1; x >>= 1) l += __shfl_xor(l, x, 64);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  for (int e = 0; e < D / 64; ++e) a.o[row * D + 64 * e + lane] = static_cast<uint16_t>(f32_to_bf16(o[e] * inv));
  if (a.lse != nullptr && lane == 0) a.lse[row] = (m + __log2f(l)) * 0.69314718055994531f;
}

}  // namespace

hipError_t launch_paged_append(hipStream_t st, const PagedAppend& a, int64_t T, int64_t d, bool fp8) {
  const int G = static_cast<int>(256 / (d / 8));
  const int HT = a.heads + 2 * a.kv_heads;
  const int per = (HT + G - 1) / G;
  const int64_t cus = device_cu_count();
  // few tokens: every head of a token at once
  const int64_t ny = T * per <= 8 * cus ? per : 1;
  const dim3 grid(static_cast<unsigned>(T), static_cast<unsigned>(ny)), block(256);
  if (d == 128 && fp8) hipLaunchKernelGGL((paged_append_kernel<128, true>), grid, block, 0, st, a);
  else if (d == 128) hipLaunchKernelGGL((paged_append_kernel<128, false>), grid, block, 0, st, a);
  else if (fp8) hipLaunchKernelGGL((paged_append_kernel<64, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_append_kernel<64, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

size_t paged_attention_ws_bytes(int64_t S, int64_t nq, int64_t heads, int64_t kv_heads, int64_t d) {
  (void)S, (void)nq, (void)heads, (void)kv_heads, (void)d;
  return 256;
}

hipError_t launch_paged_attention(hipStream_t st, const PagedAttn& a, int64_t d, bool fp8, void* ws) {
  (void)ws;
  const dim3 grid(static_cast<unsigned>(a.S) * a.nq * a.heads), block(64);
  if (d == 128 && fp8) hipLaunchKernelGGL((paged_attention_simple_kernel<128, true>), grid, block, 0, st, a);
  else if (d == 128) hipLaunchKernelGGL((paged_attention_simple_kernel<128, false>), grid, block, 0, st, a);
  else if (fp8) hipLaunchKernelGGL((paged_attention_simple_kernel<64, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_attention_simple_kernel<64, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace lacache
