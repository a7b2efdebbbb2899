// dc_rotate.cu -- norms of queries and keys for each head with the position
// rotation in the same pass (dc_norm_rotate).
//
// For a head's vector x of D dims: y = x / sqrt(mean(x^2) + eps) * w, then the
// pairs of y's first R dims turned by the angles pos * f_j, rounded once.
//
// Each value is read and written once, so a long call is bound by HBM and a short
// one by its launch. A lane holds 8 neighbouring dims (one 16-byte access), 8, 16
// or 32 lanes a head; the mean and, in the half layout, the other dim of a pair
// come from shuffles. A warp takes one token's heads, or a block of them when there
// are few tokens: the token's sines and cosines are computed once for all of them.
//
// Angles: the fraction of a turn that pos * f_j leaves is pos * (f_j / 2 pi) modulo
// 1. f_j / 2 pi is held as a 64-bit fraction (48 good bits), whose product with the
// integer position wraps exactly; the top 32 bits go to sincospif. The error stays below
// 1e-6 rad up to position 2^21, where an angle in 32-bit floating point is off by 0.06.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/distillcache.h"
#include "dc_common.cuh"
#include "dc_device.h"

namespace dc {
namespace {

constexpr int kRotWarps = 4;  // warps of a block

struct Half {
  static __device__ __forceinline__ float2 two(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};

struct Bf16 {
  static __device__ __forceinline__ float2 two(uint32_t u) { return make_float2(bf16lo(u), bf16hi(u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};

// f / 2 pi as a 64-bit fraction of a turn: f times 1 / 2 pi in two 24-bit parts,
// the products' rounding errors kept.
__device__ __forceinline__ unsigned long long turn_fraction(float f) {
  constexpr float hi = 0x1.45f306p-3f, lo = 0x1.b9391p-28f;  // 1 / (2 pi) = hi + lo + 2^-54
  const float p = __fmul_rn(f, hi);
  const float e = __fmaf_rn(f, lo, __fmaf_rn(f, hi, -p));
  const float r = p - floorf(p);  // exact: whole turns do not matter, the position is whole
  return 2ull * ((unsigned long long)(r * 0x1p63f) + (unsigned long long)(long long)(e * 0x1p63f));
}

// One token's heads [h0, h1) of q (heads below Hq) and k.
template <class T, int LPH, bool INTER>
__global__ void __launch_bounds__(kRotWarps * kWarp) rotate_kernel(dc_rotate_args a, long long units, int blocks,
                                                                   int per_block) {
  constexpr int HPI = kWarp / LPH;  // heads of a warp at once
  const int lane = threadIdx.x & 31, c = lane % LPH, hs = lane / LPH;
  const int D = a.head_dim, R = a.rotary_dim, H = a.q_heads + a.kv_heads;
  const bool on = c * 8 < D, turned = c * 8 < R;
  const bool upper = !INTER && c * 16 >= R;  // holds the second dims of the pairs
  const int partner = !INTER && turned ? lane + (upper ? -(R / 16) : R / 16) : lane;
  constexpr int NA = INTER ? 4 : 8;  // this lane's angles
  unsigned long long f[NA];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int j = INTER ? c * 4 + i : (upper ? c * 8 - R / 2 : c * 8) + i;
    f[i] = turned ? turn_fraction(a.inv_freq[j]) : 0;
  }
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    wq[i] = a.norm && a.q_weight && on ? a.q_weight[c * 8 + i] : 1.f;
    wk[i] = a.norm && a.k_weight && on ? a.k_weight[c * 8 + i] : 1.f;
  }
  const float inv_d = 1.f / (float)D;

  for (long long u = (long long)blockIdx.x * kRotWarps + threadIdx.x / kWarp; u < units;
       u += (long long)gridDim.x * kRotWarps) {
    const long long t = u / blocks;
    const int h0 = (int)(u % blocks) * per_block, h1 = min(H, h0 + per_block);
    const int pos = a.positions[t];
    float cs[NA], sn[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int turn = (int)(((unsigned long long)(long long)pos * f[i] + (1ull << 31)) >> 32);  // in 2^-32 turns
      sincospif((float)turn * 0x1p-31f, &sn[i], &cs[i]);
      if (!turned) { cs[i] = 1.f; sn[i] = 0.f; }
      if (upper) sn[i] = -sn[i];
    }
    auto at = [&](const void* p, long long st, long long sh, int h) {
      return reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + t * st + h * sh) + c;
    };
#pragma unroll 4
    for (int hb = h0; hb < h1; hb += HPI) {
      const int h = hb + hs;
      const bool live = on && h < h1, isq = h < a.q_heads;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (live)
        raw = __ldcs(isq ? at(a.q, a.q_token_stride, a.q_head_stride, h)
                         : at(a.k, a.k_token_stride, a.k_head_stride, h - a.q_heads));
      float x[8];
      const uint32_t w4[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = T::two(w4[i]);
        x[2 * i] = v.x;
        x[2 * i + 1] = v.y;
      }
      if (a.norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float r = rsqrtf(fmaf(ss, inv_d, a.eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= r * (isq ? wq[i] : wk[i]);
      }
      uint32_t y[4];
      if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = T::pack(x[2 * i] * cs[i] - x[2 * i + 1] * sn[i], x[2 * i + 1] * cs[i] + x[2 * i] * sn[i]);
      } else {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float other = __shfl_sync(0xffffffffu, x[i], partner);
          z[i] = turned ? x[i] * cs[i] - other * sn[i] : x[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = T::pack(z[2 * i], z[2 * i + 1]);
      }
      if (live)
        *const_cast<uint4*>(isq ? at(a.q_out, a.q_out_token_stride, a.q_out_head_stride, h)
                                : at(a.k_out, a.k_out_token_stride, a.k_out_head_stride, h - a.q_heads)) =
            make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
}

template <class T, int LPH>
cudaError_t launch_rotate(const dc_rotate_args& a, int num_sms, cudaStream_t s) {
  constexpr int HPI = kWarp / LPH;
  const int H = a.q_heads + a.kv_heads;
  // A warp per token where the tokens fill the GPU (16 warps an SM); below that, blocks
  // of heads, down to as many as a warp holds at once.
  const long long want = (long long)num_sms * 16;
  const int rounds = (H + HPI - 1) / HPI;
  long long per = (long long)rounds * a.tokens / want;
  if (per < 1) per = 1;
  if (per > rounds) per = rounds;
  const int blocks = (int)((rounds + per - 1) / per);
  const long long units = a.tokens * blocks;
  const long long grid = std::min<long long>((units + kRotWarps - 1) / kRotWarps, (long long)num_sms * 8);
  if (a.interleaved)
    rotate_kernel<T, LPH, true><<<(unsigned)grid, kRotWarps * kWarp, 0, s>>>(a, units, blocks, (int)per * HPI);
  else
    rotate_kernel<T, LPH, false><<<(unsigned)grid, kRotWarps * kWarp, 0, s>>>(a, units, blocks, (int)per * HPI);
  return cudaGetLastError();
}

thread_local std::string g_rotate_error;

dc_status rotate_fail(dc_status s, const char* msg) {
  g_rotate_error = msg;
  return s;
}

PerDevice<int> g_sms;

int sm_count() {
  return g_sms.get([] {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    return n;
  });
}

}  // namespace
}  // namespace dc

extern "C" const char* dc_rotate_last_error(void) { return dc::g_rotate_error.c_str(); }

extern "C" dc_status dc_norm_rotate(const dc_rotate_args* args, void* stream) {
  using dc::rotate_fail;
  if (!args) return rotate_fail(DC_ERR_INVALID_ARG, "args is NULL");
  const dc_rotate_args& a = *args;
  if (a.tokens < 0 || a.tokens > 0x7FFFFFFFll || a.q_heads < 0 || a.kv_heads < 0 || a.q_heads > 65535 || a.kv_heads > 65535)
    return rotate_fail(DC_ERR_INVALID_ARG, "bad token or head count");
  if (a.head_dim < 16 || a.head_dim > 256 || a.head_dim % 8)
    return rotate_fail(DC_ERR_INVALID_ARG, "head_dim must be a multiple of 8 in [16, 256]");
  if (a.rotary_dim < 16 || a.rotary_dim > a.head_dim || a.rotary_dim % 16)
    return rotate_fail(DC_ERR_INVALID_ARG, "rotary_dim must be a multiple of 16 in [16, head_dim]");
  if (a.dtype != DC_BF16 && a.dtype != DC_FP16) return rotate_fail(DC_ERR_INVALID_ARG, "dtype must be DC_BF16 or DC_FP16");
  if (a.norm && !(a.eps >= 0.f)) return rotate_fail(DC_ERR_INVALID_ARG, "eps must be >= 0");
  if (a.tokens == 0 || a.q_heads + a.kv_heads == 0) return DC_OK;
  if (!a.positions || !a.inv_freq || (a.q_heads && (!a.q || !a.q_out)) || (a.kv_heads && (!a.k || !a.k_out)))
    return rotate_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  const uintptr_t at = (a.q_heads ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0) | (a.kv_heads ? (uintptr_t)a.k | (uintptr_t)a.k_out : 0);
  const long long st = (a.q_heads ? a.q_token_stride | a.q_head_stride | a.q_out_token_stride | a.q_out_head_stride : 0) |
                       (a.kv_heads ? a.k_token_stride | a.k_head_stride | a.k_out_token_stride | a.k_out_head_stride : 0);
  if ((at & 15) || (st & 7))
    return rotate_fail(DC_ERR_INVALID_ARG, "q, k and their outputs must start every head on 16 bytes (strides multiples of 8)");
  const int sms = dc::sm_count();
  if (sms < 1) return rotate_fail(DC_ERR_CUDA, "no CUDA device");
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
#define DC_ROTATE(LPH) e = a.dtype == DC_BF16 ? dc::launch_rotate<dc::Bf16, LPH>(a, sms, s) : dc::launch_rotate<dc::Half, LPH>(a, sms, s)
  if (a.head_dim <= 64) DC_ROTATE(8);
  else if (a.head_dim <= 128) DC_ROTATE(16);
  else DC_ROTATE(32);
#undef DC_ROTATE
  if (e != cudaSuccess) {
    dc::g_rotate_error = std::string("launch: ") + cudaGetErrorString(e);
    return DC_ERR_CUDA;
  }
  return DC_OK;
}
