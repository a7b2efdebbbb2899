// dc_rotate.cu -- norms of queries and keys for each head with the position
// rotation in the same pass (dc_norm_rotate).
//
// For a head's vector x of D dims: y = x / sqrt(mean(x^2) + eps) * w, then the
// pairs of y's first R dims turned by the angles pos * f_j, rounded once.
//
// Each value is read and written once, so a long call is bound by HBM (32768 tokens of 40
// heads of 128 dims: 99 us, 6.77 TB/s, a copy's rate) and a short one by its launch (8 such
// tokens: 2.5 us on the device). A lane holds both dims of eight pairs (two 16-byte accesses),
// so a pair needs no exchange; 4, 8 or 16 lanes hold a head, whose mean takes 2 to 4 shuffles. A
// warp takes one token's heads, or a block of them when there are few tokens: the lanes that hold
// the same dims of different heads compute a share of the token's sines and cosines each and pass
// them on. What it took from 270 us: pairs within a lane (130), gains, sines and cosines folded
// into four factors a pair, loads that run ahead through shared memory across tokens without
// holding registers (114), and far more blocks than fit at once, so that SMs that finish early
// take more (99; 5 blocks an SM, all resident, 114).
//
// Angles: the fraction of a turn that pos * f_j leaves is pos * (f_j / 2 pi) modulo
// 1. f_j / 2 pi is held as a 64-bit fraction (about 50 good bits), whose product with the
// integer position wraps exactly; the top 32 bits go to sincospif. The angle is off by at most
// 1e-7 + 5e-15 |pos * f_j| rad (5e-7 at position 2^21 and f_j 100; an angle of 2^21 in 32-bit floating
// point is off by 0.06), for f_j of either sign below 2^26.
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

constexpr int kRotWarps = 4;   // warps of a block
constexpr int kRotBlocks = 40; // blocks for an SM, at most

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

// f / 2 pi as a 64-bit fraction of a turn, of either sign: f times 1 / 2 pi in two 24-bit parts,
// the products' rounding errors kept.
__device__ __forceinline__ unsigned long long turn_fraction(float f) {
  constexpr float hi = 0x1.45f306p-3f, lo = 0x1.b9391p-28f;  // 1 / (2 pi) = hi + lo + 2^-54
  const float p = __fmul_rn(f, hi);
  const float e = __fmaf_rn(f, lo, __fmaf_rn(f, hi, -p));
  const float r = p - truncf(p);  // exact (p - floor(p) is not, below 0): whole turns do not matter, the position is whole
  return 2ull * (unsigned long long)((long long)(r * 0x1p63f) + (long long)(e * 0x1p63f));
}

// Two 32-bit values in one 64-bit register, for the paired arithmetic of sm_100.
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 f2_out(F2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// 16 bytes from global to shared memory behind the thread's back; zeros if !on.
__device__ __forceinline__ void copy_async(uint4* dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(on ? 16 : 0)
               : "memory");
}

// A token's heads go in rounds of HPI: q's, then k's. A unit of work is `per` of its rounds,
// and there are `blocks` units a token.
template <class T, int LPH, bool INTER, bool NORM>
__global__ void __launch_bounds__(kRotWarps * kWarp) rotate_kernel(const dc_rotate_args a, int blocks, int per) {
  constexpr int HPI = kWarp / LPH;  // heads of a warp at once
  constexpr int OWN = 8 / HPI;      // of its eight pairs' angles, those that a lane computes itself
  // Rounds on their way to a lane's own places in shared memory, whatever units they belong to.
  constexpr int P = 6;
  __shared__ uint4 ring[kRotWarps][P][2][kWarp];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / kWarp, c = lane % LPH, hs = lane / LPH;
  const int D = a.head_dim, R = a.rotary_dim;
  const int rq = (a.q_heads + HPI - 1) / HPI, rounds = rq + (a.kv_heads + HPI - 1) / HPI;
  // This lane's two chunks of 8 dims. Half layout: pair i is dim i of each; behind the rotated
  // dims, and interleaved, the chunks are neighbours.
  const bool turned = c * 16 < R;
  const int c0 = !INTER && turned ? c : 2 * c, c1 = !INTER && turned ? c + R / 16 : 2 * c + 1;
  const bool on0 = c0 * 8 < D, on1 = c1 * 8 < D;
  // this warp's units: token and part of it, and the steps from one to the next
  const int steps = (int)gridDim.x * kRotWarps, w0 = (int)blockIdx.x * kRotWarps + warp;
  const int dt = steps / blocks, db = steps % blocks, t0 = w0 / blocks, b0 = w0 % blocks, tokens = (int)a.tokens;

  // the next round to fetch
  int ft = t0, fb = b0, fr = b0 * per, fend = min(rounds, fr + per), fh = 0, fheads = 0, fslot = 0;
  const uint16_t* fp = nullptr;
  long long fstep = 0;
  auto seek = [&] {  // to round fr of token ft
    const bool kv = fr >= rq;
    const long long sh = kv ? a.k_head_stride : a.q_head_stride;
    fh = (kv ? fr - rq : fr) * HPI + hs;
    fheads = kv ? a.kv_heads : a.q_heads;
    fp = static_cast<const uint16_t*>(kv ? a.k : a.q) + ft * (kv ? a.k_token_stride : a.q_token_stride) + fh * sh;
    fstep = HPI * sh;
  };
  auto fetch = [&] {
    if (ft < tokens) {
      const bool live = fh < fheads;
      copy_async(&ring[warp][fslot][0][lane], fp + c0 * 8, live && on0);
      copy_async(&ring[warp][fslot][1][lane], fp + c1 * 8, live && on1);
      fp += fstep;
      fh += HPI;
      if (++fr == fend) {
        ft += dt;
        fb += db;
        if (fb >= blocks) fb -= blocks, ++ft;
        fr = fb * per;
        fend = min(rounds, fr + per);
        seek();
      } else if (fr == rq) {
        seek();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    fslot = fslot == P - 1 ? 0 : fslot + 1;
  };
  seek();
#pragma unroll 1
  for (int i = 0; i < P - 1; ++i) fetch();

  unsigned long long f[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) f[i] = turned ? turn_fraction(a.inv_freq[c * 8 + hs * OWN + i]) : 0;
  const float inv_d = 1.f / (float)D;
  int slot = 0;

  int pos = t0 < tokens ? __ldg(a.positions + t0) : 0;
  int t = t0, b = b0;
#pragma unroll 1
  while (t < tokens) {
    const int r0 = b * per, r1 = min(rounds, r0 + per), tt = t;
    t += dt;
    b += db;
    if (b >= blocks) b -= blocks, ++t;
    float co[8], so[8];  // of this lane's pairs
    {
      float x[OWN], y[OWN];
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const int turn = (int)(((unsigned long long)(long long)pos * f[i] + (1ull << 31)) >> 32);  // in 2^-32 turns
        sincospif((float)turn * 0x1p-31f, &y[i], &x[i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        co[i] = __shfl_sync(0xffffffffu, x[i % OWN], i / OWN * LPH + c);
        so[i] = __shfl_sync(0xffffffffu, y[i % OWN], i / OWN * LPH + c);
      }
    }
    if (t < tokens) pos = __ldg(a.positions + t);
#pragma unroll 1
    for (int kv = r0 < rq ? 0 : 1; kv < 2; ++kv) {
      const int from = kv ? max(r0, rq) : r0, to = kv ? r1 : min(r1, rq);
      if (from >= to) continue;
      const int heads = kv ? a.kv_heads : a.q_heads;
      int h = (kv ? from - rq : from) * HPI + hs;
      const long long oh = kv ? a.k_out_head_stride : a.q_out_head_stride;
      uint16_t* dst = static_cast<uint16_t*>(kv ? a.k_out : a.q_out) +
                      tt * (kv ? a.k_out_token_stride : a.q_out_token_stride) + h * oh;
      const float* w = kv ? a.k_weight : a.q_weight;
      // pair (x, y) with gains (g, z): x' = x g cos - y z sin, y' = y z cos + x g sin
      F2 xx[4], xy[4], yy[4], yx[4];
      {
        float g[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          g[i] = NORM && w && on0 ? __ldg(w + c0 * 8 + i) : 1.f;
          g[8 + i] = NORM && w && on1 ? __ldg(w + c1 * 8 + i) : 1.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const F2 wa = INTER ? f2(g[4 * i], g[4 * i + 2]) : f2(g[2 * i], g[2 * i + 1]);
          const F2 wb = INTER ? f2(g[4 * i + 1], g[4 * i + 3]) : f2(g[8 + 2 * i], g[9 + 2 * i]);
          const F2 cs = f2(co[2 * i], co[2 * i + 1]);
          xx[i] = wa * cs;
          yy[i] = wb * cs;
          yx[i] = wa * f2(so[2 * i], so[2 * i + 1]);
          xy[i] = wb * f2(-so[2 * i], -so[2 * i + 1]);
        }
      }
#pragma unroll 1
      for (int r = from; r < to; ++r, h += HPI, dst += HPI * oh) {
        fetch();
        asm volatile("cp.async.wait_group %0;" ::"n"(P - 1) : "memory");
        const uint4 x = ring[warp][slot][0][lane], y = ring[warp][slot][1][lane];
        slot = slot == P - 1 ? 0 : slot + 1;
        const uint32_t wx[4] = {x.x, x.y, x.z, x.w}, wy[4] = {y.x, y.y, y.z, y.w};
        F2 p[4], q[4];  // first and second dims of pairs 2i, 2i + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (INTER) {
            const float2 v = T::two(i < 2 ? wx[2 * i] : wy[2 * i - 4]), z = T::two(i < 2 ? wx[2 * i + 1] : wy[2 * i - 3]);
            p[i] = f2(v.x, z.x);
            q[i] = f2(v.y, z.y);
          } else {
            const float2 v = T::two(wx[i]), z = T::two(wy[i]);
            p[i] = f2(v.x, v.y);
            q[i] = f2(z.x, z.y);
          }
        }
        F2 r2;
        if constexpr (NORM) {
          F2 ss = p[0] * p[0], st = q[0] * q[0];
#pragma unroll
          for (int i = 1; i < 4; ++i) {
            ss = fma2(p[i], p[i], ss);
            st = fma2(q[i], q[i], st);
          }
          const float2 e = f2_out(ss), o = f2_out(st);
          float sum = (e.x + e.y) + (o.x + o.y);
#pragma unroll
          for (int o2 = LPH / 2; o2 > 0; o2 >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o2);
          const float rs = rsqrtf(fmaf(sum, inv_d, a.eps));
          r2 = f2(rs, rs);
        }
        uint32_t ox[4], oy[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          F2 sm = q[i] * xy[i], sn = p[i] * yx[i];
          // (0 times a value that is not finite must not reach a dim that is not rotated)
          if (R < D && !turned) sm = sn = f2(0.f, 0.f);
          F2 m = fma2(p[i], xx[i], sm), n = fma2(q[i], yy[i], sn);
          if constexpr (NORM) {
            m = m * r2;
            n = n * r2;
          }
          const float2 mv = f2_out(m), nv = f2_out(n);
          if constexpr (INTER) {
            (i < 2 ? ox[2 * i] : oy[2 * i - 4]) = T::pack(mv.x, nv.x);
            (i < 2 ? ox[2 * i + 1] : oy[2 * i - 3]) = T::pack(mv.y, nv.y);
          } else {
            ox[i] = T::pack(mv.x, mv.y);
            oy[i] = T::pack(nv.x, nv.y);
          }
        }
        if (h < heads) {
          if (on0) reinterpret_cast<uint4*>(dst)[c0] = make_uint4(ox[0], ox[1], ox[2], ox[3]);
          if (on1) reinterpret_cast<uint4*>(dst)[c1] = make_uint4(oy[0], oy[1], oy[2], oy[3]);
        }
      }
    }
  }
}

template <class T, int LPH>
cudaError_t launch_rotate(const dc_rotate_args& a, int num_sms, cudaStream_t s) {
  constexpr int HPI = kWarp / LPH;
  const int rounds = (a.q_heads + HPI - 1) / HPI + (a.kv_heads + HPI - 1) / HPI;
  // A warp takes a token's heads at once where that fills the GPU (16 warps an SM); below
  // that, as many rounds as leave every SM its share, down to one.
  const long long want = (long long)num_sms * 16;
  long long per = (long long)rounds * a.tokens / want;
  per = per < 1 ? 1 : per > rounds ? rounds : per;
  const int blocks = (int)((rounds + per - 1) / per);
  const long long units = a.tokens * blocks;
  const long long grid = std::min<long long>((units + kRotWarps - 1) / kRotWarps, (long long)num_sms * kRotBlocks);
  auto run = [&](auto* kernel) { kernel<<<(unsigned)grid, kRotWarps * kWarp, 0, s>>>(a, blocks, (int)per); };
  if (a.interleaved) a.norm ? run(rotate_kernel<T, LPH, true, true>) : run(rotate_kernel<T, LPH, true, false>);
  else a.norm ? run(rotate_kernel<T, LPH, false, true>) : run(rotate_kernel<T, LPH, false, false>);
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
  if (a.tokens < 0 || a.tokens > (1ll << 30) || a.q_heads < 0 || a.kv_heads < 0 || a.q_heads > 65535 || a.kv_heads > 65535)
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
  if (((uintptr_t)a.positions | (uintptr_t)a.inv_freq | (uintptr_t)a.q_weight | (uintptr_t)a.k_weight) & 3)
    return rotate_fail(DC_ERR_INVALID_ARG, "positions, inv_freq and weights must be 4-byte aligned");
  const int sms = dc::sm_count();
  if (sms < 1) return rotate_fail(DC_ERR_CUDA, "no CUDA device");
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
#define DC_ROTATE(LPH) e = a.dtype == DC_BF16 ? dc::launch_rotate<dc::Bf16, LPH>(a, sms, s) : dc::launch_rotate<dc::Half, LPH>(a, sms, s)
  if (a.head_dim <= 64) DC_ROTATE(4);
  else if (a.head_dim <= 128) DC_ROTATE(8);
  else DC_ROTATE(16);
#undef DC_ROTATE
  if (e != cudaSuccess) {
    dc::g_rotate_error = std::string("launch: ") + cudaGetErrorString(e);
    return DC_ERR_CUDA;
  }
  return DC_OK;
}
