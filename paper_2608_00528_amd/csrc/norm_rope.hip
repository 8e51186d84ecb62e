// Norms of the query and key heads with the position rotation, in one pass:
//
//   y = x / sqrt(mean(x^2) + eps) * w   (per head; without a weight y = x)
//   (y_i, y_{i + d_h/2}) turned by pos * theta^(-2 i / d_h)
//
// Reads and writes each element once: bound by HBM for a prompt, by one launch's
// latency for a few tokens.  A lane holds dims 4 p .. + 3 and their partners
// d_h / 2 above them, so the rotation stays in the lane and d_h / 8 lanes hold a
// head; a wave takes 512 / d_h heads at a time, the next ones on their way, and keeps
// the turns of its token over all its heads.  Sums of squares are fp32, and fp64 for
// heads where those would leave its range.
#include "s4r_device.h"
#include "s4r_internal.h"

namespace s4r {
namespace {

// four consecutive elements as stored, and as fp32
template <typename T>
struct Four;
template <>
struct Four<uint16_t> {
  typedef uint32_t raw __attribute__((ext_vector_type(2)));
  __device__ __forceinline__ static void get(raw u, float* x) {
    x[0] = __uint_as_float(u[0] << 16);
    x[1] = __uint_as_float(u[0] & 0xFFFF0000u);
    x[2] = __uint_as_float(u[1] << 16);
    x[3] = __uint_as_float(u[1] & 0xFFFF0000u);
  }
};
template <>
struct Four<float> {
  typedef floatx4 raw;
  __device__ __forceinline__ static void get(raw u, float* x) { x[0] = u[0], x[1] = u[1], x[2] = u[2], x[3] = u[3]; }
};
template <typename T>
__device__ __forceinline__ void load4(const T* p, float* x) {
  Four<T>::get(*reinterpret_cast<const typename Four<T>::raw*>(p), x);
}
__device__ __forceinline__ void store4(uint16_t* p, const float* x) {
  typename Four<uint16_t>::raw u = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  __builtin_nontemporal_store(u, reinterpret_cast<typename Four<uint16_t>::raw*>(p));
}
__device__ __forceinline__ void store4(float* p, const float* x) {
  __builtin_nontemporal_store(floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<floatx4*>(p));
}

// sum over the d_h / 8 lanes of a head (every one of them gets it)
template <int DH>
__device__ __forceinline__ float head_sum(float x) {
  x += dpp_f<0xB1>(x);                  // quad_perm [1,0,3,2]
  x += dpp_f<0x4E>(x);                  // quad_perm [2,3,0,1]
  x += dpp_f<0x141>(x);                 // row_half_mirror: the other quad of eight lanes
  if (DH == 128) x += dpp_f<0x128>(x);  // row_ror:8
  return x;
}
template <int DH>
__device__ __forceinline__ double head_sum(double x) {
  x += dpp_d<0xB1>(x);                  // quad_perm [1,0,3,2]
  x += dpp_d<0x4E>(x);                  // quad_perm [2,3,0,1]
  x += dpp_d<0x141>(x);                 // row_half_mirror: the other quad of eight lanes
  if (DH == 128) x += dpp_d<0x128>(x);  // row_ror:8
  return x;
}

// a head's elements times 1 / sqrt(mean(x^2) + eps), where fp32 sums leave the range
template <int DH>
__device__ __forceinline__ void norm_far(float (&x)[8], double eps) {
  double ss = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss = fma((double)x[e], (double)x[e], ss);
  const double ms = head_sum<DH>(ss) * (1.0 / DH) + eps;
  double r = __builtin_amdgcn_rsq(ms);                 // the hardware's estimate and two Newton steps
  if (ms > 0.0 && ms < INFINITY) {
    r *= 1.5 - 0.5 * ms * r * r;
    r *= 1.5 - 0.5 * ms * r * r;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)((double)x[e] * r);
}

// cos and sin of pos * F revolutions; F a 0.64 fixed-point number, so the fraction
// of a revolution is exact in 64-bit integer arithmetic for any position.  bf16 rows take
// the hardware's functions of its upper 24 bits (off by up to 2^-22, next to a bf16
// step of 2^-8).  fp32 rows would lose by it what they hold: they take the fraction from the
// nearest quarter, its first 24 bits wherever they begin, and the functions' series, which on
// [-pi / 4, pi / 4] end below 2^-28.
template <typename T>
__device__ __forceinline__ void turn(int32_t pos, uint64_t F, float& c, float& s);
template <>
__device__ __forceinline__ void turn<uint16_t>(int32_t pos, uint64_t F, float& c, float& s) {
  const uint64_t phase = (uint64_t)(int64_t)pos * F;
  const float x = (float)(int32_t)(phase >> 32) * 2.3283064365386963e-10f;   // revolutions in [-1/2, 1/2)
  c = __builtin_amdgcn_cosf(x);
  s = __builtin_amdgcn_sinf(x);
}
template <>
__device__ __forceinline__ void turn<float>(int32_t pos, uint64_t F, float& c, float& s) {
  constexpr double A = 6.283185307179586, B = A * A;   // the series in revolutions: powers of 2 pi over factorials
  constexpr float A1 = (float)A, A0 = (float)(A - (double)A1);
  constexpr float s3 = (float)(-A * B / 6), s5 = (float)(A * B * B / 120), s7 = (float)(-A * B * B * B / 5040),
                  s9 = (float)(A * B * B * B * B / 362880);
  constexpr float c2 = (float)(-B / 2), c4 = (float)(B * B / 24), c6 = (float)(-B * B * B / 720),
                  c8 = (float)(B * B * B * B / 40320), c10 = (float)(-B * B * B * B * B / 3628800);
  const uint64_t phase = (uint64_t)(int64_t)pos * F, near = phase + (1ull << 61);
  const uint32_t quarter = (uint32_t)(near >> 62);
  const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));          // in [-2^61, 2^61)
  const uint64_t size = rest < 0 ? -rest : rest;
  const float r = fmaf((float)(uint32_t)size, 0x1p-64f, (float)(uint32_t)(size >> 32) * 0x1p-32f);
  const float x = rest < 0 ? -r : r, z = x * x;
  const float sx = fmaf(x, A1, x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, s9, s7), s5), s3), A0));
  const float cx = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, c10, c8), c6), c4), c2), 1.f);
  const float u = quarter & 1 ? sx : cx, v = quarter & 1 ? cx : sx;
  c = (quarter + 1) & 2 ? -u : u;
  s = quarter & 2 ? -v : v;
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_qk_norm_rope(const T* q, int64_t q_stride, const T* k, int64_t k_stride,
                                                      const T* __restrict__ q_weight,
                                                      const T* __restrict__ k_weight, float eps,
                                                      const int32_t* __restrict__ positions, T* q_out,
                                                      int64_t q_out_stride, T* k_out, int64_t k_out_stride,
                                                      int64_t n_tokens, int hq, int heads, int per, double ratio) {
  constexpr int LPH = DH / 8, HPW = 64 / LPH;         // lanes per head, heads a wave takes at a time
  const int lane = threadIdx.x & 63, p = lane % LPH, hl = lane / LPH;
  const int d0 = 4 * p, d1 = d0 + DH / 2;
  // this lane's frequencies as revolutions per position
  uint64_t F[4] = {0, 0, 0, 0};
  if (ratio != 0.0) {
    double f = 1.0, base = ratio;
    for (int e = d0; e > 0; e >>= 1) {
      if (e & 1) f *= base;
      base *= base;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const double rev = f * 0.15915494309189535;
      F[v] = (uint64_t)((rev - floor(rev)) * 18446744073709551616.0);
      f *= ratio;
    }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (q_weight) load4(q_weight + d0, wq), load4(q_weight + d1, wq + 4);
  if (k_weight) load4(k_weight + d0, wk), load4(k_weight + d1, wk + 4);

  // a unit: `per` groups of HPW heads of one token
  const int groups = (heads + HPW - 1) / HPW, parts = (groups + per - 1) / per;
  const int64_t units = n_tokens * parts;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), waves = (int64_t)gridDim.x * 4;
  typename Four<T>::raw r0, r1;                        // the group that comes next
  auto fetch = [&](int64_t tok, int g) __attribute__((always_inline)) {
    const int h = min(g * HPW + hl, heads - 1);
    const T* src = h < hq ? q + tok * q_stride + (int64_t)h * DH : k + tok * k_stride + (int64_t)(h - hq) * DH;
    r0 = *reinterpret_cast<const typename Four<T>::raw*>(src + d0);
    r1 = *reinterpret_cast<const typename Four<T>::raw*>(src + d1);
  };
  for (int64_t u = wave; u < units; u += waves) {
    const int64_t tok = u / parts;
    int g = (int)(u - tok * parts) * per;
    const int g1 = min(g + per, groups);
    fetch(tok, g);
    float c[4], s[4];
    if (ratio != 0.0) {
      const int32_t pos = positions[tok];
#pragma unroll
      for (int v = 0; v < 4; ++v) turn<T>(pos, F[v], c[v], s[v]);
    }
    for (; g < g1; ++g) {
      float x[8];
      Four<T>::get(r0, x);
      Four<T>::get(r1, x + 4);
      if (g + 1 < g1) fetch(tok, g + 1);
      const int h = g * HPW + hl;
      const bool is_q = h < hq;
      if (is_q ? q_weight != nullptr : k_weight != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        const float ms = head_sum<DH>(ss) * (1.f / DH) + eps;
        if (ms > 0x1p-60f && ms < 0x1p100f) {
          const float r = __builtin_amdgcn_rsqf(ms);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= r;
        } else {
          norm_far<DH>(x, eps);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= is_q ? wq[e] : wk[e];
      }
      if (ratio != 0.0) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float a = x[v], b = x[4 + v];
          x[v] = a * c[v] - b * s[v];
          x[4 + v] = b * c[v] + a * s[v];
        }
      }
      if (h < heads) {
        T* dst = is_q ? q_out + tok * q_out_stride + (int64_t)h * DH : k_out + tok * k_out_stride + (int64_t)(h - hq) * DH;
        store4(dst + d0, x);
        store4(dst + d1, x + 4);
      }
    }
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const Problem& P, int64_t n_tokens, const void* q, int64_t q_stride, const void* k,
                               int64_t k_stride, const void* q_weight, const void* k_weight, float eps,
                               const int32_t* positions, void* q_out, int64_t q_out_stride, void* k_out,
                               int64_t k_out_stride, hipStream_t st) {
  const int hq = q ? P.hq : 0, heads = hq + (k ? P.hkv : 0);
  const int hpw = 512 / P.dh, groups = (heads + hpw - 1) / hpw;
  // few tokens: a wave for each group of heads; many: a token's heads in one wave,
  // which then works out the token's turns once (32764 tokens of 32 + 8 heads: 124 us,
  // 5.4 TB/s; waves that take several tokens, 256 / 512 / 1024 / 1536 workgroups in all: 281 /
  // 175 / 126 / 148 us; stores through the caches 132 us).  One side / the other: 32 tokens 3.2 /
  // 7.4 us, 512 tokens 5.5 / 8.6, 819 tokens 7.9 / 9.3, 1000 tokens 9.5 / 11.2, 2000 tokens
  // 17.4 / 14.3
  const int per = n_tokens * groups <= 8192 ? 1 : groups;
  const int64_t units = n_tokens * ((groups + per - 1) / per);
  const dim3 grid((unsigned)std::min<int64_t>((units + 3) / 4, 1 << 20));
  auto go = [&](auto elem, auto dh) {
    using T = decltype(elem);
    hipLaunchKernelGGL((k_qk_norm_rope<T, dh()>), grid, dim3(256), 0, st, (const T*)q, q_stride, (const T*)k, k_stride,
                       (const T*)q_weight, (const T*)k_weight, eps, positions, (T*)q_out, q_out_stride,
                       (T*)k_out, k_out_stride, n_tokens, hq, heads, per, rope_ratio(P));
  };
  auto by_type = [&](auto dh) {
    if (P.dtype == S4R_BF16)
      go(uint16_t(), dh);
    else
      go(float(), dh);
  };
  if (P.dh == 128)
    by_type(std::integral_constant<int, 128>());
  else
    by_type(std::integral_constant<int, 64>());
  return hipGetLastError();
}

}  // namespace s4r
