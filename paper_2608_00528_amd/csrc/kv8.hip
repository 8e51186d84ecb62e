// The 8-bit KV cache's writer and reader (layout and number formats: kv8.h).
//
// A workgroup owns one block (64 tokens) of one KV head, sequence and side: 2 d_h
// threads, thread (c = t / (d_h / 8), dc = t % (d_h / 8)) holds dims 8 dc .. + 7 of
// the tokens c, 16 + c, 32 + c and 48 + c.  Those four tokens are neighbours in
// the value order, so a thread writes dwords there and 8-byte pieces in the key
// order; the block's image is put together in LDS and leaves in 16-byte stores.
// Both directions are bound by HBM: d_h * 64 elements of the rows' type and as many
// bytes of codes per block.
#include "kv8.h"

namespace s4r {
namespace {

// eight consecutive elements of a row
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                            pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// the numbers of this thread's pieces of a block image, x[i][e]: token 16 i + c, dim 8 dc + e
template <int FMT, int DH>
__device__ __forceinline__ void pieces_of(const uint8_t* img, bool keys, int c, int dc, float (&x)[4][8]) {
  if (keys) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>(img + key_offset(16 * i + c, 8 * dc, DH));
      float a[4], b[4];
      kv8_numbers<FMT>(w.x, a);
      kv8_numbers<FMT>(w.y, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = a[e], x[i][4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a[4];
      kv8_numbers<FMT>(*reinterpret_cast<const uint32_t*>(img + value_offset(c, 8 * dc + e)), a);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i][e] = a[i];
    }
  }
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}

template <typename T, int FMT, int DH>
__global__ __launch_bounds__(DH * 2) void k_kv8_write(const T* __restrict__ k_rows, int64_t k_stride,
                                                      const T* __restrict__ v_rows, int64_t v_stride,
                                                      uint8_t* __restrict__ k_codes, float* __restrict__ k_scales,
                                                      uint8_t* __restrict__ v_codes, float* __restrict__ v_scales,
                                                      const int32_t* __restrict__ starts,
                                                      const int32_t* __restrict__ counts, int64_t row0, int n_rows,
                                                      int64_t cap, int tiles) {
  constexpr int NT = DH * 2, NW = NT / 64;
  const int j = blockIdx.y, b = blockIdx.z >> 1, hkv = gridDim.y;
  const bool keys = (blockIdx.z & 1) == 0;
  const int t = threadIdx.x, c = t / (DH / 8), dc = t % (DH / 8);
  int64_t start;
  int count;
  kv8_rows(starts, counts, b, row0, n_rows, cap, start, count);
  const int64_t tile = start / kKv8Block + blockIdx.x;
  const int64_t first = tile * kKv8Block - start;              // the block's first token among the call's rows
  if (first >= count) return;
  const int lo = first < 0 ? (int)-first : 0;                  // tokens [lo, hi) of the block are written
  const int hi = (int)min<int64_t>(kKv8Block, count - first);
  const int64_t at = ((int64_t)b * hkv + j) * tiles + tile;
  uint8_t* codes = (keys ? k_codes : v_codes) + at * (kKv8Block * DH);
  float* scale = (keys ? k_scales : v_scales) + at;
  const T* rows = keys ? k_rows : v_rows;
  const int64_t stride = keys ? k_stride : v_stride;

  __shared__ __align__(16) uint8_t img[kKv8Block * DH];
  __shared__ uint32_t wave_top[NW];
  const bool whole = lo == 0 && hi == kKv8Block;
  uint4 old[2];
  float s_old = 0.f;
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 2; ++i) old[i] = reinterpret_cast<const uint4*>(codes)[t + i * NT];
    if (lo > 0) s_old = *scale;
  }
  float x[4][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = min(max(16 * i + c, lo), hi - 1);            // a row that is there, masked below
    load8(rows + ((int64_t)b * n_rows + first + r) * stride + (int64_t)j * DH + 8 * dc, x[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (16 * i + c >= lo && 16 * i + c < hi) {
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7FFFFFFFu);
    }
  top = wave_max_u32(top);
  if ((t & 63) == 0) wave_top[t >> 6] = top;
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<uint4*>(img)[t + i * NT] = old[i];
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) top = max(top, wave_top[w]);
  float s = kv8_scale<FMT>(top);
  if (lo > 0) s = (s != s || s_old != s_old) ? __uint_as_float(0x7FC00000u) : fmaxf(s, s_old);
  const float inv = kv8_inverse<FMT>(s);
  // the tokens of this thread that stay as they are: those past the last written,
  // and the older ones unless the scale grew
  uint32_t keep = 0;
  if (!whole) {
    const bool redo = lo > 0 && !(s == s_old);
    float z[4][8];
    pieces_of<FMT, DH>(img, keys, c, dc, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + c;
      if (r >= hi || (r < lo && !redo)) keep |= 0xFFu << (8 * i);
      if (r < lo) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = z[i][e] * s_old;
      }
    }
  }
  if (keys) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (keep >> (8 * i) & 0xFFu) continue;
      uint2 w;
      w.x = kv8_code4<FMT>(x[i][0], x[i][1], x[i][2], x[i][3], s, inv);
      w.y = kv8_code4<FMT>(x[i][4], x[i][5], x[i][6], x[i][7], s, inv);
      *reinterpret_cast<uint2*>(img + key_offset(16 * i + c, 8 * dc, DH)) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t* p = reinterpret_cast<uint32_t*>(img + value_offset(c, 8 * dc + e));
      uint32_t w = kv8_code4<FMT>(x[0][e], x[1][e], x[2][e], x[3][e], s, inv);
      if (keep) w = (w & ~keep) | (*p & keep);
      *p = w;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) reinterpret_cast<uint4*>(codes)[t + i * NT] = reinterpret_cast<const uint4*>(img)[t + i * NT];
  if (t == 0) *scale = s;
}

template <typename T, int FMT, int DH>
__global__ __launch_bounds__(DH * 2) void k_kv8_read(const uint8_t* __restrict__ k_codes,
                                                     const float* __restrict__ k_scales,
                                                     const uint8_t* __restrict__ v_codes,
                                                     const float* __restrict__ v_scales,
                                                     const int32_t* __restrict__ starts,
                                                     const int32_t* __restrict__ counts, int64_t row0, int n_rows,
                                                     int64_t cap, int tiles, T* __restrict__ k_out,
                                                     T* __restrict__ v_out) {
  constexpr int NT = DH * 2;
  const int j = blockIdx.y, b = blockIdx.z >> 1, hkv = gridDim.y;
  const bool keys = (blockIdx.z & 1) == 0;
  const int t = threadIdx.x, c = t / (DH / 8), dc = t % (DH / 8);
  int64_t start;
  int count;
  kv8_rows(starts, counts, b, row0, n_rows, cap, start, count);
  const int64_t tile = start / kKv8Block + blockIdx.x;
  const int64_t first = tile * kKv8Block - start;
  if (first >= n_rows) return;
  float x[4][8];
  if (first < count) {
    const int64_t at = ((int64_t)b * hkv + j) * tiles + tile;
    const uint8_t* codes = (keys ? k_codes : v_codes) + at * (kKv8Block * DH);
    const float s = (keys ? k_scales : v_scales)[at];
    __shared__ __align__(16) uint8_t img[kKv8Block * DH];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      reinterpret_cast<uint4*>(img)[t + i * NT] = reinterpret_cast<const uint4*>(codes)[t + i * NT];
    __syncthreads();
    pieces_of<FMT, DH>(img, keys, c, dc, x);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] *= s;
  }
  T* out = (keys ? k_out : v_out) + (int64_t)b * n_rows * hkv * DH + (int64_t)j * DH + 8 * dc;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = first + 16 * i + c;
    if (r < 0 || r >= n_rows) continue;
    if (r >= count) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    }
    store8(out + r * hkv * DH, x[i]);
  }
}

// blocks that n rows touch: one more than they fill where their first row is known
// only on the device
int blocks_touched(const Kv8& C, int64_t n_rows) {
  const int64_t n = C.starts ? (n_rows + 2 * kKv8Block - 2) / kKv8Block
                             : (C.row0 + n_rows + kKv8Block - 1) / kKv8Block - C.row0 / kKv8Block;
  return (int)n;
}

template <typename F>
void by_type(const Problem& P, int format, F f) {
  auto by_dh = [&](auto elem, auto fmt) {
    if (P.dh == 128)
      f(elem, fmt, std::integral_constant<int, 128>());
    else
      f(elem, fmt, std::integral_constant<int, 64>());
  };
  auto by_fmt = [&](auto elem) {
    if (format == S4R_KV_INT8)
      by_dh(elem, std::integral_constant<int, S4R_KV_INT8>());
    else
      by_dh(elem, std::integral_constant<int, S4R_KV_E4M3>());
  };
  if (P.dtype == S4R_BF16)
    by_fmt(uint16_t());
  else
    by_fmt(float());
}

}  // namespace

hipError_t launch_kv8_write(const Problem& P, const Kv8& C, int64_t n_rows, const void* k_rows, int64_t k_stride,
                            const void* v_rows, int64_t v_stride, hipStream_t st) {
  by_type(P, C.format, [&](auto elem, auto fmt, auto dh) {
    using T = decltype(elem);
    hipLaunchKernelGGL((k_kv8_write<T, fmt(), dh()>), dim3(blocks_touched(C, n_rows), P.hkv, 2 * P.B), dim3(2 * dh()),
                       0, st, (const T*)k_rows, k_stride, (const T*)v_rows, v_stride, C.k_codes, C.k_scales, C.v_codes,
                       C.v_scales, C.starts, C.counts, C.row0, (int)n_rows, P.cap, kv8_tiles(P));
  });
  return hipGetLastError();
}

hipError_t launch_kv8_read(const Problem& P, const Kv8& C, int64_t n_rows, void* k_out, void* v_out, hipStream_t st) {
  by_type(P, C.format, [&](auto elem, auto fmt, auto dh) {
    using T = decltype(elem);
    hipLaunchKernelGGL((k_kv8_read<T, fmt(), dh()>), dim3(blocks_touched(C, n_rows), P.hkv, 2 * P.B), dim3(2 * dh()), 0,
                       st, C.k_codes, C.k_scales, C.v_codes, C.v_scales, C.starts, C.counts, C.row0, (int)n_rows, P.cap,
                       kv8_tiles(P), (T*)k_out, (T*)v_out);
  });
  return hipGetLastError();
}

}  // namespace s4r
