// The 8-bit KV cache's writer and reader (layout and number formats: kv8.h).
//
// A workgroup owns one block (64 tokens) of one KV head, sequence and side: 2 d_h
// threads, thread (c = t / (d_h / 8), dc = t % (d_h / 8)) holds dims 8 dc .. + 7 of
// the tokens c, 16 + c, 32 + c and 48 + c.  Those four tokens are neighbours in
// the value order, so a thread writes dwords there and 8-byte pieces in the key
// order; the block's image is put together in LDS and leaves in 16-byte stores.
// Both directions are bound by HBM: d_h * 64 elements of the rows' type and as many
// bytes of codes per block.  The heads of a block run side by side, so the rows' lines
// are used whole (a head's blocks side by side: 624 us and 816 us), and what passes
// through once goes past the caches (without: 563 and 583).  4 x 131068 rows of 8 heads
// of 128, bf16, K and V: written in 520 us (6.2 TB/s), read in 571 us (5.6 TB/s); one
// row for each of 32 sequences 6.9 us, most of it the chain start -> rows -> scale.
#include "kv8.h"

namespace s4r {
namespace {

// eight consecutive elements of a row
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const kv8_u4 u = __builtin_nontemporal_load(reinterpret_cast<const kv8_u4*>(p));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const floatx4 a = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(p)),
                b = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(p + 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  const kv8_u4 u = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  __builtin_nontemporal_store(u, reinterpret_cast<kv8_u4*>(p));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  __builtin_nontemporal_store(floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<floatx4*>(p));
  __builtin_nontemporal_store(floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<floatx4*>(p + 4));
}

// this thread's codes in a block image: w[e] holds dim 8 dc + e of the tokens c, 16 + c,
// 32 + c, 48 + c (a dword of the value order; turned from and to the key order's
// 8 bytes per token)
template <int DH>
__device__ __forceinline__ void get_codes(const uint8_t* img, bool keys, int c, int dc, uint32_t (&w)[8]) {
  if (keys) {
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const kv8_u2 u = *reinterpret_cast<const kv8_u2*>(img + key_offset(16 * i + c, 8 * dc, DH));
      lo[i] = u[0];
      hi[i] = u[1];
    }
    kv8_turn4(lo, w);
    kv8_turn4(hi, w + 4);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint32_t*>(img + value_offset(c, 8 * dc + e));
  }
}
template <int DH>
__device__ __forceinline__ void put_codes(uint8_t* img, bool keys, int c, int dc, const uint32_t (&w)[8]) {
  if (keys) {
    uint32_t lo[4], hi[4];
    kv8_turn4(w, lo);
    kv8_turn4(w + 4, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<kv8_u2*>(img + key_offset(16 * i + c, 8 * dc, DH)) = kv8_u2{lo[i], hi[i]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) *reinterpret_cast<uint32_t*>(img + value_offset(c, 8 * dc + e)) = w[e];
  }
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));    // quad_perm [1,0,3,2]
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));    // quad_perm [2,3,0,1]
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, false));   // row_ror:4
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false));   // row_ror:8
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}

// workgroup -> (head, block of the call, sequence, side); the heads of a block next to
// each other, so the rows are read and written whole
struct Place {
  int j, blk, b;
  bool keys;
};
__device__ __forceinline__ Place place(int hkv) {
  Place p;
  p.blk = blockIdx.x / hkv;
  p.j = blockIdx.x - p.blk * hkv;
  p.keys = blockIdx.y == 0;
  p.b = blockIdx.z;
  return p;
}

template <typename T, int FMT, int DH>
__global__ __launch_bounds__(DH * 2) void k_kv8_write(const T* __restrict__ k_rows, int64_t k_stride,
                                                      const T* __restrict__ v_rows, int64_t v_stride,
                                                      uint8_t* __restrict__ k_codes, float* __restrict__ k_scales,
                                                      uint8_t* __restrict__ v_codes, float* __restrict__ v_scales,
                                                      const int32_t* __restrict__ starts,
                                                      const int32_t* __restrict__ counts, int64_t row0, int n_rows,
                                                      int64_t cap, int tiles, int hkv) {
  constexpr int NT = DH * 2, NW = NT / 64;
  const Place at = place(hkv);
  const bool keys = at.keys;
  const int t = threadIdx.x, c = t / (DH / 8), dc = t % (DH / 8);
  int64_t start;
  int count;
  kv8_rows(starts, counts, at.b, row0, n_rows, cap, start, count);
  const int64_t tile = start / kKv8Block + at.blk;
  const int64_t first = tile * kKv8Block - start;              // the block's first token among the call's rows
  if (first >= count) return;
  const int lo = first < 0 ? (int)-first : 0;                  // tokens [lo, hi) of the block are written
  const int hi = (int)min<int64_t>(kKv8Block, count - first);
  const int64_t blk = ((int64_t)at.b * hkv + at.j) * tiles + tile;
  kv8_u4* codes = reinterpret_cast<kv8_u4*>((keys ? k_codes : v_codes) + blk * (kKv8Block * DH)) + t;
  float* scale = (keys ? k_scales : v_scales) + blk;
  const int64_t stride = keys ? k_stride : v_stride;
  const T* rows = (keys ? k_rows : v_rows) + ((int64_t)at.b * n_rows + first) * stride + (int64_t)at.j * DH + 8 * dc;

  __shared__ __align__(16) uint8_t img[kKv8Block * DH];
  __shared__ uint32_t wave_top[NW];
  kv8_u4* image = reinterpret_cast<kv8_u4*>(img) + t;
  const bool whole = lo == 0 && hi == kKv8Block;
  kv8_u4 old0 = {0, 0, 0, 0}, old1 = old0;
  float s_old = 0.f;
  if (!whole) {
    old0 = codes[0];
    old1 = codes[NT];
    s_old = *scale;
  }
  float x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) load8(rows + min(max(16 * i + c, lo), hi - 1) * stride, x[i]);   // a row that is there
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7FFFFFFFu);        // repeats change nothing
  top = wave_max_u32(top);
  if ((t & 63) == 0) wave_top[t >> 6] = top;
  if (!whole) {
    image[0] = old0;
    image[NT] = old1;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) top = max(top, wave_top[w]);
  float s = kv8_scale<FMT>(top);
  if (lo > 0) s = (s != s || s_old != s_old) ? __uint_as_float(0x7FC00000u) : fmaxf(s, s_old);
  const float inv = kv8_inverse<FMT>(s);
  // bytes of this thread's codes that stay as they are: the tokens past the last
  // written, and the older ones unless the scale grew
  uint32_t keep = 0, w_old[8];
  if (!whole) {
    get_codes<DH>(img, keys, c, dc, w_old);
    const bool redo = !(s == s_old);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + c;
      if (r >= hi || (r < lo && !redo)) keep |= 0xFFu << (8 * i);
    }
    if (lo > 0 && redo) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float z[4];
        kv8_numbers<FMT>(w_old[e], z);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * i + c < lo) x[i][e] = z[i] * s_old;
      }
    }
  }
  uint32_t w[8];
  if (FMT == S4R_KV_INT8) {
    float worst = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = kv8_int8x4(x[0][e], x[1][e], x[2][e], x[3][e], s, inv, worst);
    if (!(worst < 0.5f * s)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = kv8_int8x4_exact(x[0][e], x[1][e], x[2][e], x[3][e], s, inv);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = kv8_e4m3x4(x[0][e], x[1][e], x[2][e], x[3][e], inv);
  }
  if (inv == 0.f) {                                            // a block of zeros, or one that holds no values
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 0;
  }
  if (!whole) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (w[e] & ~keep) | (w_old[e] & keep);
  }
  put_codes<DH>(img, keys, c, dc, w);
  __syncthreads();
  codes[0] = image[0];
  codes[NT] = image[NT];
  if (t == 0) *scale = s;
}

template <typename T, int FMT, int DH>
__global__ __launch_bounds__(DH * 2) void k_kv8_read(const uint8_t* __restrict__ k_codes,
                                                     const float* __restrict__ k_scales,
                                                     const uint8_t* __restrict__ v_codes,
                                                     const float* __restrict__ v_scales,
                                                     const int32_t* __restrict__ starts,
                                                     const int32_t* __restrict__ counts, int64_t row0, int n_rows,
                                                     int64_t cap, int tiles, int hkv, T* __restrict__ k_out,
                                                     T* __restrict__ v_out) {
  constexpr int NT = DH * 2;
  const Place at = place(hkv);
  const int t = threadIdx.x, c = t / (DH / 8), dc = t % (DH / 8);
  int64_t start;
  int count;
  kv8_rows(starts, counts, at.b, row0, n_rows, cap, start, count);
  const int64_t tile = start / kKv8Block + at.blk;
  const int64_t first = tile * kKv8Block - start;
  if (first >= n_rows) return;
  __shared__ __align__(16) uint8_t img[kKv8Block * DH];
  kv8_u4* image = reinterpret_cast<kv8_u4*>(img) + t;
  float s = 0.f;
  if (first < count) {
    const int64_t blk = ((int64_t)at.b * hkv + at.j) * tiles + tile;
    const kv8_u4* codes = reinterpret_cast<const kv8_u4*>((at.keys ? k_codes : v_codes) + blk * (kKv8Block * DH)) + t;
    const kv8_u4 a = __builtin_nontemporal_load(codes), b = __builtin_nontemporal_load(codes + NT);
    s = (at.keys ? k_scales : v_scales)[blk];
    image[0] = a;
    image[NT] = b;
  }
  __syncthreads();
  uint32_t w[8];
  get_codes<DH>(img, at.keys, c, dc, w);
  float x[4][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float z[4];
    kv8_numbers<FMT>(w[e], z);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i][e] = 16 * i + c < count - first ? z[i] * s : 0.f;
  }
  const int64_t width = (int64_t)hkv * DH;
  T* out = (at.keys ? k_out : v_out) + ((int64_t)at.b * n_rows + first) * width + (int64_t)at.j * DH + 8 * dc;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = first + 16 * i + c;
    if (r >= 0 && r < n_rows) store8(out + (16 * i + c) * width, x[i]);
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
    hipLaunchKernelGGL((k_kv8_write<T, fmt(), dh()>), dim3(blocks_touched(C, n_rows) * P.hkv, 2, P.B),
                       dim3(2 * dh()), 0, st, (const T*)k_rows, k_stride, (const T*)v_rows, v_stride, C.k_codes, C.k_scales, C.v_codes,
                       C.v_scales, C.starts, C.counts, C.row0, (int)n_rows, P.cap, kv8_tiles(P), P.hkv);
  });
  return hipGetLastError();
}

hipError_t launch_kv8_read(const Problem& P, const Kv8& C, int64_t n_rows, void* k_out, void* v_out, hipStream_t st) {
  by_type(P, C.format, [&](auto elem, auto fmt, auto dh) {
    using T = decltype(elem);
    hipLaunchKernelGGL((k_kv8_read<T, fmt(), dh()>), dim3(blocks_touched(C, n_rows) * P.hkv, 2, P.B),
                       dim3(2 * dh()), 0, st, C.k_codes, C.k_scales, C.v_codes, C.v_scales, C.starts, C.counts, C.row0, (int)n_rows, P.cap,
                       kv8_tiles(P), P.hkv, (T*)k_out, (T*)v_out);
  });
  return hipGetLastError();
}

}  // namespace s4r
