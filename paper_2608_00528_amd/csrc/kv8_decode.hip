// Attention of one or a few query tokens per sequence over the 8-bit KV cache
// (layout: kv8.h).
//
//   s_t = (q . k_t) * scale_k(block) / sqrt(d_h),  p = exp(s - M),
//   out = sum_t p_t scale_v(block) v_t / sum_t p_t
//
// with the running maximum M and sum of one pass over the tokens.  Bound by HBM:
// 2 d_h bytes per token and KV head, so every other cost has to hide under the
// stream:
//  - the codes are operands as loaded (16 bytes per lane, 1 KiB per wave load) and
//    become bf16 exactly; 16 or 32 query rows (query token x group member) share them;
//  - logits as K q^T: 16 tokens x 16 query rows per MFMA, so lane l ends with
//    query row l % 16 and the tokens 16 i + 4 (l / 16) + v of the block - which is
//    the A operand of P V, with no exchange between lanes;
//  - scales are one number per block: the logits' goes into the exponent's factor,
//    the values' into the addition of the block's sums;
//  - bf16 queries are operands as they are, fp32 ones three bf16 parts, all of their 24
//    bits (two fp16 parts kept 22: at logits of 64 a weight was off by 2.3e-5); a row is
//    scaled by a power of two to below 1, so that its products with the codes stay finite;
//  - softmax weights enter as three bf16 parts, all of their 24 bits and fp32's range: a
//    token that holds nearly all the weight may have a value of zero (an attention sink),
//    and the output is then made of weights far below the largest (two fp16 parts lost
//    all of it at e^-23 and 3e-3 of it at e^-15).  Products with the codes are exact, sums
//    are fp32.
//
// Work is split over one workgroup per CU by the tokens that are there: the blocks of
// all (sequence, KV head) pairs in a row, an equal run of them for each workgroup, whose
// four waves take the blocks in turn.  A pair inside one run is finished there; one cut
// by the ends of runs leaves a partial (max, sum, output) per run and k_kv8_combine
// merges them in order.  Lengths are read on the device, so a captured graph follows them.
// Short caches have a workgroup or, in large batches, a wave for each pair instead.
//
// Measured (kernel): 4 x 131068 tokens, 8 KV heads of 128: 161 us, 6.7 TB/s (a large
// read reaches 6.2, a copy 5.1), 621 VALU and 64 MFMA instructions a block of int8 codes, 365
// and 64 of e4m3.  Workgroups in all, with k_kv8_combine: 128 / 192 / 256 / 320 / 384 / 512
// take 221 / 167 / 165 / 213 / 181 / 168 us: more reads on their way than 64 KB per CU make
// the memory no faster.  A block takes a wave 1.6 to 1.8 us of a quiet chip (8 pairs of 512 /
// 1024 / 2048 tokens, a workgroup each: 7.7 / 10.8 / 17.9 us) and 2.4 at the memory's rate; 1 x
// 32764 tokens are 17.2 us for four blocks a wave, and 3.9 for k_kv8_combine.
#include "kv8.h"

namespace s4r {
namespace {

constexpr int kWaves = 4;
constexpr float kGrow = 6.f;            // the running maximum follows once a logit is 2^6 above it
constexpr int kWeightParts = 3;         // bf16 parts of a softmax weight

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// the upper halves of two fp32 values: packed bf16, cut off
__device__ __forceinline__ uint32_t upper2(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
// the same, and what is left of the values (exact)
__device__ __forceinline__ uint32_t take_bf16x2(float& a, float& b) {
  const uint32_t u = upper2(a, b);
  a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
  b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
  return u;
}

// eight codes -> eight bf16 values (exact)
template <int FMT>
__device__ __forceinline__ Op8 codes_to_bf16(uint32_t w0, uint32_t w1) {
  Op8 o;
  if (FMT == S4R_KV_INT8) {
    float a[4], b[4];
    kv8_numbers<FMT>(w0, a);
    kv8_numbers<FMT>(w1, b);
    o.u = make_uint4(upper2(a[0], a[1]), upper2(a[2], a[3]), upper2(b[0], b[1]), upper2(b[2], b[3]));
  } else {
    o.u.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false));
    o.u.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true));
    o.u.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false));
    o.u.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true));
  }
  return o;
}

// max / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float rows_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// the sequences' tokens: lengths on the device (clamped to [0, n_max]) or n_max each
struct Seqs {
  const int32_t* lengths;
  int n_max, B, hkv;
  __device__ __forceinline__ int tokens(int b) const { return lengths ? min(max(lengths[b], 0), n_max) : n_max; }
};
__device__ __forceinline__ int blocks_of(int tokens) { return (tokens + kKv8Block - 1) / kKv8Block; }
__device__ __forceinline__ int wave_scan(int x) {               // inclusive prefix sum over the lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
  return x;
}

// The (sequence, KV head) pairs lie on a line that is cut into equal runs.  A pair takes
// its blocks rounded up to one for every wave, and room for another round where it is
// shorter than a run: ending a pair costs a run about as much, and a run of many short
// pairs would end long after the others (with / without: 32 sequences of 0 to 32765 tokens 167 /
// 169 us, 256 of 1 to 1000 69 / 88).
__host__ __device__ inline int pair_length(int blocks, int shorter) {
  return blocks == 0 ? 0 : (blocks + kWaves - 1) / kWaves * kWaves + (blocks < shorter ? kWaves : 0);
}
__host__ __device__ inline int run_length(int total, int nwg) {
  return ((total + nwg - 1) / nwg + kWaves - 1) / kWaves * kWaves;
}

// the line; every wave holds the same, one sequence per lane, 64 at a time
struct Order {
  Seqs S;
  int shorter;                // pairs of fewer blocks than this have the room
  int all;                    // the line's length
  int base;                   // the lanes hold sequences base .. base + 63
  int tok, mine, upto;        // this lane's sequence: tokens, its pairs' length, and the line up to its end
  __device__ __forceinline__ explicit Order(const Seqs& s) : S(s), shorter(0), all(0) {}
  __device__ __forceinline__ int length(int blocks) const { return pair_length(blocks, shorter); }
  __device__ __forceinline__ void load(int b0, int before) {
    const int b = b0 + (int)(threadIdx.x & 63);
    base = b0;
    tok = b < S.B ? S.tokens(b) : 0;
    place(before);
  }
  __device__ __forceinline__ void place(int before) {
    mine = length(blocks_of(tok)) * S.hkv;
    upto = before + wave_scan(mine);
  }
  __device__ __forceinline__ int end() const { return __builtin_amdgcn_readlane(upto, 63); }
  __device__ __forceinline__ int total() const {
    if (S.B <= 64) return end();
    if (!S.lengths) return S.B * S.hkv * length(blocks_of(S.n_max));
    int n = 0;
#pragma unroll 4
    for (int b = threadIdx.x & 63; b < S.B; b += 64) n += length(blocks_of(S.tokens(b)));
    return __builtin_amdgcn_readlane(wave_scan(n), 63) * S.hkv;
  }
  // the line laid out for nwg runs; returns the length of a run, a multiple of the waves
  __device__ __forceinline__ int lay_out(int nwg) {
    load(0, 0);
    shorter = (total() + nwg - 1) / nwg;
    place(0);
    all = total();
    return run_length(all, nwg);
  }
  // the sequence at u (the lanes move on to it): its number, place and tokens
  __device__ __forceinline__ void find(int u, int& seq, int& begin, int& tokens) {
    if (S.B > 64 && !S.lengths) {
      const int per = length(blocks_of(S.n_max)) * S.hkv;
      seq = u / per;
      begin = seq * per;
      tokens = S.n_max;
      return;
    }
    while (end() <= u && base + 64 < S.B) load(base + 64, end());
    const int l = __ffsll((unsigned long long)__ballot(upto > u)) - 1;
    seq = base + l;
    begin = __builtin_amdgcn_readlane(upto - mine, l);
    tokens = __builtin_amdgcn_readlane(tok, l);
  }
  // the place and tokens of sequence b
  __device__ __forceinline__ void of(int b, int& begin, int& tokens) {
    if (S.B > 64 && !S.lengths) {
      begin = b * length(blocks_of(S.n_max)) * S.hkv;
      tokens = S.n_max;
      return;
    }
    while (base + 64 <= b) load(base + 64, end());
    begin = __builtin_amdgcn_readlane(upto - mine, b & 63);
    tokens = __builtin_amdgcn_readlane(tok, b & 63);
  }
};

// eight query elements as fp32; bf16 parts that hold them
template <typename T>
struct Query;
template <>
struct Query<uint16_t> {
  static constexpr int parts = 1;
  __device__ __forceinline__ static void load(const uint16_t* p, float* x) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Query<float> {
  static constexpr int parts = 3;
  __device__ __forceinline__ static void load(const float* p, float* x) {
    const floatx4 a = *reinterpret_cast<const floatx4*>(p), b = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
};

// partials: run w leaves slot 2 w for a pair that began before the run and slot
// 2 w + 1 for one that begins in it and goes on behind it; per slot, chunk of query
// rows and row a (max, sum) and d_h sums
__device__ __forceinline__ int64_t part_row(int slot, int chunks, int chunk, int row) {
  return ((int64_t)slot * chunks + chunk) * kKv8Rows + row;
}

// RC: chunks of 16 query rows that a workgroup works on; they share its blocks and
// their conversion.  SHARE: waves that take a pair's blocks in turn - the workgroup's, or
// 1: a pair to each wave, nothing to merge, and a workgroup's waves never wait for each
// other (one_wave_per_pair).  Two workgroups' registers fit a CU but for fp32 queries over
// 128 dims, whose parts take 264: held to 256, 8 x 16256 tokens of 8 KV heads take 57.0 us,
// not 51.0, 4 x 131068 of e4m3 171.7, not 165.0, and 512 pairs of 512 21.8, not 20.0
template <typename T, int FMT, int DH, int RC, int SHARE>
__global__ __launch_bounds__(kWaves * 64, RC == 1 && (sizeof(T) == 2 || DH == 64) ? 2 : 1) void k_kv8_decode(
    const T* __restrict__ q, const uint8_t* __restrict__ k_codes, const float* __restrict__ k_scales,
    const uint8_t* __restrict__ v_codes, const float* __restrict__ v_scales, float* __restrict__ part_ml,
    float* __restrict__ part_o, float* __restrict__ out, Seqs S, int nwg, int by_pair, int chunks, int n_q, int G,
    int tiles) {
  constexpr int NP = Query<T>::parts, NK = DH / 16, NV = DH / 16;   // 1 KiB pieces of a block per side
  constexpr int KB = DH / 64, ROWS = RC * kKv8Rows;
  static_assert(SHARE == 1 || SHARE == kWaves, "a wave or a workgroup per pair");
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // workgroups of one run's query rows 8 ids apart: on one XCD, sharing its L2
  const int sets = (chunks + RC - 1) / RC;
  const int id = blockIdx.x, set = (id >> 3) % sets, wg = (id >> 3) / sets * 8 + (id & 7);
  const int w = SHARE == 1 ? wg * kWaves + wave : wg, turn = SHARE == 1 ? 0 : wave;
  if (w >= nwg) return;
  const int col = lane & 15, kg = lane >> 4;
  const int hkv = S.hkv, hq = hkv * G, rows = n_q * G;
  constexpr int MROWS = SHARE == 1 ? 1 : ROWS;                  // rows to merge
  __shared__ float wm[SHARE][MROWS], wl[SHARE][MROWS];
  __shared__ float wo[SHARE][MROWS][DH];

  // this lane's query rows in the logits, the tokens that their query tokens do not see
  // yet, and the same of the rows it holds in the outputs
  int row[RC], back[RC], back_out[RC][4];
  auto not_seen = [&](int r) { return r < rows ? n_q - 1 - r / G : 0; };
#pragma unroll
  for (int r = 0; r < RC; ++r) {
    row[r] = set * ROWS + r * kKv8Rows + col;
    back[r] = not_seen(row[r]);
#pragma unroll
    for (int v = 0; v < 4; ++v) back_out[r][v] = not_seen(set * ROWS + r * kKv8Rows + 4 * kg + v);
  }
  const float to_log2 = 1.4426950408889634f / sqrtf((float)DH);

  // a pair's blocks are [begin, end) of the line, the next pair begins at `next`;
  // block0: its first block in the cache
  struct Pair {
    int b, j, N, begin, end, next, block0;
  };
  Order order(S);
  auto pair_at = [&](int u) __attribute__((always_inline)) {
    Pair p;
    int begin;
    order.find(u, p.b, begin, p.N);
    const int blocks = blocks_of(p.N), length = order.length(blocks);
    p.j = (u - begin) / length;
    p.begin = begin + p.j * length;
    p.end = p.begin + blocks;
    p.next = p.begin + length;
    p.block0 = (p.b * hkv + p.j) * tiles;
    return p;
  };
  Pair pair, after;
  int u0 = 0, u1;                                               // this workgroup's run
  if (SHARE == 1 || by_pair) {
    pair.b = w / hkv;
    pair.j = w - pair.b * hkv;
    pair.N = __builtin_amdgcn_readfirstlane(S.tokens(pair.b));
    pair.begin = 0;
    u1 = pair.end = pair.next = blocks_of(pair.N);
    pair.block0 = w * tiles;
  } else {
    const int run = order.lay_out(nwg);
    u0 = w * run;
    u1 = min(u0 + run, order.all);
    if (u0 >= u1) return;
    pair = pair_at(u0);
  }
  const u32x4* kp = reinterpret_cast<const u32x4*>(k_codes) + lane;
  const u32x4* vp = reinterpret_cast<const u32x4*>(v_codes) + lane;
  u32x4 kk[NK], vv[NV];
  float sk, sv;
  auto load_keys = [&](int block) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NK; ++i) kk[i] = __builtin_nontemporal_load(kp + (int64_t)block * (kKv8Block * DH / 16) + i * 64);
    sk = k_scales[block];
  };
  auto load_values = [&](int block) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) vv[i] = __builtin_nontemporal_load(vp + (int64_t)block * (kKv8Block * DH / 16) + i * 64);
    sv = v_scales[block];
  };

  // Workgroups start a sixteenth of their part of a pair apart and come round to its
  // beginning: in step, with caches a few blocks short of a power of two, their streams
  // meet on the same memory channels (8 x 16256 tokens, 8 KV heads: 57 us; so 50 us).
  // The block of a pair that is read for position p of its part [us, ue):
  auto block_at = [&](const Pair& at, int p, int us, int ue) __attribute__((always_inline)) {
    const int rounds = (ue - us) / SHARE, turned = us + rounds * SHARE;
    int x = p + ((w & 15) * rounds >> 4) * SHARE;
    x -= x >= turned ? rounds * SHARE : 0;
    return (p < turned ? x : p) - at.begin;
  };
  // a wave takes every fourth block of the run, its next one on the way while it works
  // on one, also where that lies in the next pair
  int p = u0 + turn, have = -1;
  if (p < min(pair.end, u1)) {
    have = p;
    const int block = pair.block0 + block_at(pair, p, u0, min(pair.end, u1));
    load_keys(block);
    load_values(block);
  }
  for (int us = u0;; us = after.begin, p = us + turn, pair = after) {
    const int ue = min(pair.end, u1);
    const bool more = SHARE != 1 && pair.next < u1;
    after = pair;
    if (more) after = pair_at(pair.next);
    const int pa0 = after.begin + turn;                         // this wave's first block there
    const bool ahead = more && pa0 < min(after.end, u1);
    const int b = pair.b, j = pair.j, N = pair.N;
    float M[RC], l[RC];
    floatx4 acc[RC][NV];
#pragma unroll
    for (int r = 0; r < RC; ++r) {
      M[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) acc[r][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    if (p < ue) {
      if (have != p) {
        const int block = pair.block0 + block_at(pair, p, us, ue);
        load_keys(block);
        load_values(block);
      }
      Op8 qb[RC][KB][2][NP];
      float fq[RC];                                             // a row's power of two with 1 / sqrt(d_h) and log2 e
#pragma unroll
      for (int r = 0; r < RC; ++r) {
        const int i = min(row[r], rows - 1);
        const T* qp = q + (((int64_t)b * n_q + i / G) * hq + (int64_t)j * G + i % G) * DH;
        float x[KB][2][8], top = 0.f;
#pragma unroll
        for (int d = 0; d < KB; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Query<T>::load(qp + d * 64 + 16 * kg + 8 * h, x[d][h]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[d][h][e]));
          }
        top = rows_max(top);
        int up;                                                 // largest element in [1/2, 1) * 2^up
        (void)frexpf(top, &up);
        up = top > 0.f && top < INFINITY ? up : 0;
        fq[r] = ldexpf(to_log2, up);
#pragma unroll
        for (int d = 0; d < KB; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[d][h][e] = ldexpf(x[d][h][e], -up);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
              uint32_t u[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) u[e] = take_bf16x2(x[d][h][2 * e], x[d][h][2 * e + 1]);
              qb[r][d][h][p].u = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
      }
      do {
        const int tile = block_at(pair, p, us, ue);
        // the wave's next block; behind the next pair, or the run: this one again
        const bool on = p + SHARE < ue;
        have = on ? p + SHARE : (ahead ? pa0 : -1);
        const int block = on ? pair.block0 + block_at(pair, p + SHARE, us, ue)
                             : (ahead ? after.block0 + block_at(after, pa0, after.begin, min(after.end, u1)) : pair.block0 + tile);
        // logits, four sums side by side: a sum's next product waits for the one before it
        floatx4 s[RC][4];
#pragma unroll
        for (int r = 0; r < RC; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[r][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < KB; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Op8 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = codes_to_bf16<FMT>(kk[i * KB + d][2 * h], kk[i * KB + d][2 * h + 1]);
#pragma unroll
            for (int r = 0; r < RC; ++r)
#pragma unroll
              for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][i] = mfma16x16x32(a[i], qb[r][d][h][p], s[r][i]);
          }
        float f[RC];
#pragma unroll
        for (int r = 0; r < RC; ++r) f[r] = sk * fq[r];
        load_keys(block);
        // tokens that a query row does not see, or that do not exist (of a pair's last
        // blocks only)
        const bool part = (tile + 1) * kKv8Block > N - (n_q - 1);
        if (part) {
          const int there = N - tile * kKv8Block;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m |= (16 * i + 4 * kg + v < there) ? 0xFFu << (8 * i) : 0u;
#pragma unroll
            for (int i = 0; i < NV; ++i) vv[i][v] &= m;
          }
        }
        Op8 pa[RC][2][kWeightParts];
#pragma unroll
        for (int r = 0; r < RC; ++r) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) s[r][i][v] *= f[r];
          const int seen = N - back[r] - tile * kKv8Block;      // this row sees the block's first `seen` tokens
          if (part) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int v = 0; v < 4; ++v) s[r][i][v] = (16 * i + 4 * kg + v < seen) ? s[r][i][v] : -INFINITY;
          }
          float top = s[r][0][0];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) top = fmaxf(top, s[r][i][v]);
          top = rows_max(top);
          const bool grow = top > M[r] + kGrow;                 // also where M is -inf and a token is seen
          if (__ballot(grow)) {
            const float to = grow ? top : M[r];
            const float a = grow ? __builtin_amdgcn_exp2f(M[r] - to) : 1.f;
            M[r] = to;
            l[r] *= a;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const float av = __shfl(a, 4 * kg + v);           // lane r holds row r
#pragma unroll
              for (int i = 0; i < NV; ++i) acc[r][i][v] *= av;
            }
          }
          const float ref = M[r] == -INFINITY ? 0.f : M[r];
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              s[r][i][v] = __builtin_amdgcn_exp2f(s[r][i][v] - ref);
              sum += s[r][i][v];
            }
          l[r] += sum;
          // contraction index 4 v + i of k-group kg
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t part[kWeightParts][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int v = 2 * h + e / 2, i = 2 * (e % 2);
              float x = s[r][i][v], y = s[r][i + 1][v];
#pragma unroll
              for (int p = 0; p < kWeightParts; ++p) part[p][e] = take_bf16x2(x, y);
            }
#pragma unroll
            for (int p = 0; p < kWeightParts; ++p) pa[r][h][p].u = make_uint4(part[p][0], part[p][1], part[p][2], part[p][3]);
          }
        }
        // the block's scale; a row that sees none of its tokens takes no part, whatever it is
        float so[RC][4];
#pragma unroll
        for (int r = 0; r < RC; ++r)
#pragma unroll
          for (int v = 0; v < 4; ++v) so[r][v] = part && N - back_out[r][v] <= tile * kKv8Block ? 0.f : sv;
        // a block's products from zero, then added: the matrix unit cuts what it adds to a
        // large sum, which over a run of 64 blocks had made 2.3e-6 of the result
#pragma unroll
        for (int i0 = 0; i0 < NV; i0 += 4) {
          floatx4 o[RC][4];
#pragma unroll
          for (int r = 0; r < RC; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[r][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Op8 bv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) bv[i] = codes_to_bf16<FMT>(vv[i0 + i][2 * h], vv[i0 + i][2 * h + 1]);
#pragma unroll
            for (int r = 0; r < RC; ++r)
#pragma unroll
              for (int p = 0; p < kWeightParts; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[r][i] = mfma16x16x32(pa[r][h][p], bv[i], o[r][i]);
          }
#pragma unroll
          for (int r = 0; r < RC; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int v = 0; v < 4; ++v) acc[r][i0 + i][v] = fmaf(o[r][i][v], so[r][v], acc[r][i0 + i][v]);
        }
        load_values(block);
        p += SHARE;
      } while (p < ue);
    }
    if (SHARE == 1) {
#pragma unroll
      for (int r = 0; r < RC; ++r) {
        const float ls = rows_sum(l[r]), inv = ls == 0.f ? 0.f : 1.f / ls;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float to_out = __shfl(inv, 4 * kg + v);         // lane r holds row r
          const int gr = set * ROWS + r * kKv8Rows + 4 * kg + v;
          if (gr >= rows) continue;
          float* dst = out + (((int64_t)b * n_q + gr / G) * hq + (int64_t)j * G + gr % G) * DH + col;
#pragma unroll
          for (int i = 0; i < NV; ++i) dst[16 * i] = acc[r][i][v] * to_out;
        }
      }
      break;
    }
    if (!by_pair && us >= pair.end) {                           // the run begins in the room behind a pair
      if (!more) break;
      continue;
    }
    // merge the waves
#pragma unroll
    for (int r = 0; r < RC; ++r) {
      const float ls = rows_sum(l[r]);
      if (kg == 0) {
        wm[wave][r * kKv8Rows + col] = M[r];
        wl[wave][r * kKv8Rows + col] = ls;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) wo[wave][r * kKv8Rows + 4 * kg + v][16 * i + col] = acc[r][i][v];
    }
    __syncthreads();
    const bool whole = us == pair.begin && ue == pair.end;
    const int slot = us > pair.begin ? 2 * w : 2 * w + 1;
    for (int e = t; e < ROWS * DH; e += kWaves * 64) {
      const int r = e / DH, d = e % DH, gr = set * ROWS + r;
      if (gr >= rows) break;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, wm[i][r]);
      float sum = 0.f, o = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        // a wave without a maximum has sums of zero, or NaN, which stay
        const float a = wm[i][r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(wm[i][r] - top);
        sum += a * wl[i][r];
        o += a * wo[i][r][d];
      }
      if (whole) {
        out[(((int64_t)b * n_q + gr / G) * hq + (int64_t)j * G + gr % G) * DH + d] = sum == 0.f ? 0.f : o / sum;
      } else {
        const int64_t pr = part_row(slot, chunks, gr / kKv8Rows, gr % kKv8Rows);
        part_o[pr * DH + d] = o;
        if (d == 0) {
          part_ml[pr * 2] = top;
          part_ml[pr * 2 + 1] = sum;
        }
      }
    }
    if (!more) break;
    __syncthreads();
  }
}

// merges the partials of the pairs that runs cut, and writes the zeros of sequences
// without tokens.  One workgroup per query row of a pair or, by_cut (more pairs than
// runs), of a run: for the pair that begins in it and goes on behind it.  Groups of DH / 4
// threads over the partials, each with its own running maximum (one round of loads).
// Each of them works out the line, so fewer are better: both kernels, a workgroup for every
// pair / every run: 3000 pairs of 1 to 200 tokens (N 2112) 135 / 64 us, 4096 of 64 (N
// 4096) 114 / 74, 1024 of 4000 169.7 / 165.6; 64 of 4000 18.5 / 19.7
template <int DH>
__global__ __launch_bounds__(256) void k_kv8_combine(const float* __restrict__ part_ml, const float* __restrict__ part_o,
                                                     float* __restrict__ out, Seqs S, int nwg, int by_cut, int chunks,
                                                     int n_q, int G) {
  constexpr int NG = 256 / (DH / 4);
  const int gr = blockIdx.x, t = threadIdx.x, g = t / (DH / 4), d4 = t % (DH / 4);
  const int hq = S.hkv * G;
  auto row_of = [&](int b, int j) { return out + (((int64_t)b * n_q + gr / G) * hq + (int64_t)j * G + gr % G) * DH; };
  Order order(S);
  const int run = order.lay_out(nwg);
  int b = blockIdx.z, j = blockIdx.y, begin, tokens;
  if (by_cut) {
    const int w = blockIdx.y;
    if (S.lengths) {
      for (b = w; b < S.B; b += nwg) {
        if (S.tokens(b)) continue;
        for (int e = t; e < S.hkv * (DH / 4); e += 256)
          *reinterpret_cast<floatx4*>(row_of(b, e / (DH / 4)) + e % (DH / 4) * 4) = floatx4{0.f, 0.f, 0.f, 0.f};
      }
    }
    const int end = (w + 1) * run;
    if (end >= order.all) return;
    order.find(end - 1, b, begin, tokens);
    j = (end - 1 - begin) / order.length(blocks_of(tokens));
  } else {
    order.of(b, begin, tokens);
  }
  float* dst = row_of(b, j) + 4 * d4;
  const int T_b = blocks_of(tokens);
  if (T_b == 0) {
    if (g == 0) *reinterpret_cast<floatx4*>(dst) = floatx4{0.f, 0.f, 0.f, 0.f};
    return;
  }
  const int u0 = begin + j * order.length(T_b), u1 = u0 + T_b;
  const int w0 = u0 / run, w1 = (u1 - 1) / run;
  if (w0 == w1) return;                                         // finished by its run
  if (by_cut && w0 != (int)blockIdx.y) return;                  // it began in an earlier one
  const int chunk = gr / kKv8Rows, row = gr % kKv8Rows;
  float M = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int w = w0 + g; w <= w1; w += NG) {
    const int64_t pr = part_row(w == w0 ? 2 * w + 1 : 2 * w, chunks, chunk, row);
    const float m = part_ml[pr * 2], pl = part_ml[pr * 2 + 1];
    const floatx4 x = *reinterpret_cast<const floatx4*>(part_o + pr * DH + 4 * d4);
    const float to = fmaxf(M, m);
    // a partial without a maximum has sums of zero, or NaN, which stay
    const float a = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - to);
    const float c = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
    l = a * l + c * pl;
    o = a * o + c * x;
    M = to;
  }
  __shared__ floatx4 so[NG][DH / 4];
  __shared__ float sm[NG], sl[NG];
  so[g][d4] = o;
  if (d4 == 0) {
    sm[g] = M;
    sl[g] = l;
  }
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int i = 0; i < NG; ++i) M = fmaxf(M, sm[i]);
    l = 0.f;
    o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float a = sm[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm[i] - M);
      l += a * sl[i];
      o += a * so[i][d4];
    }
    const float r = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<floatx4*>(dst) = o * r;
  }
}

int row_chunks(const Problem& P, int n_q) { return (n_q * P.G + kKv8Rows - 1) / kKv8Rows; }
// workgroups over the query rows: two chunks each where there are two (against one each,
// query tokens of four heads over 120001 tokens: 5 59.8 / 66.9 us, 8 65.5 / 67.7, 12 102.5 / 101.8,
// 16 103 / 112, 32 179 / 195; fp32 ones, 8 74 / 84, 32 206 / 250)
int row_sets(const Problem& P, int n_q) { return (row_chunks(P, n_q) + 1) / 2; }
// a workgroup for each pair where the caches are short: its waves take 4 blocks each at
// most, 8 where the pairs fill half the chip, and nothing is left to merge.  One launch
// against two, in a graph: 512 tokens, 8 pairs 7.7 / 9.3 us; 1024 tokens, 8 pairs 10.8 / 9.4
// (but calls from Python, which pay for each launch, 11.0 / 13.1), 64 pairs 11.6 / 11.2, 128
// pairs 11.9 / 14.1; 2048 tokens, 8 pairs 17.9 / 10.1, 128 pairs 18.7 / 18.9, 512 pairs
// 47.6 / 48.7
bool one_workgroup_per_pair(const Problem& P, int sets, int64_t n_max) {
  const int64_t groups = (int64_t)P.B * P.hkv * sets;
  const int blocks = groups >= 128 ? 8 * kWaves : 4 * kWaves;
  return n_max <= (int64_t)blocks * kKv8Block && groups <= 1 << 23;   // workgroups of a grid
}
// a wave for each pair where there are enough of them to fill the chip and the caches are
// shorter still: nothing is merged, and the chip holds 2048 pairs at a time, not 512.  A
// wave's blocks come one after the other (512 tokens take 20 us), so longer ones only where
// there are many, or 32 query rows to merge.  Pairs count once for each set of rows.  In us, a
// workgroup / a wave per pair: 640 pairs of 512 tokens 22.5 / 20.7, 1024 of 200 22.4 / 15.1, of
// 512 32.1 / 25.4, of 1 to 512 23.0 / 21.0; 2048 of 1024 100 / 87; 8192 of 64 87 / 37, of 1024
// 411 / 357; nine query tokens over 1000, 1280 sets of rows 105 / 95, 4096 334 / 205.  The other
// way: 512 pairs of 512 16.6 / 20.1, 1024 of 1 to 2000 53.2 / 62.3
bool one_wave_per_pair(const Problem& P, int n_q, int64_t n_max) {
  const int64_t groups = (int64_t)P.B * P.hkv * row_sets(P, n_q);
  const int blocks = groups >= 2048 || row_chunks(P, n_q) > 1 ? 16 : 8;
  return groups >= 640 && n_max <= (int64_t)blocks * kKv8Block && one_workgroup_per_pair(P, row_sets(P, n_q), n_max);
}
// runs of a call over at most n_max tokens per sequence: a block for every wave at least
int runs(const Problem& P, int n_q, int64_t n_max) {
  const int64_t blocks = (int64_t)P.B * P.hkv * pair_length((int)((n_max + kKv8Block - 1) / kKv8Block), 1 << 30);
  return (int)std::max<int64_t>(1, std::min<int64_t>((blocks + kWaves - 1) / kWaves, kKv8Wgs / row_sets(P, n_q)));
}

}  // namespace

// (max, sum) and d_h sums for two slots per run, sixteen rows per chunk; what a call
// with fewer query tokens needs is inside
size_t kv8_ws_bytes(const Problem& P, int n_q) {
  size_t part_rows = 0;
  for (int n = 1; n <= n_q; ++n)
    part_rows = std::max(part_rows, (size_t)2 * runs(P, n, P.cap) * row_chunks(P, n) * kKv8Rows);
  return part_rows * (P.dh + 2) * sizeof(float);
}

hipError_t launch_kv8_decode(const Problem& P, const Kv8& C, int64_t n_max, const int32_t* lengths, int n_q,
                             const void* q, float* out, void* ws, hipStream_t st) {
  const int chunks = row_chunks(P, n_q), sets = row_sets(P, n_q);
  const bool by_pair = one_workgroup_per_pair(P, sets, n_max);
  const int nwg = by_pair ? P.B * P.hkv : runs(P, n_q, n_max);
  const size_t part_rows = (size_t)2 * nwg * chunks * kKv8Rows;
  float* part_o = (float*)ws;
  float* part_ml = part_o + part_rows * P.dh;
  const Seqs S{lengths, (int)n_max, P.B, P.hkv};
  const bool by_wave = one_wave_per_pair(P, n_q, n_max);
  const int wgs = by_wave ? (nwg + kWaves - 1) / kWaves : nwg;
  const dim3 grid((wgs + 7) / 8 * 8 * sets);
  auto go = [&](auto elem, auto fmt, auto dh) {
    using T = decltype(elem);
    auto with = [&](auto rc, auto share) {
      hipLaunchKernelGGL((k_kv8_decode<T, fmt(), dh(), rc(), share()>), grid, dim3(kWaves * 64), 0, st, (const T*)q, C.k_codes,
                         C.k_scales, C.v_codes, C.v_scales, part_ml, part_o, out, S, nwg, (int)by_pair, chunks, n_q,
                         P.G, kv8_tiles(P));
    };
    auto by_share = [&](auto rc) {
      if (by_wave)
        with(rc, std::integral_constant<int, 1>());
      else
        with(rc, std::integral_constant<int, kWaves>());
    };
    if (chunks == 1)
      by_share(std::integral_constant<int, 1>());
    else
      by_share(std::integral_constant<int, 2>());
  };
  auto by_fmt = [&](auto elem, auto dh) {
    if (C.format == S4R_KV_INT8)
      go(elem, std::integral_constant<int, S4R_KV_INT8>(), dh);
    else
      go(elem, std::integral_constant<int, S4R_KV_E4M3>(), dh);
  };
  auto by_type = [&](auto dh) {
    if (P.dtype == S4R_BF16)
      by_fmt(uint16_t(), dh);
    else
      by_fmt(float(), dh);
  };
  if (P.dh == 128)
    by_type(std::integral_constant<int, 128>());
  else
    by_type(std::integral_constant<int, 64>());
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || by_pair) return e;
  // sequences of one length: no pair is cut where the runs hold whole ones
  if (!lengths) {
    const int blocks = (int)((n_max + kKv8Block - 1) / kKv8Block), pairs = P.B * P.hkv;
    const int length = pair_length(blocks, (pair_length(blocks, 0) * pairs + nwg - 1) / nwg);
    if (run_length(length * pairs, nwg) % length == 0) return hipSuccess;
  }
  const bool by_cut = (int64_t)P.B * P.hkv > nwg;
  const dim3 cgrid(n_q * P.G, by_cut ? nwg : P.hkv, by_cut ? 1 : P.B);
  if (P.dh == 128)
    hipLaunchKernelGGL(k_kv8_combine<128>, cgrid, dim3(256), 0, st, part_ml, part_o, out, S, nwg, (int)by_cut, chunks, n_q,
                       P.G);
  else
    hipLaunchKernelGGL(k_kv8_combine<64>, cgrid, dim3(256), 0, st, part_ml, part_o, out, S, nwg, (int)by_cut, chunks, n_q,
                       P.G);
  return hipGetLastError();
}

}  // namespace s4r
