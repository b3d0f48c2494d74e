// One int4 group-64 projection with its unmerged adapter, for T rows (Sec. 2,
// Quantization; Sec. 3.3, Fig. 1):  y = W x + lora_scale B (A x),  W = s q + z.
//
// Per 64-input group g of an output row the products are summed as
//   y += s_g (q_g . x_g) + z_g sum(x_g):
// the codes q enter the matrix cores as exact fp16 numbers (q 2^-9, whose 2^9 goes
// into s), x is fp16, the sums are fp32 and s and z are applied in fp32, so that no
// weight is rounded.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "moe_linear.h"
#include "moe_tile.h"

namespace moe {
namespace {

constexpr int kCus = 256;
constexpr float kCodeUnit = 512.f;

// Eight codes (one dword, even input in the low nibble) as halves q 2^-9, in order: the
// nibble is the subnormal q 2^-24, times 2^15. (The matrix cores take the subnormals
// themselves too, but align their products to the smallest normal number's exponent:
// a group's sum then loses up to 10 of its bits, 1.2e-6 of a row against 1e-7.)
__device__ __forceinline__ h8 codes8(uint32_t w) {
  const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
  u4 v;
  v.x = __builtin_amdgcn_perm(hi, lo, 0x0C040C00u);
  v.y = __builtin_amdgcn_perm(hi, lo, 0x0C050C01u);
  v.z = __builtin_amdgcn_perm(hi, lo, 0x0C060C02u);
  v.w = __builtin_amdgcn_perm(hi, lo, 0x0C070C03u);
  return __builtin_bit_cast(h8, v) * (_Float16)32768.f;
}

__device__ __forceinline__ h8 ones8() {
  const _Float16 o = (_Float16)1.f;
  return h8{o, o, o, o, o, o, o, o};
}

__device__ __forceinline__ void store_out(const LinearArgs& a, int t, int o, float v) {
  const size_t at = (size_t)t * a.y_stride + o;
  if (a.y_type == MOE_OUT_F16)
    static_cast<__half*>(a.y)[at] = __float2half(v);
  else if (a.y_type == MOE_OUT_F32)
    static_cast<float*>(a.y)[at] = v;
  else
    static_cast<float*>(a.y)[at] += v;
}

// ---- few rows: the weights are read once, 16 NT output rows a workgroup --------
// The NW waves take quads of groups in turn (a 128-byte line of codes per output row)
// and their sums meet in LDS. A lane holds the codes of output row c = lane % 16,
// inputs 16 g .. + 15 of a group (g = lane / 16). sum(x_g) is the product with ones,
// and A x rides along as RT further tiles of 16 adapter rows, formed again by every
// workgroup (from L2) rather than by a launch of its own. Latency bounds it (one row, 6144 x
// 2048, rank 16: 7.4 MB in 8.0 us; 4096 x 4096, 13 rows: 10.0 MB in 11.4): every load of a
// run of groups, and B's, is asked for before the first product.
template <int TT, int RT, int NT, int NW>
__global__ void __launch_bounds__(64 * NW) linear_rows_kernel(LinearArgs a) {
  __shared__ float red[NW][TT * (NT + RT)][4][kWave];
  __shared__ float axs[RT ? TT * 16 : 1][RT ? RT * 16 + 1 : 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int ng = a.in_dim >> 6, t0 = blockIdx.y * TT * 16, o0 = blockIdx.x * NT * 16;
  const char* q[NT];
  const __half2* sz[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const size_t row = min(o0 + 16 * n + c, a.out_dim - 1);
    q[n] = static_cast<const char*>(a.q) + row * (a.in_dim / 2) + 8 * g;
    sz[n] = static_cast<const __half2*>(a.sz) + row * ng;
  }
  const _Float16* x[TT];
#pragma unroll
  for (int m = 0; m < TT; ++m)  // (a row past T repeats the last one and is not stored)
    x[m] = static_cast<const _Float16*>(a.x) + (size_t)min(t0 + 16 * m + c, a.T - 1) * a.x_stride + 16 * g;
  const _Float16* ad[RT ? RT : 1];
#pragma unroll
  for (int n = 0; n < RT; ++n)
    ad[n] = static_cast<const _Float16*>(a.lora_a) + (size_t)min(16 * n + c, a.r - 1) * a.in_dim + 16 * g;
  // this thread's first output, for the adapter's B
  constexpr int OUTS = TT * NT * 256;
  auto output = [&](int e, int& tl, int& o) {  // output e: its row of the tile and its column
    const int l = e & 63, i = (e >> 6) & 3, tile = e >> 8;
    tl = 16 * (tile / NT) + 4 * (l >> 4) + i;
    o = o0 + 16 * (tile % NT) + (l & 15);
  };
  h8 lb[2] = {};
  const bool early = RT == 1 && (a.r == 8 || a.r == 16);
  if (early) {
    int tl, o;
    output(min((int)threadIdx.x, OUTS - 1), tl, o);
    const _Float16* p = static_cast<const _Float16*>(a.lora_b) + (size_t)min(o, a.out_dim - 1) * a.r;
    lb[0] = ld_h8(p);
    if (a.r == 16) lb[1] = ld_h8(p + 8);
  }
  f4 y[TT][NT] = {}, ax[TT][RT ? RT : 1] = {};
  const h8 one = ones8();
  auto groups = [&](int g0, auto count) {      // N groups from g0 on
    constexpr int N = decltype(count)::value;
    u2 w[N][NT];
    float2 s[N][NT];
    h8 x0[N][TT], x1[N][TT], b0[N][RT ? RT : 1], b1[N][RT ? RT : 1];
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        w[k][n] = *reinterpret_cast<const u2*>(q[n] + 32 * (g0 + k));
        s[k][n] = __half22float2(sz[n][g0 + k]);
      }
#pragma unroll
      for (int m = 0; m < TT; ++m) {
        x0[k][m] = ld_h8(x[m] + 64 * (g0 + k));
        x1[k][m] = ld_h8(x[m] + 64 * (g0 + k) + 8);
      }
#pragma unroll
      for (int n = 0; n < RT; ++n) {
        b0[k][n] = ld_h8(ad[n] + 64 * (g0 + k));
        b1[k][n] = ld_h8(ad[n] + 64 * (g0 + k) + 8);
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int m = 0; m < TT; ++m) {
        const f4 xs = mfma16(x1[k][m], one, mfma16(x0[k][m], one, f4{}));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const h8 w0 = codes8(w[k][n].x), w1 = codes8(w[k][n].y);
          const f4 d = mfma16(x1[k][m], w1, mfma16(x0[k][m], w0, f4{}));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y[m][n][i] = fmaf(s[k][n].x * kCodeUnit, d[i], fmaf(s[k][n].y, xs[i], y[m][n][i]));
        }
#pragma unroll
        for (int n = 0; n < RT; ++n) ax[m][n] = mfma16(x1[k][m], b1[k][n], mfma16(x0[k][m], b0[k][n], ax[m][n]));
      }
  };
  // (registers of a group: 4 for each tile of outputs, 8 for each of x and A)
  constexpr int PER = 4 * NT + 8 * TT + 8 * RT, N = PER <= 24 ? 4 : PER <= 40 ? 2 : 1;
  for (int quad = wave; quad * 4 < ng; quad += NW) {
    const int end = min(quad * 4 + 4, ng);
    int gi = quad * 4;
    for (; gi + N <= end; gi += N) groups(gi, std::integral_constant<int, N>());
    if constexpr (N > 1)
      for (; gi < end; ++gi) groups(gi, std::integral_constant<int, 1>());
  }
#pragma unroll
  for (int m = 0; m < TT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int n = 0; n < NT; ++n) red[wave][m * NT + n][i][lane] = y[m][n][i];
#pragma unroll
      for (int n = 0; n < RT; ++n) red[wave][TT * NT + m * RT + n][i][lane] = ax[m][n][i];
    }
  __syncthreads();
  auto total = [&](int tile, int i, int l) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += red[w][tile][i][l];
    return v;
  };
  if constexpr (RT > 0) {
    for (int e = threadIdx.x; e < TT * RT * 256; e += 64 * NW) {
      const int l = e & 63, i = (e >> 6) & 3, tile = e >> 8;
      axs[16 * (tile / RT) + 4 * (l >> 4) + i][16 * (tile % RT) + (l & 15)] = total(TT * NT + tile, i, l);
    }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < OUTS; e += 64 * NW) {
    int tl, o;
    output(e, tl, o);
    if (t0 + tl >= a.T || o >= a.out_dim) continue;
    float v = total(e >> 8, (e >> 6) & 3, e & 63);
    if constexpr (RT > 0) {
      float delta = 0.f;
      if (early && e == (int)threadIdx.x) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < a.r) delta = fmaf((float)lb[k / 8][k % 8], axs[tl][k], delta);
      } else {
        const _Float16* p = static_cast<const _Float16*>(a.lora_b) + (size_t)o * a.r;
        for (int k = 0; k < a.r; ++k) delta = fmaf((float)p[k], axs[tl][k], delta);
      }
      v = fmaf(a.lora_scale, delta, v);
    }
    store_out(a, t0 + tl, o, v);
  }
}

// ---- many rows -------------------------------------------------------------------
// What multiplies z and B is small: per row the group sums of x and lora_scale A x.
// One launch forms them (16 rows a workgroup) as E [T][KE] = (group sums, zeros to a
// multiple of 32, lora_scale A x, zeros), scaled per row by a power of two to less than
// 2^15 and split into two halves, hi + lo (22 bits of each number down to 2^-18 of the row's
// largest, and 2^-39 of that below): the tile products then add them as KE more inputs whose
// weights z and B are exact in fp16.
// Bound by latency, few workgroups for x's reads: 1,555 rows of 4,096, rank 16 (13 MB), 10 us.
template <int RT>
__global__ void __launch_bounds__(512) linear_sums_kernel(LinearArgs a) {
  constexpr int NW = 8;
  extern __shared__ float es[];                         // [16][KE]
  __shared__ float red[NW][RT ? RT : 1][4][kWave];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int ng = a.in_dim >> 6, KE = linear_extra(a.in_dim, a.r), az = (ng + 31) / 32 * 32;
  const int t0 = blockIdx.x * 16;
  for (int e = threadIdx.x; e < 16 * KE; e += 512) es[e] = 0.f;
  __syncthreads();
  const _Float16* x = static_cast<const _Float16*>(a.x) + (size_t)min(t0 + c, a.T - 1) * a.x_stride + 8 * g;
  const _Float16* ad[RT ? RT : 1];
#pragma unroll
  for (int n = 0; n < RT; ++n)
    ad[n] = static_cast<const _Float16*>(a.lora_a) + (size_t)min(16 * n + c, a.r - 1) * a.in_dim + 8 * g;
  f4 ax[RT ? RT : 1] = {};
  const h8 one = ones8();
  auto groups = [&](int g0, auto count) {                // N groups, NW apart, asked for at once
    constexpr int N = decltype(count)::value;
    h8 x0[N], x1[N], b0[N][RT ? RT : 1], b1[N][RT ? RT : 1];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int gi = g0 + NW * k;
      x0[k] = ld_h8(x + 64 * gi);
      x1[k] = ld_h8(x + 64 * gi + 32);
#pragma unroll
      for (int n = 0; n < RT; ++n) {
        b0[k][n] = ld_h8(ad[n] + 64 * gi);
        b1[k][n] = ld_h8(ad[n] + 64 * gi + 32);
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const f4 xs = mfma16(x1[k], one, mfma16(x0[k], one, f4{}));
      if (c == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) es[(4 * g + i) * KE + g0 + NW * k] = xs[i];
#pragma unroll
      for (int n = 0; n < RT; ++n) ax[n] = mfma16(x1[k], b1[k][n], mfma16(x0[k], b0[k][n], ax[n]));
    }
  };
  constexpr int N = RT <= 1 ? 4 : 2;
  int gi = wave;
  for (; gi + (N - 1) * NW < ng; gi += N * NW) groups(gi, std::integral_constant<int, N>());
  for (; gi < ng; gi += NW) groups(gi, std::integral_constant<int, 1>());
  if constexpr (RT > 0) {
#pragma unroll
    for (int n = 0; n < RT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][n][i][lane] = ax[n][i];
    __syncthreads();
    for (int e = threadIdx.x; e < RT * 256; e += 512) {
      const int l = e & 63, i = (e >> 6) & 3, n = e >> 8, k = 16 * n + (l & 15);
      if (k >= a.r) continue;
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) v += red[w][n][i][l];
      es[(4 * (l >> 4) + i) * KE + az + k] = a.lora_scale * v;
    }
  }
  __syncthreads();
  for (int k = 0; k < 2; ++k) {                         // two rows a wave
    const int t = 2 * wave + k;
    if (t0 + t >= a.T) break;
    const float* e = es + t * KE;
    float top = 0.f;
    for (int j = lane; j < KE; j += kWave) top = fmaxf(top, fabsf(e[j]));
    top = __uint_as_float(wave_max_u32(__float_as_uint(top)));  // (of numbers >= 0)
    const int ex = top > 0.f && top < INFINITY ? max(ilogbf(top), -86) - 14 : 0;
    for (int j = lane; j < KE; j += kWave) {
      const float v = ldexpf(e[j], -ex);
      const _Float16 hi = (_Float16)v;
      const size_t at = (size_t)(t0 + t) * KE + j;
      a.e_hi[at] = __builtin_bit_cast(__half, hi);
      a.e_lo[at] = __float2half(v - (float)hi);
    }
    if (lane == 0) a.e_scale[t0 + t] = ldexpf(1.f, ex);
  }
}

// XOR key of a 128-byte row (8 pieces of 16 bytes) whose pieces 2 g + u a lane reads:
// the 16 pieces that a quarter of a b128 read touches lie on all banks (see tile_key).
__device__ __forceinline__ int x_key(int row) { return ((row >> 1) & 1) | ((row >> 1) & 4); }

// The products on the matrix cores: 128 rows of x by 128 outputs, four waves of 64 x 64,
// one 64-input group a step. x, codes and (s, z) come through LDS, two steps ahead in three
// slots. Bound by three pipes that overlap in part: a step of a CU's two workgroups reads 88 KB
// of LDS and has 41 KB copied in (about 1,200 clocks), unpacks codes and applies scales (1,100 a
// SIMD) and has 64 products a SIMD (1,030), and takes 2,600. 1,555 rows, 5001 x 4096, rank 16:
// 109 us, 0.59 PFLOP/s.
// Workgroups come in rounds of kSlots. The tiles that do not fill a round are split along
// the inputs into as many parts as fill it (first in the grid, so that whole tiles follow
// the short parts); a part writes fp32 sums, which one more launch adds in order.
struct TilePlan {
  int cols, tiles, rest, parts;   // tiles of a row block, all tiles; of them split, and into how many parts
  int workgroups() const { return tiles - rest + rest * parts; }
};
constexpr int kSlots = 512, kMostParts = 16, kTileSums = 128 * 128;
static_assert(kSlots * kTileSums * sizeof(float) <= kLinearSums, "parts fit the workspace");

TilePlan tile_plan(int out_dim, int T, int ng) {
  TilePlan p{};
  p.cols = (out_dim + 127) / 128;
  p.tiles = p.cols * ((T + 127) / 128);
  p.rest = p.tiles % kSlots;
  p.parts = p.rest ? std::min({kSlots / p.rest, kMostParts, std::max(1, ng / 4)}) : 1;
  if (p.parts < 2) p.rest = 0, p.parts = 1;
  return p;
}

__global__ void __launch_bounds__(256, 2) linear_tile_kernel(LinearArgs a, TilePlan p) {
  constexpr int XB = 128 * 128, CB = 128 * 32, SB = 128 * 4, SLOT = XB + CB + SB;
  __shared__ __attribute__((aligned(16))) char ring[3][SLOT];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4, ng = a.in_dim >> 6;
  const int split = p.rest * p.parts;
  int tile = blockIdx.x - split + p.rest, part = 0, from = 0, to = ng;
  if ((int)blockIdx.x < split) {
    tile = blockIdx.x / p.parts;
    part = blockIdx.x % p.parts;
    from = ng * part / p.parts;
    to = ng * (part + 1) / p.parts;
  }
  const int t0 = tile / p.cols * 128, o0 = tile % p.cols * 128;
  const int tw = (wave & 1) * 64, nw = (wave >> 1) * 64, ow = o0 + nw;
  const char* xs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 8 * (4 * wave + j) + (lane >> 3);
    xs[j] = static_cast<const char*>(a.x) + (size_t)min(t0 + r, a.T - 1) * a.x_stride * 2 + 16 * ((lane & 7) ^ x_key(r));
  }
  // codes: 32 rows of two pieces a copy, a row's pieces swapped in every other four rows
  const int cr = 32 * wave + (lane >> 1);
  const char* cs = static_cast<const char*>(a.q) + (size_t)min(o0 + cr, a.out_dim - 1) * (a.in_dim / 2) +
                   16 * ((lane & 1) ^ (cr >> 2 & 1));
  const uint32_t* ss = static_cast<const uint32_t*>(a.sz) + (size_t)min(o0 + 64 * (wave & 1) + lane, a.out_dim - 1) * ng;
  const uint32_t at0 = lds_at(ring);
  auto copy = [&](int gi, int slot) {
    const uint32_t at = at0 + slot * SLOT;
#pragma unroll
    for (int j = 0; j < 4; ++j) dma16(xs[j] + 128 * (size_t)gi, at + 1024 * (4 * wave + j));
    dma16(cs + 32 * (size_t)gi, at + XB + 1024 * wave);
    dma4(ss + gi, at + XB + CB + 256 * (wave & 1));      // (two waves each write the same scales)
  };
  constexpr int kCopies = 6;
  copy(from, 0);
  if (from + 1 < to) copy(from + 1, 1);
  f4 y[4][4] = {};
  // first the group sums by z and lora_scale A x by B, which the sums then start from
  const int KE = part ? 0 : linear_extra(a.in_dim, a.r), az = (ng + 31) / 32 * 32;
  for (int k = 0; k < KE; k += 32) {
    h8 w[4];                                             // (past the groups or the rank: any weight, times E's zero)
    const int j = k + 8 * g;
    if (k < az) {
      // 32 (s, z) of each output through the last slot, two rows a copy, keyed like x
      char* zt = ring[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 2 * (16 * wave + i) + (lane >> 5), d = (lane & 31) ^ (4 * x_key(r));
        const size_t row = min(o0 + r, a.out_dim - 1);
        dma4(static_cast<const uint32_t*>(a.sz) + row * ng + min(k + d, ng - 1), at0 + 2 * SLOT + 256 * (16 * wave + i));
      }
      vm_wait<0>();
      lds_barrier();
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int r = nw + 16 * n + c;
        const u4 lo = *reinterpret_cast<const u4*>(zt + 128 * r + 16 * ((2 * g) ^ x_key(r)));
        const u4 hi = *reinterpret_cast<const u4*>(zt + 128 * r + 16 * ((2 * g + 1) ^ x_key(r)));
        // the upper halves
        const u4 z = {__builtin_amdgcn_perm(lo.y, lo.x, 0x07060302u), __builtin_amdgcn_perm(lo.w, lo.z, 0x07060302u),
                      __builtin_amdgcn_perm(hi.y, hi.x, 0x07060302u), __builtin_amdgcn_perm(hi.w, hi.z, 0x07060302u)};
        w[n] = __builtin_bit_cast(h8, z);
      }
      lds_barrier();
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const _Float16* lb = static_cast<const _Float16*>(a.lora_b) + (size_t)min(ow + 16 * n + c, a.out_dim - 1) * a.r;
        if (a.r % 8 == 0)
          w[n] = ld_h8(lb + min(j - az, a.r - 8));
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) w[n][e] = lb[min(j + e - az, a.r - 1)];
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const size_t at = (size_t)min(t0 + tw + 16 * m + c, a.T - 1) * KE + j;
      const h8 hi = ld_h8(a.e_hi + at), lo = ld_h8(a.e_lo + at);
#pragma unroll
      for (int n = 0; n < 4; ++n) y[m][n] = mfma16(lo, w[n], mfma16(hi, w[n], y[m][n]));
    }
  }
  if (KE)
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f4 es = *reinterpret_cast<const f4*>(a.e_scale + t0 + tw + 16 * m + 4 * g);  // (rows past T: not stored)
#pragma unroll
      for (int n = 0; n < 4; ++n) y[m][n] *= es;
    }
  vm_drain();
  int slot = 0;
  for (int gi = from; gi < to; ++gi) {
    if (gi + 1 < to)
      vm_wait<kCopies>();
    else
      vm_wait<0>();
    lds_barrier();
    if (gi + 2 < to) copy(gi + 2, slot >= 1 ? slot - 1 : 2);
    const char* xt = ring[slot];
    const char* codes = xt + XB;
    const uint32_t* scales = reinterpret_cast<const uint32_t*>(codes + CB);
    h8 b0[4], b1[4];
    float s[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int r = nw + 16 * n + c;
      const u2 w = *reinterpret_cast<const u2*>(codes + 32 * r + 16 * ((g >> 1) ^ (r >> 2 & 1)) + 8 * (g & 1));
      b0[n] = codes8(w.x);
      b1[n] = codes8(w.y);
      s[n] = __low2float(__builtin_bit_cast(__half2, scales[r])) * kCodeUnit;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int r = tw + 16 * m + c;
      const h8 x0 = ld_h8(xt + 128 * r + 16 * ((2 * g) ^ x_key(r)));
      const h8 x1 = ld_h8(xt + 128 * r + 16 * ((2 * g + 1) ^ x_key(r)));
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const f4 d = mfma16(x1, b1[n], mfma16(x0, b0[n], f4{}));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[m][n][i] = fmaf(s[n], d[i], y[m][n][i]);
      }
    }
    slot = slot == 2 ? 0 : slot + 1;
  }
  if ((int)blockIdx.x < split) {
    // a tile's sums as the lanes hold them: [m][n] of each wave, four rows a lane
    float* sums = a.sums + (size_t)blockIdx.x * kTileSums + threadIdx.x * 4;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int n = 0; n < 4; ++n) *reinterpret_cast<f4*>(sums + (4 * m + n) * 1024) = y[m][n];
    return;
  }
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + tw + 16 * m + 4 * g + i, o = ow + 16 * n + c;
        if (t < a.T && o < a.out_dim) store_out(a, t, o, y[m][n][i]);
      }
}

// The parts of the split tiles, added in order: one of a tile's sixteen [m][n] a workgroup
// (8 tiles of 16 parts: 4.8 us). Without splitting, 520 tiles took two rounds of 512
// (1,555 rows as above, the call: 174 us, 123 with this and the sums' loads batched).
__global__ void __launch_bounds__(256) linear_parts_kernel(LinearArgs a, TilePlan p) {
  const int tile = blockIdx.x / 16, mn = blockIdx.x % 16;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float* sums = a.sums + (size_t)tile * p.parts * kTileSums + mn * 1024 + threadIdx.x * 4;
  f4 y = {};
#pragma unroll 8
  for (int k = 0; k < p.parts; ++k) y += *reinterpret_cast<const f4*>(sums + (size_t)k * kTileSums);
  const int t0 = tile / p.cols * 128 + (wave & 1) * 64 + 16 * (mn >> 2) + 4 * (lane >> 4);
  const int o = tile % p.cols * 128 + (wave >> 1) * 64 + 16 * (mn & 3) + (lane & 15);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + i < a.T && o < a.out_dim) store_out(a, t0 + i, o, y[i]);
}

template <int TT, int RT, int NT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const dim3 grid((a.out_dim + 16 * NT - 1) / (16 * NT), (a.T + 16 * TT - 1) / (16 * TT));
  hipLaunchKernelGGL((linear_rows_kernel<TT, RT, NT, 8>), grid, dim3(512), 0, st, a);
  return hipGetLastError();
}
template <int TT, int NT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  if (a.r == 0) return launch_rows<TT, 0, NT>(a, st);
  if (a.r <= 16) return launch_rows<TT, 1, NT>(a, st);
  return launch_rows<TT, 4, NT>(a, st);
}

// E of 16 rows lies beside the partial sums of A x, which above rank 16 take half of the 64 KB
// that a launch has without being asked (68 KB at the most inputs and adapter rows).
template <int RT>
hipError_t launch_sums(const LinearArgs& a, hipStream_t st) {
  auto kernel = linear_sums_kernel<RT>;
  if constexpr (RT > 1) {
    constexpr int most = 16 * linear_extra(kMostIn, kMostRank) * sizeof(float);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != hipSuccess) return e;
  }
  const size_t lds = 16 * (size_t)linear_extra(a.in_dim, a.r) * sizeof(float);
  hipLaunchKernelGGL(kernel, dim3((a.T + 15) / 16), dim3(512), lds, st, a);
  return hipGetLastError();
}

// 32 outputs a workgroup where 16 would give more workgroups than CUs: half the reads of x
// and A (one row, 6144 x 2048, rank 16: 8.2 against 10.4 us; 8192 x 8192: 24 against 30;
// 64 rows, 4096 x 4096: 21 against 30), 16 below, for the CUs (4096 x 2048: 6.8 against 7.9).
template <int TT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const int64_t groups = (int64_t)((a.out_dim + 15) / 16) * ((a.T + 16 * TT - 1) / (16 * TT));
  return groups > kCus ? launch_rows<TT, 2>(a, st) : launch_rows<TT, 1>(a, st);
}

}  // namespace

// The rows kernel as long as its workgroups (32 outputs by 32 rows) are on the CUs at once,
// or twice that where the inputs are few: it has one launch and reads the weights once per
// 32 rows, from L2 after the first time. Against the tiles, us: 64 rows 4096 x 4096, rank 32
// (256 workgroups) 27 : 40, 80 rows (384) 49 : 40; 8192 x 8192, 32 rows (256) 38 : 58, 64
// rows (512) 73 : 60; 6144 x 2048, 64 rows (384) 22 : 27, 80 rows (576) 29 : 27; 640 x 2048,
// 192 rows (120) 9.5 : 19.
bool linear_by_rows(int out_dim, int in_dim, int T) {
  const int64_t groups = (int64_t)((out_dim + 31) / 32) * ((T + 31) / 32);
  return T <= 16 || (T <= kRowsMost && groups <= (in_dim <= 2048 ? 2 : 1) * kCus);
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  if (a.T <= 16) return launch_rows<1>(a, st);
  if (linear_by_rows(a.out_dim, a.in_dim, a.T)) return launch_rows<2>(a, st);
  hipError_t e = a.r == 0 ? launch_sums<0>(a, st) : a.r <= 16 ? launch_sums<1>(a, st) : launch_sums<4>(a, st);
  if (e != hipSuccess) return e;
  const TilePlan p = tile_plan(a.out_dim, a.T, a.in_dim / 64);
  hipLaunchKernelGGL(linear_tile_kernel, dim3(p.workgroups()), dim3(256), 0, st, a, p);
  e = hipGetLastError();
  if (e != hipSuccess || !p.rest) return e;
  hipLaunchKernelGGL(linear_parts_kernel, dim3(16 * p.rest), dim3(256), 0, st, a, p);
  return hipGetLastError();
}

}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {

constexpr int kMaxOut = 1 << 20, kMaxRows = 1 << 20;
constexpr int64_t kMaxOutputs = int64_t(1) << 37;      // (a grid's threads: 2^24 tiles of 128 x 128, 256 each)

bool linear_shape_ok(int out_dim, int in_dim, int rank, int T) {
  return out_dim >= 1 && out_dim <= kMaxOut && in_dim >= 64 && in_dim <= moe::kMostIn && in_dim % 64 == 0 &&
         rank >= 0 && rank <= moe::kMostRank && T >= 0 && T <= kMaxRows && (int64_t)T * out_dim <= kMaxOutputs;
}
size_t round256(size_t v) { return (v + 255) / 256 * 256; }
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace

extern "C" {

size_t moe_linear_workspace_bytes(int out_dim, int in_dim, int rank, int T) {
  if (!linear_shape_ok(out_dim, in_dim, rank, T)) return 0;
  const size_t t = T < 1 ? 1 : T, ke = moe::linear_extra(in_dim, rank);
  const size_t sums = moe::linear_by_rows(out_dim, in_dim, T) ? 0 : (size_t)moe::kLinearSums;
  return 2 * round256(t * ke * 2) + round256(t * 4) + sums;
}

int moe_linear_int4_lora(const moe_proj* w, int out_dim, int in_dim, int rank, float lora_scale,
                         const void* x_f16, int64_t x_stride, int T, void* y, int y_type,
                         int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!w || !linear_shape_ok(out_dim, in_dim, rank, T)) return MOE_EINVAL;
  if (y_type != MOE_OUT_F32 && y_type != MOE_OUT_F16 && y_type != MOE_OUT_F32_ADD) return MOE_EINVAL;
  if (!(lora_scale == lora_scale)) return MOE_EINVAL;
  if (x_stride < in_dim || x_stride % 8 || y_stride < out_dim || x_stride > (int64_t(1) << 40) ||
      y_stride > (int64_t(1) << 40))
    return MOE_EINVAL;
  const bool lora = w->lora_a && w->lora_b;
  if (lora && rank < 1) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!w->q || !w->sz || !x_f16 || !y || !workspace) return MOE_EINVAL;
  if (misaligned(w->q, 16) || misaligned(w->sz, 16) || misaligned(x_f16, 16) || misaligned(y, 16) ||
      misaligned(workspace, 16) || (lora && (misaligned(w->lora_a, 16) || misaligned(w->lora_b, 16))))
    return MOE_EALIGN;
  if (workspace_bytes < moe_linear_workspace_bytes(out_dim, in_dim, lora ? rank : 0, T)) return MOE_ENOMEM;
  moe::LinearArgs a{};
  a.q = w->q;
  a.sz = w->sz;
  a.lora_a = lora ? w->lora_a : nullptr;
  a.lora_b = lora ? w->lora_b : nullptr;
  a.out_dim = out_dim;
  a.in_dim = in_dim;
  a.r = lora ? rank : 0;
  a.lora_scale = lora_scale;
  a.x = x_f16;
  a.x_stride = x_stride;
  a.T = T;
  a.y = y;
  a.y_type = y_type;
  a.y_stride = y_stride;
  const size_t part = round256((size_t)T * moe::linear_extra(in_dim, a.r) * 2);
  a.e_hi = static_cast<__half*>(workspace);
  a.e_lo = reinterpret_cast<__half*>(static_cast<char*>(workspace) + part);
  a.e_scale = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * part);
  a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * part + round256((size_t)T * 4));
  return moe::launch_linear(a, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
