// One int4 group-64 projection with its unmerged adapter, for T rows (Sec. 2,
// Quantization; Sec. 3.3, Fig. 1):  y = W x + lora_scale B (A x),  W = s q + z.
//
// Per 64-input group g of an output row the products are summed as
//   y += s_g (q_g . x_g) + z_g sum(x_g):
// the codes q enter the matrix cores as exact fp16 numbers (q 2^-9, whose 2^9 goes
// into s), x is fp16, the sums are fp32 and s and z are applied in fp32, so that no
// weight is rounded.
#include <hip/hip_runtime.h>

#include "moe_linear.h"
#include "moe_tile.h"

namespace moe {
namespace {

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

// ---- few rows: the weights are read once, 16 output rows a workgroup -----------
// The NW waves take quads of groups in turn (a 128-byte line of codes per output row)
// and their sums meet in LDS. A lane holds the codes of output row c = lane % 16,
// inputs 16 g .. + 15 of a group (g = lane / 16). sum(x_g) is the product with ones,
// and A x rides along as RT further tiles of 16 adapter rows, formed again by every
// workgroup (from L2) rather than by a launch of its own.
template <int TT, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) linear_rows_kernel(LinearArgs a) {
  __shared__ float red[NW][TT * (1 + RT)][4][kWave];
  __shared__ float axs[RT ? TT * 16 : 1][RT ? RT * 16 + 1 : 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int ng = a.in_dim >> 6, t0 = blockIdx.y * TT * 16;
  const int row = min((int)blockIdx.x * 16 + c, a.out_dim - 1);
  const char* q = static_cast<const char*>(a.q) + (size_t)row * (a.in_dim / 2) + 8 * g;
  const __half2* sz = static_cast<const __half2*>(a.sz) + (size_t)row * ng;
  const _Float16* x[TT];
#pragma unroll
  for (int m = 0; m < TT; ++m)  // (a row past T repeats the last one and is not stored)
    x[m] = static_cast<const _Float16*>(a.x) + (size_t)min(t0 + 16 * m + c, a.T - 1) * a.x_stride + 16 * g;
  const _Float16* ad[RT ? RT : 1];
#pragma unroll
  for (int n = 0; n < RT; ++n)
    ad[n] = static_cast<const _Float16*>(a.lora_a) + (size_t)min(16 * n + c, a.r - 1) * a.in_dim + 16 * g;
  f4 y[TT] = {}, ax[TT][RT ? RT : 1] = {};
  const h8 one = ones8();
  for (int quad = wave; quad * 4 < ng; quad += NW) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int gi = quad * 4 + k;
      if (gi >= ng) break;
      const u2 w = *reinterpret_cast<const u2*>(q + 32 * gi);
      const float2 s = __half22float2(sz[gi]);
      const h8 w0 = codes8(w.x), w1 = codes8(w.y);
      h8 b0[RT ? RT : 1], b1[RT ? RT : 1];
#pragma unroll
      for (int n = 0; n < RT; ++n) {
        b0[n] = ld_h8(ad[n] + 64 * gi);
        b1[n] = ld_h8(ad[n] + 64 * gi + 8);
      }
#pragma unroll
      for (int m = 0; m < TT; ++m) {
        const h8 x0 = ld_h8(x[m] + 64 * gi), x1 = ld_h8(x[m] + 64 * gi + 8);
        const f4 d = mfma16(x1, w1, mfma16(x0, w0, f4{}));
        const f4 xs = mfma16(x1, one, mfma16(x0, one, f4{}));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[m][i] = fmaf(s.x * kCodeUnit, d[i], fmaf(s.y, xs[i], y[m][i]));
#pragma unroll
        for (int n = 0; n < RT; ++n) ax[m][n] = mfma16(x1, b1[n], mfma16(x0, b0[n], ax[m][n]));
      }
    }
  }
#pragma unroll
  for (int m = 0; m < TT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      red[wave][m][i][lane] = y[m][i];
#pragma unroll
      for (int n = 0; n < RT; ++n) red[wave][TT + m * RT + n][i][lane] = ax[m][n][i];
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
      axs[16 * (tile / RT) + 4 * (l >> 4) + i][16 * (tile % RT) + (l & 15)] = total(TT + tile, i, l);
    }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < TT * 256; e += 64 * NW) {
    const int l = e & 63, i = (e >> 6) & 3, m = e >> 8;
    const int tl = 16 * m + 4 * (l >> 4) + i, t = t0 + tl, o = blockIdx.x * 16 + (l & 15);
    if (t >= a.T || o >= a.out_dim) continue;
    float v = total(m, i, l);
    if constexpr (RT > 0) {
      const __half* lb = static_cast<const __half*>(a.lora_b) + (size_t)o * a.r;
      float delta = 0.f;
      for (int k = 0; k < a.r; ++k) delta = fmaf(__half2float(lb[k]), axs[tl][k], delta);
      v = fmaf(a.lora_scale, delta, v);
    }
    store_out(a, t, o, v);
  }
}

// ---- many rows -------------------------------------------------------------------
// What multiplies z and B is small: per row the group sums of x and lora_scale A x.
// One launch forms them (16 rows a workgroup) as E [T][KE] = (group sums, zeros to a
// multiple of 32, lora_scale A x, zeros), scaled per row by a power of two to at most
// 2 and split into two halves, hi + lo (22 bits of the row's largest): the tile
// products then add them as KE more inputs whose weights z and B are exact in fp16.
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
  const _Float16* x = static_cast<const _Float16*>(a.x) + (size_t)min(t0 + c, a.T - 1) * a.x_stride + 16 * g;
  const _Float16* ad[RT ? RT : 1];
#pragma unroll
  for (int n = 0; n < RT; ++n)
    ad[n] = static_cast<const _Float16*>(a.lora_a) + (size_t)min(16 * n + c, a.r - 1) * a.in_dim + 16 * g;
  f4 ax[RT ? RT : 1] = {};
  const h8 one = ones8();
  for (int gi = wave; gi < ng; gi += NW) {
    const h8 x0 = ld_h8(x + 64 * gi), x1 = ld_h8(x + 64 * gi + 8);
    const f4 xs = mfma16(x1, one, mfma16(x0, one, f4{}));
    if (c == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) es[(4 * g + i) * KE + gi] = xs[i];
#pragma unroll
    for (int n = 0; n < RT; ++n)
      ax[n] = mfma16(x1, ld_h8(ad[n] + 64 * gi + 8), mfma16(x0, ld_h8(ad[n] + 64 * gi), ax[n]));
  }
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
    const int ex = top > 0.f && top < INFINITY ? max(ilogbf(top), -100) : 0;
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
// one 64-input group a step. x comes through LDS one step ahead, codes and (s, z) one run
// of four groups ahead (a 128-byte line of codes per output). Bound by the VALU beside the
// matrix cores: a wave's 32 products a step (512 clocks) come with 88 instructions to
// unpack codes and 64 to apply scales.
constexpr int kRun = 4;                                  // groups of a run
__global__ void __launch_bounds__(256, 2) linear_tile_kernel(LinearArgs a) {
  __shared__ __attribute__((aligned(16))) char xt[2][128 * 128];
  __shared__ __attribute__((aligned(16))) char ct[2][128 * 32 * kRun];
  __shared__ uint32_t st[2][kRun][128];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4, ng = a.in_dim >> 6;
  const int t0 = blockIdx.y * 128, o0 = blockIdx.x * 128;
  const int tw = (wave & 1) * 64, nw = (wave >> 1) * 64, ow = o0 + nw;
  const uint32_t x_at = lds_at(xt), c_at = lds_at(ct), s_at = lds_at(st);
  const char *xs[4], *cs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 8 * (4 * wave + j) + (lane >> 3);
    xs[j] = static_cast<const char*>(a.x) + (size_t)min(t0 + r, a.T - 1) * a.x_stride * 2 + 16 * ((lane & 7) ^ x_key(r));
    cs[j] = static_cast<const char*>(a.q) + (size_t)min(o0 + r, a.out_dim - 1) * (a.in_dim / 2);
  }
  const int piece = (lane & 7) ^ (lane >> 4 & 7);        // of a line of codes: its key is row / 2, of 8 rows a copy
  auto copy_x = [&](int gi) {
#pragma unroll
    for (int j = 0; j < 4; ++j) dma16(xs[j] + 128 * (size_t)gi, x_at + (gi & 1) * 16384 + 1024 * (4 * wave + j));
  };
  // (pieces past a row's end, in its last run, are the row's first one again; not used)
  auto copy_run = [&](int run) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = piece ^ (4 * (j & 1));
      const int at = kRun * 32 * run + 16 * p;
      dma16(cs[j] + (at < a.in_dim / 2 ? at : 0), c_at + (run & 1) * 16384 + 1024 * (4 * wave + j));
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = min(o0 + 64 * j + lane, a.out_dim - 1), gi = min(kRun * run + wave, ng - 1);
      dma4(static_cast<const uint32_t*>(a.sz) + (size_t)row * ng + gi, s_at + (run & 1) * kRun * 512 + wave * 512 + 256 * j);
    }
  };
  f4 y[4][4] = {};
  copy_run(0);
  copy_x(0);
  for (int gi = 0; gi < ng; ++gi) {
    const int run = gi / kRun, k = gi % kRun;
    vm_wait<0>();
    lds_barrier();
    if (gi + 1 < ng) copy_x(gi + 1);
    if (k == 0 && gi + kRun < ng) copy_run(run + 1);
    const char* tile = xt[gi & 1];
    const char* codes = ct[run & 1];
    h8 b0[4], b1[4];
    float s[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int r = nw + 16 * n + c;
      const u2 w = *reinterpret_cast<const u2*>(codes + 128 * r + 16 * ((2 * k + (g >> 1)) ^ (r >> 1 & 7)) + 8 * (g & 1));
      b0[n] = codes8(w.x);
      b1[n] = codes8(w.y);
      s[n] = __low2float(__builtin_bit_cast(__half2, st[run & 1][k][r])) * kCodeUnit;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int r = tw + 16 * m + c;
      const h8 x0 = ld_h8(tile + 128 * r + 16 * ((2 * g) ^ x_key(r)));
      const h8 x1 = ld_h8(tile + 128 * r + 16 * ((2 * g + 1) ^ x_key(r)));
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const f4 d = mfma16(x1, b1[n], mfma16(x0, b0[n], f4{}));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[m][n][i] = fmaf(s[n], d[i], y[m][n][i]);
      }
    }
  }
  // the group sums by z and lora_scale A x by B
  const int KE = linear_extra(a.in_dim, a.r), az = (ng + 31) / 32 * 32;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int row = min(ow + 16 * n + c, a.out_dim - 1);
    const __half2* zrow = static_cast<const __half2*>(a.sz) + (size_t)row * ng;
    const _Float16* brow = static_cast<const _Float16*>(a.lora_b) + (size_t)row * a.r;
    f4 d[4] = {};
    for (int k = 0; k < KE; k += 32) {
      h8 b;                                              // (past the groups or the rank: any weight, times E's zero)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = k + 8 * g + e;
        b[e] = k < az ? __builtin_bit_cast(_Float16, __high2half(zrow[min(j, ng - 1)])) : brow[min(j - az, a.r - 1)];
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const size_t at = (size_t)min(t0 + tw + 16 * m + c, a.T - 1) * KE + k + 8 * g;
        d[m] = mfma16(ld_h8(a.e_lo + at), b, mfma16(ld_h8(a.e_hi + at), b, d[m]));
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + tw + 16 * m + 4 * g + i, o = ow + 16 * n + c;
        if (t < a.T && o < a.out_dim) store_out(a, t, o, fmaf(a.e_scale[t], d[m][i], y[m][n][i]));
      }
  }
}

template <int TT, int RT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const dim3 grid((a.out_dim + 15) / 16, (a.T + 16 * TT - 1) / (16 * TT));
  hipLaunchKernelGGL((linear_rows_kernel<TT, RT, 8>), grid, dim3(512), 0, st, a);
  return hipGetLastError();
}
template <int TT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  if (a.r == 0) return launch_rows<TT, 0>(a, st);
  if (a.r <= 16) return launch_rows<TT, 1>(a, st);
  return launch_rows<TT, 4>(a, st);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  if (a.T <= 16) return launch_rows<1>(a, st);
  if (a.T <= 64) return launch_rows<2>(a, st);
  const size_t lds = 16 * (size_t)linear_extra(a.in_dim, a.r) * sizeof(float);
  const dim3 grid((a.T + 15) / 16), block(512);
  if (a.r == 0)
    hipLaunchKernelGGL((linear_sums_kernel<0>), grid, block, lds, st, a);
  else if (a.r <= 16)
    hipLaunchKernelGGL((linear_sums_kernel<1>), grid, block, lds, st, a);
  else
    hipLaunchKernelGGL((linear_sums_kernel<4>), grid, block, lds, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(linear_tile_kernel, dim3((a.out_dim + 127) / 128, (a.T + 127) / 128), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {

constexpr int kMaxIn = 32768, kMaxOut = 1 << 20, kMaxRows = 1 << 20;

bool linear_shape_ok(int out_dim, int in_dim, int rank, int T) {
  return out_dim >= 1 && out_dim <= kMaxOut && in_dim >= 64 && in_dim <= kMaxIn && in_dim % 64 == 0 &&
         rank >= 0 && rank <= 64 && T >= 0 && T <= kMaxRows;
}
size_t round256(size_t v) { return (v + 255) / 256 * 256; }
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace

extern "C" {

size_t moe_linear_workspace_bytes(int out_dim, int in_dim, int rank, int T) {
  if (!linear_shape_ok(out_dim, in_dim, rank, T)) return 0;
  const size_t t = T < 1 ? 1 : T, ke = moe::linear_extra(in_dim, rank);
  return 2 * round256(t * ke * 2) + round256(t * 4);
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
  return moe::launch_linear(a, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
