// Latent attention for prompts, in its expanded form: a ragged batch of chunks, each the
// last tokens of its sequence's cached context, attends causally to that context.
//   k_j = (W_uk,h c_j, k_r,j),  v_j = W_uv,h c_j,  o_i = sum_{j <= i} softmax(scale q_i . k_j) v_j
// With many query rows the product over Dn + Dr + Dv columns a pair (the absorbed form
// has 2 Dc + Dr) pays for expanding every context token once, 2 (Dn + Dv) Dc operations
// a head: one launch expands keys and values into the workspace, a second attends.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "moe_latent.h"
#include "moe_tile.h"

namespace moe {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kWaves = 8, kRows = 32 * kWaves;  // of a workgroup of the attention: waves, query rows

struct Span {
  int first, len;
};
// Entries b and b + 1 of a list of starts, held inside [0, total].
__device__ __forceinline__ Span span_of(const int32_t* starts, int b, int total) {
  const int s = min(max(starts[b], 0), total), e = min(max(starts[b + 1], s), total);
  return Span{s, e - s};
}
// The last b in [0, B) whose key is at most v (keys ascend).
template <typename Key>
__device__ __forceinline__ int last_at_most(int B, int v, Key key) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (key(mid) <= v)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}
// Context tokens of sequence b: what the table can hold of them.
__device__ __forceinline__ Span context_of(const PrefillArgs& a, int b) {
  Span s = span_of(a.kv_start, b, a.kv_total);
  s.len = (int)min((int64_t)s.len, (int64_t)a.l.max_pages * a.l.page);
  return s;
}
// First 64-token tile of sequence b among all sequences' tiles (with gaps).
__device__ __forceinline__ int tile_base(const PrefillArgs& a, int b) {
  return min(max(a.kv_start[b], 0), a.kv_total) / kTile + b;
}

// ---- expanding the context ----------------------------------------------------------
// 256 of the H (Dn + Dv) columns by up to 512 context tokens a workgroup. A wave keeps its
// columns' weights of all Dc latents in registers and reads whole tokens, 32 a step, through
// LDS in four slots, copied three ahead: with the weights through LDS too, 128 x 128 tiles
// and one step ahead, 3,100 tokens of 512 latents by 32 heads of 256 columns took 54 us, now
// 39 (0.67 PFLOP/s): 13 until the first step (weights, page ids) and 1.9 a step, of which
// the LDS reads need 1.0 and the products 0.9. 256 latents, 64 columns a wave: 22 us for
// 14,500 tokens by 8 heads of 128 columns.
// Keys and values are rounded to fp16, as operands of the matrix cores: held as two halves
// each, the workspace and the attention's products and LDS reads, which bound it, would double.
// Before that the workgroups share the 64-token tiles of the sequences (`side` numbers):
// they copy a tile's rotated keys into one run, and note which of its four 16-token groups
// have no page.
constexpr int kExpandTokens = 32, kExpandMost = 512, kExpandCols = 256, kExpandSlots = 4;

// Products of 16 columns that a wave has: 512 latents' weights of four would be copied out of
// the accumulator registers for every product (43 us against 38 with two, below).
template <int DC>
constexpr int kExpandProducts = DC == 512 ? 2 : 4;
template <int DC>
constexpr int kExpandWaves = 16 / kExpandProducts<DC>;

template <int DC>
__global__ void __launch_bounds__(64 * kExpandWaves<DC>, 2)
    latent_expand_kernel(PrefillArgs a, int side, int col_groups, int splits) {
  constexpr int NM = kExpandProducts<DC>, NW = kExpandWaves<DC>, PR = DC / 8, CW = PR / 2 / NW, SLOT = kExpandTokens * DC * 2, KS = DC / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int64_t* where = reinterpret_cast<int64_t*>(lds + kExpandSlots * SLOT);
  __shared__ uint32_t lost[4];
  const LatentArgs& l = a.l;
  const int row_halves = DC + l.Dr;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4, hd = l.Dn + l.Dv, N = l.H * hd;
  const int split = blockIdx.x / col_groups, col0 = (blockIdx.x % col_groups) * kExpandCols + 16 * NM * wave;
  const int tiles = (a.kv_total + kExpandTokens - 1) / kExpandTokens;
  const int even = tiles / splits, more = tiles % splits;
  const int from = split * even + min(split, more), n = even + (split < more);
  const int first = from * kExpandTokens;
  // Columns: row i of product m is 4 NM (i / 4) + 4 m + i % 4 of the wave's, so that a lane has
  // 4 NM neighbouring columns of a token.
  h8 w[KS][NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    const __half* from_w = l.w + (size_t)min(col0 + 4 * NM * (c >> 2) + 4 * m + (c & 3), N - 1) * DC + 8 * g;
#pragma unroll
    for (int k = 0; k < KS; ++k) w[k][m] = ld_h8(from_w + 32 * k);
  }
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    // (the lists are looked at once, by one wave)
    bool good = a.q_start[0] >= 0 && a.kv_start[0] >= 0 && a.q_start[a.B] <= a.T && a.kv_start[a.B] <= a.kv_total;
    for (int k = threadIdx.x; k < a.B; k += 64) {
      const int nq = a.q_start[k + 1] - a.q_start[k], nk = a.kv_start[k + 1] - a.kv_start[k];
      good = good && nq >= 0 && nq <= a.max_q && nk >= nq && nk <= (int64_t)l.max_pages * l.page;
    }
    if (!good && l.status) atomicOr(l.status, MOE_STATUS_BAD_LENGTH);
  }
  for (int t = blockIdx.x; t < side; t += gridDim.x) {
    const int b = last_at_most(a.B, t, [&](int k) { return tile_base(a, k); });
    const Span s = context_of(a, b);
    const int tok0 = (t - tile_base(a, b)) * kTile;
    if (tok0 < 0 || tok0 >= s.len) continue;
    const int tok = tok0 + 16 * wave;                    // (a group a wave)
    int32_t page = -1;
    if (wave < 4 && tok < s.len) page = l.table[b * l.table_stride + tok / l.page];
    const bool there = page >= 0 && page < l.n_pages;
    if (there) {
      const __half* rope = l.pages + ((size_t)page * l.page + tok % l.page) * row_halves + DC;
      const int pieces = l.Dr / 8, rows = min(16, s.len - tok);
      for (int e = lane; e < rows * pieces; e += 64)
        *reinterpret_cast<U4*>(a.kr + (size_t)(s.first + tok + e / pieces) * l.Dr + 8 * (e % pieces)) =
            ld16(rope + (size_t)(e / pieces) * row_halves + 8 * (e % pieces));
    }
    __syncthreads();
    if (lane == 0 && wave < 4) lost[wave] = !there && tok < s.len;
    __syncthreads();
    if (threadIdx.x == 0) {
      const uint32_t mask = lost[0] | lost[1] << 1 | lost[2] << 2 | lost[3] << 3;
      a.lost[t] = mask;
      if (mask && l.status) atomicOr(l.status, MOE_STATUS_BAD_PAGE);
    }
  }
  if (n < 1) return;
  // Where the tokens' rows are, as byte offsets (one without a page: -1; zeros are stored).
  // Behind the last token its own values are stored again.
  for (int i = threadIdx.x; i < n * kExpandTokens; i += 64 * NW) {
    const int at = min(first + i, a.kv_total - 1);
    const int b = last_at_most(a.B, at, [&](int k) { return a.kv_start[k]; });
    const Span s = context_of(a, b);
    const int tok = at - s.first;
    int page = -1;
    if (tok >= 0 && tok < s.len) page = l.table[b * l.table_stride + tok / l.page];
    where[i] = page >= 0 && page < l.n_pages ? ((int64_t)page * l.page + tok % l.page) * (2 * row_halves) : -1;
  }
  vm_drain();                                            // (the weights: asked for before the page ids)
  __syncthreads();
  const uint32_t at0 = lds_at(lds);
  auto copy = [&](int u) {                               // (past the last tile: it again, into a free slot)
    const int t = min(u, n - 1), slot = u % kExpandSlots;
    const char* src[CW];
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      const int p = 64 * (CW * wave + j) + lane, r = p / PR;
      src[j] = reinterpret_cast<const char*>(l.pages) + max(where[t * kExpandTokens + r], (int64_t)0) +
               16 * ((p % PR) ^ tile_key<PR>(r));
    }
#pragma unroll
    for (int j = 0; j < CW; ++j) dma16(src[j], at0 + slot * SLOT + 1024 * (CW * wave + j));
  };
  for (int u = 0; u < 3; ++u) copy(u);
  const int h = min(col0, N - 1) / hd, in = min(col0, N - 1) % hd;
  // Values are stored finite: a row's weight 0 of a token that it does not see then gives 0,
  // whatever the token holds. (Its keys stay as they are, and make NaN of the rows that see it.)
  // Not so where the weights of the wave's columns are not finite, which no key would show:
  // times zeros they add up to NaN, else to 0. (Formed while the copies are on their way.)
  __builtin_amdgcn_sched_barrier(0);
  f4 whole[4] = {};
  if (in >= l.Dn)
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        f4& sum = whole[(k * NM + m) % 4];
        sum = mfma16(w[k][m], h8{}, sum);
      }
  const f4 odd = whole[0] + whole[1] + whole[2] + whole[3];
  const bool values = in >= l.Dn && !__any(odd[0] + odd[1] + odd[2] + odd[3] != 0.f);
  const bool idle = col0 >= N;
  __half* to = in < l.Dn ? a.k + (size_t)h * a.kv_total * l.Dn + in : a.v + (size_t)h * a.kv_total * l.Dv + in - l.Dn;
  const int to_row = in < l.Dn ? l.Dn : l.Dv;
  for (int u = 0; u < n; ++u) {
    // what was asked for after tile u: the copies of two tiles, and NM stores a tile
    if (idle || u == 0)
      vm_wait<2 * CW>();
    else if (u == 1)
      vm_wait<2 * CW + NM>();
    else
      vm_wait<2 * CW + 2 * NM>();
    lds_barrier();
    copy(u + 3);
    if (idle) continue;
    const char* x = lds + (u % kExpandSlots) * SLOT;
    // (the reads of KR steps are asked for before the products of the KR before them)
    f4 y[2][NM] = {};
    constexpr int KR = 4;
    h8 v[2][KR][2];
    auto read = [&](int k) {
#pragma unroll
      for (int i = 0; i < KR; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          v[k / KR & 1][i][t] =
              ld_h8(x + (16 * t + c) * (DC * 2) + 16 * ((4 * (k + i) + g) ^ tile_key<PR>(c)));
    };
    read(0);
#pragma unroll
    for (int k = 0; k < KS; k += KR) {
      if (k + KR < KS) read(k + KR);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KR; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int m = 0; m < NM; ++m) y[t][m] = mfma16(w[k + i][m], v[k / KR & 1][i][t], y[t][m]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = u * kExpandTokens + 16 * t + c;
      const bool there = where[r] >= 0;
      __half* row = to + (size_t)min(first + r, a.kv_total - 1) * to_row + 4 * NM * g;
#pragma unroll
      for (int half = 0; half < NM / 2; ++half) {
        h8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float e = y[t][2 * half + i / 4][i % 4];
          if (values) e = fminf(fmaxf(e, -65504.f), 65504.f);
          o[i] = there ? (_Float16)e : (_Float16)0.f;
        }
        *reinterpret_cast<h8*>(row + 8 * half) = o;
      }
    }
  }
  vm_wait<0>();                                          // (copies may be in flight into this workgroup's LDS)
}

// ---- attention ------------------------------------------------------------------------
// 256 query rows of one head a workgroup, 32 a wave, with the query in registers; tiles of
// 64 context tokens in LDS, copied one ahead, one barrier each. Scores are formed
// transposed (tokens x rows): a lane then holds its row's weights of the tokens
// 16 t + 4 g .. + 3, which are the operand of the product with the values as they are,
// when the values' rows are read (transposed) in the same order. The reference and the
// sum of a row are in the four lanes of its column. Late tiles first, and the heads of a
// tile next to each other, so that one head's workgroups share a chiplet's L2.
// With fewer workgroups than CUs the context is cut into parts, a workgroup each, whose
// (m, l, O) one more launch joins.
// Between a tile's copies and the next barrier no load is waited for: loads come back in
// order, and the wait would be for the copies.
// 3,100 tokens, 32 heads of 128 + 64 and 128: 119 us, 0.83 PFLOP/s; bound by LDS, whose reads
// (every wave reads all keys and values) take 3,600 of a tile's 5,300 clocks.
template <int DN, int DR, int DV, bool PARTS>
__global__ void __launch_bounds__(64 * kWaves, 2) latent_prefill_kernel(PrefillArgs a) {
  constexpr int KB = kTile * DN * 2, RB = kTile * DR * 2, VB = kTile * DV * 2, BUF = KB + RB + VB;
  constexpr int KS = (DN + DR) / 32, CT = DV / 16, RT = 2, OWN = kTile / kWaves;  // OWN: token rows a wave copies
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const LatentArgs& l = a.l;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4;
  const int part = PARTS ? blockIdx.x % a.parts : 0, whole = PARTS ? blockIdx.x / a.parts : blockIdx.x;
  const int heads = l.H * a.B, qt = (a.max_q + kRows - 1) / kRows - 1 - whole / heads;
  const int hb = whole % heads, h = hb % l.H, b = hb / l.H;
  const Span qs = span_of(a.q_start, b, a.T), ks = context_of(a, b);
  if (qt * kRows >= qs.len) return;
  const int shift = ks.len - qs.len;                     // position of query row 0
  const int row0 = qt * kRows + 32 * wave;               // this wave's first row
  const int last_row = min(qt * kRows + kRows, qs.len) - 1;
  const int all = shift + last_row >= 0 ? (shift + last_row) / kTile + 1 : 0;
  const int first = PARTS ? (int)((int64_t)all * part / a.parts) : 0;  // the tiles of this part: first .. tiles - 1
  const int tiles = PARTS ? (int)((int64_t)all * (part + 1) / a.parts) : all;
  const int mine = row0 < qs.len ? shift + min(row0 + 31, qs.len - 1) : -1;  // last position that the wave's rows see
  h8 q[RT][KS];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const size_t row = qs.first + min(row0 + 16 * r + c, qs.len - 1);
#pragma unroll
    for (int k = 0; k < KS; ++k) q[r][k] = ld_h8(l.q + (row * l.H + h) * (DN + DR) + 32 * k + 8 * g);
  }
  const char* kb = reinterpret_cast<const char*>(a.k + ((size_t)h * a.kv_total + ks.first) * DN);
  const char* vb = reinterpret_cast<const char*>(a.v + ((size_t)h * a.kv_total + ks.first) * DV);
  const char* rb = reinterpret_cast<const char*>(a.kr + (size_t)ks.first * DR);
  // rows of P pieces of 16 bytes, R rows a copy; rows past the context repeat its last one
  auto rows = [&](const char* from, int tile, uint32_t to, auto pieces) {
    constexpr int P = decltype(pieces)::value, R = kWave / P;
    int ln = lane;
    if constexpr (PARTS) asm volatile("" : "+v"(ln));
    const char* base = from + (size_t)tile * kTile * (P * 16);
    const int most = ks.len - 1 - tile * kTile;
#pragma unroll
    for (int j = 0; j < (OWN + R - 1) / R; ++j) {
      const int r0 = OWN * wave + j * R, r = r0 + ln / P;
      if (R <= OWN || wave % (R / OWN) == 0)             // (a copy of 16 rows is two waves' share)
        dma16(base, (uint32_t)min(r, most) * (P * 16) + 16 * ((ln % P) ^ tile_key<P>(r)), to + r0 * P * 16);
    }
  };
  const uint32_t at0 = lds_at(lds);
  auto copy = [&](int tile) {
    const uint32_t buf = at0 + (tile & 1) * BUF;
    rows(kb, tile, buf, std::integral_constant<int, DN / 8>());
    rows(rb, tile, buf + KB, std::integral_constant<int, DR / 8>());
    rows(vb, tile, buf + KB + RB, std::integral_constant<int, DV / 8>());
  };
  f4 o[CT][RT] = {};
  float m[RT], ref[RT], sum[RT];                         // reference (an unscaled score), m unit - kRaise (or 0), sum
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = -INFINITY;
    ref[r] = sum[r] = 0.f;
  }
  const float unit = l.scale * kLog2e;
  const uint32_t* lost_of = a.lost + tile_base(a, b);
  uint32_t lost_next = 0;
  if (first < tiles) {
    lost_next = lost_of[first];
    copy(first);
  }
  for (int i = first; i < tiles; ++i) {
    const char* buf = lds + (i & 1) * BUF;
    vm_drain();
    lds_barrier();
    const uint32_t lost = __builtin_amdgcn_readfirstlane(lost_next);
    if (i + 1 < tiles) {
      lost_next = lost_of[i + 1];
      copy(i + 1);
    }
    if (i * kTile > mine) continue;
    // (with parts the addresses are formed tile by tile: held, they would spill, and a
    // register that comes back from memory waits for the copies)
    int c1 = c, g1 = g, c2 = c, g2 = g;
    if constexpr (PARTS) asm volatile("" : "+v"(c1), "+v"(g1));
    f4 s[4][RT] = {};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int tok = 16 * t + c1;
        const char* p = k < DN / 32 ? buf + tok * DN * 2 + 16 * ((4 * k + g1) ^ tile_key<DN / 8>(c1))
                                    : buf + KB + tok * DR * 2 + 16 * ((4 * (k - DN / 32) + g1) ^ tile_key<DR / 8>(c1));
        const h8 kk = ld_h8(p);
#pragma unroll
        for (int r = 0; r < RT; ++r) s[t][r] = mfma16(kk, q[r][k], s[t][r]);
      }
    if (lost || (i + 1) * kTile > shift + row0 + 1) {    // some row does not see the whole tile
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int see = shift + row0 + 16 * r + c - i * kTile - 4 * g;  // the row sees tokens 0 .. see + 4 g of the tile
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * t + e > see || (lost >> t & 1)) s[t][r][e] = -INFINITY;
      }
    }
    // the reference of a row follows its maximum only where that passes it by kSlack
    float top[RT];
    bool far = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      top[r] = fmaxf(s[0][r][0], s[0][r][1]);
#pragma unroll
      for (int e = 2; e < 16; e += 2) top[r] = max3(top[r], s[e >> 2][r][e & 3], s[e >> 2][r][(e & 3) + 1]);
      far = far || (top[r] - m[r]) * unit > kSlack;      // (no token so far: any score is)
    }
    if (__any(far)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float mx = fmaxf(m[r], col_max(top[r]));
        const bool past = (mx - m[r]) * unit > kSlack;   // (a row's roundings are its own)
        const float now = past ? mx * unit - kRaise : ref[r];
        const float keep = !past ? 1.f : m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[r] - now);
        m[r] = past ? mx : m[r];
        ref[r] = now;
        sum[r] *= keep;
#pragma unroll
        for (int k = 0; k < CT; ++k) o[k][r] *= keep;
      }
    }
    h8 p[2][RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float add = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __builtin_amdgcn_exp2f(fmaf(s[t][r][e], unit, -ref[r]));
          add += v;
          p[t >> 1][r][4 * (t & 1) + e] = (_Float16)v;
        }
      sum[r] += add;
    }
    const char* vt = buf + KB + RB;
    if constexpr (PARTS) asm volatile("" : "+v"(c2), "+v"(g2));
    const int t0 = 4 * g2 + (c2 >> 2);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int k = 0; k < CT; ++k) {
        h4 part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int tok = 32 * hf + 16 * u + t0, col = 16 * k + 4 * (c2 & 3);
          part[u] = ld_tr(vt + tok * DV * 2 + 16 * ((col >> 3) ^ tile_key<DV / 8>(t0)) + 2 * (col & 7));
        }
        const h8 v = join(part[0], part[1]);
#pragma unroll
        for (int r = 0; r < RT; ++r) o[k][r] = mfma16(v, p[hf][r], o[k][r]);
      }
  }
  uint32_t mine_at = blockIdx.x;
  if constexpr (PARTS) asm volatile("" : "+s"(mine_at));
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float total = col_sum(sum[r]);
    const int row = row0 + 16 * r + c;
    if (row >= qs.len) continue;
    if constexpr (PARTS) {
      const size_t at = (size_t)mine_at * kRows + 32 * wave + 16 * r + c;
      if (g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = float2{m[r] == -INFINITY ? m[r] : ref[r], total};
      // (divided by its sum: stored as it is, o would be held twice over the loop, and spill)
      const float inv = total > 0.f ? 1.f / total : 0.f;
#pragma unroll
      for (int k = 0; k < CT; ++k) *reinterpret_cast<f4*>(a.part_o + at * DV + 16 * k + 4 * g) = o[k][r] * inv;
      continue;
    }
    const float inv = total > 0.f ? 1.f / total : total != total ? total : 0.f;  // (no token: zeros)
    __half* to = l.out + ((size_t)(qs.first + row) * l.H + h) * DV + 4 * g;
#pragma unroll
    for (int k = 0; k < CT; ++k) {
      const f4 d = o[k][r] * inv;
      const h4 v = {(_Float16)d[0], (_Float16)d[1], (_Float16)d[2], (_Float16)d[3]};
      *reinterpret_cast<h4*>(to + 16 * k) = v;
    }
  }
}

// The parts of a row's context, joined: four values a thread, Dv / 4 threads a row (40
// row blocks of 5 parts: 6.7 us, latency).
__global__ void __launch_bounds__(256) latent_parts_kernel(PrefillArgs a) {
  const LatentArgs& l = a.l;
  const int per = l.Dv / 4, rows = 256 / per, blocks = kRows / rows;
  const int whole = blockIdx.x / blocks, in = blockIdx.x % blocks * rows + threadIdx.x / per, col = 4 * (threadIdx.x % per);
  const int heads = l.H * a.B, qt = (a.max_q + kRows - 1) / kRows - 1 - whole / heads;
  const int hb = whole % heads, h = hb % l.H, b = hb / l.H;
  const Span qs = span_of(a.q_start, b, a.T);
  const int row = qt * kRows + in;
  if (row >= qs.len) return;
  const size_t at = (size_t)whole * a.parts * kRows + in;
  float top = -INFINITY;
  for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.part_ml[2 * (at + (size_t)p * kRows)]);
  float sum = 0.f;
  f4 o = {};
#pragma unroll 4
  for (int p = 0; p < a.parts; ++p) {
    const size_t i = at + (size_t)p * kRows;
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * i);
    const f4 v = *reinterpret_cast<const f4*>(a.part_o + i * l.Dv + col);
    if (ml.x == -INFINITY) {                             // (no score of it is above that: its sum is 0, or NaN)
      sum += ml.y;
      continue;
    }
    const float w = __builtin_amdgcn_exp2f(ml.x - top) * ml.y;
    sum += w;
    o += v * w;
  }
  const float inv = sum > 0.f ? 1.f / sum : sum != sum ? sum : 0.f;
  const h4 v = {(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
  *reinterpret_cast<h4*>(l.out + ((size_t)(qs.first + row) * l.H + h) * l.Dv + col) = v;
}

template <int DN, int DR, int DV, bool PARTS>
hipError_t launch_attention(const PrefillArgs& a, unsigned wholes, hipStream_t st) {
  constexpr int lds = 2 * kTile * (DN + DR + DV) * 2;
  auto kernel = latent_prefill_kernel<DN, DR, DV, PARTS>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(wholes * a.parts), dim3(64 * kWaves), lds, st, a);
  return hipGetLastError();
}
template <int DN, int DR, int DV>
hipError_t launch_attention(const PrefillArgs& a, hipStream_t st) {
  const unsigned wholes = (a.max_q + kRows - 1) / kRows * a.l.H * a.B;
  if (a.parts == 1) return launch_attention<DN, DR, DV, false>(a, wholes, st);
  const hipError_t e = launch_attention<DN, DR, DV, true>(a, wholes, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(latent_parts_kernel, dim3(wholes * (kRows * DV / 1024)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int DN, int DR>
hipError_t launch_attention(const PrefillArgs& a, hipStream_t st) {
  return a.l.Dv == 128 ? launch_attention<DN, DR, 128>(a, st) : launch_attention<DN, DR, 64>(a, st);
}
template <int DN>
hipError_t launch_attention(const PrefillArgs& a, hipStream_t st) {
  return a.l.Dr == 64 ? launch_attention<DN, 64>(a, st) : launch_attention<DN, 32>(a, st);
}

// As many splits of the tokens as fill the CUs (the weights of 512 latent columns leave room
// for one workgroup there, else two), and at least one per kExpandMost tokens.
template <int DC>
hipError_t launch_expand(const PrefillArgs& a, hipStream_t st) {
  constexpr int lds = kExpandSlots * kExpandTokens * DC * 2 + kExpandMost * 8, slots = 256 * (DC == 512 ? 1 : 2);
  const int groups = (a.l.H * (a.l.Dn + a.l.Dv) + kExpandCols - 1) / kExpandCols;
  const int tiles = (a.kv_total + kExpandTokens - 1) / kExpandTokens, most = kExpandMost / kExpandTokens;
  const int splits = std::max({1, std::min((slots + groups - 1) / groups, tiles), (tiles + most - 1) / most});
  auto kernel = latent_expand_kernel<DC>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups * splits), dim3(64 * kExpandWaves<DC>), lds, st, a, a.kv_total / kTile + a.B, groups, splits);
  return hipGetLastError();
}

}  // namespace

// Into how many parts the contexts are cut: as fill the CUs, of eight tiles at least on
// average (777 tokens in five chunks on 14,500, 8 heads: the call in 53 us; uncut, with an
// earlier expansion, 121 against 62).
int prefill_parts(int max_q, int H, int B, int kv_total) {
  static_assert(kRows == kPartRows, "rows of a partial result");
  const int64_t wholes = (int64_t)((max_q + kRows - 1) / kRows) * H * B;
  const int64_t most = std::max<int64_t>(1, kv_total / ((int64_t)B * kTile * 8));
  return (int)std::max<int64_t>(1, std::min<int64_t>({kPartGroups / wholes, most, 16}));
}

hipError_t launch_latent_prefill(const PrefillArgs& a, hipStream_t st) {
  const LatentArgs& l = a.l;
  const hipError_t e = l.Dc == 512 ? launch_expand<512>(a, st) : l.Dc == 256 ? launch_expand<256>(a, st) : launch_expand<128>(a, st);
  if (e != hipSuccess) return e;
  return l.Dn == 128 ? launch_attention<128>(a, st) : launch_attention<64>(a, st);
}

}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct PrefillLayout {
  size_t k, v, kr, lost, part_o, part_ml, total;
};
constexpr int kMaxTotal = 1 << 24, kMaxBatch = 1 << 16;

bool prefill_shape_ok(const moe_latent_spec* s, int T, int B, int kv_total) {
  return moe_latent_spec_check(s) == MOE_OK && T >= 0 && T <= kMaxTotal && B >= 0 && B <= kMaxBatch && kv_total >= 0 &&
         kv_total <= kMaxTotal;
}
PrefillLayout prefill_layout(const moe_latent_spec* s, int B, int kv_total) {
  PrefillLayout p{};
  const size_t n = kv_total;
  p.k = 0;
  p.v = round256((size_t)s->heads * n * s->d_nope * 2);
  p.kr = p.v + round256((size_t)s->heads * n * s->d_v * 2);
  p.lost = p.kr + round256(n * s->d_rope * 2);
  p.part_o = p.lost + round256((n / moe::kTile + B) * 4);
  p.part_ml = p.part_o + (size_t)moe::kPartGroups * moe::kPartRows * s->d_v * 4;
  p.total = p.part_ml + (size_t)moe::kPartGroups * moe::kPartRows * 8;
  return p;
}

}  // namespace

extern "C" {

size_t moe_latent_prefill_workspace_bytes(const moe_latent_spec* s, int B, int kv_total) {
  if (!prefill_shape_ok(s, 0, B, kv_total)) return 0;
  return prefill_layout(s, B < 1 ? 1 : B, kv_total < 1 ? 1 : kv_total).total;
}

int moe_latent_prefill(const moe_latent_spec* spec, const moe_latent_cache* cache, const void* w_kvb_f16,
                       const void* q_f16, int T, const int32_t* q_start, const int32_t* kv_start, int B, int kv_total,
                       int max_q, void* out_f16, uint32_t* status, void* workspace, size_t workspace_bytes,
                       void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (!prefill_shape_ok(spec, T, B, kv_total) || B > cache->n_seqs || max_q < 0 || max_q > T)
    return MOE_EINVAL;
  if (T == 0 || B == 0) return T == 0 ? MOE_OK : MOE_EINVAL;
  if (max_q < 1 || (int64_t)((max_q + moe::kPartRows - 1) / moe::kPartRows) * spec->heads * B * 512 > (int64_t)UINT32_MAX)
    return MOE_EINVAL;  // (a grid's threads)
  if (!w_kvb_f16 || !q_f16 || !q_start || !kv_start || !out_f16 || !workspace) return MOE_EINVAL;
  if (misaligned(w_kvb_f16, 16) || misaligned(q_f16, 16) || misaligned(q_start, 4) || misaligned(kv_start, 4) ||
      misaligned(out_f16, 16) || misaligned(status, 4) || misaligned(workspace, 16))
    return MOE_EALIGN;
  const PrefillLayout p = prefill_layout(spec, B, kv_total);
  if (workspace_bytes < p.total) return MOE_ENOMEM;
  moe::PrefillArgs a{};
  a.l = moe::latent_args(spec, cache);
  a.l.w = static_cast<const __half*>(w_kvb_f16);
  a.l.q = static_cast<const __half*>(q_f16);
  a.l.out = static_cast<__half*>(out_f16);
  a.l.status = status;
  a.T = T;
  a.B = B;
  a.kv_total = kv_total;
  a.max_q = max_q;
  a.q_start = q_start;
  a.kv_start = kv_start;
  char* ws = static_cast<char*>(workspace);
  a.k = reinterpret_cast<__half*>(ws + p.k);
  a.v = reinterpret_cast<__half*>(ws + p.v);
  a.kr = reinterpret_cast<__half*>(ws + p.kr);
  a.lost = reinterpret_cast<uint32_t*>(ws + p.lost);
  a.part_o = reinterpret_cast<float*>(ws + p.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + p.part_ml);
  a.parts = moe::prefill_parts(max_q, spec->heads, B, kv_total);
  return moe::launch_latent_prefill(a, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
