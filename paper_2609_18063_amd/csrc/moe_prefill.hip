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
constexpr float kSlack = 8.f;    // (as a power of two)
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
// Workgroups [0, side): one 64-token tile of one sequence each. They copy its rotated
// keys into one run, and note which of its four 16-token groups have no page.
// Workgroups from `side` on: 128 context tokens by 128 of the H (Dn + Dv) columns on the
// matrix cores, four waves of 64 x 64, 64 latent columns a step through LDS, one ahead.
template <int DC>
__global__ void __launch_bounds__(256) latent_expand_kernel(PrefillArgs a, int side, int col_tiles) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][128 * 128];
  __shared__ int64_t where[128];
  const LatentArgs& l = a.l;
  const int row_halves = DC + l.Dr;
  if ((int)blockIdx.x < side) {
    const int b = last_at_most(a.B, blockIdx.x, [&](int k) { return tile_base(a, k); });
    const Span s = context_of(a, b);
    const int tok0 = ((int)blockIdx.x - tile_base(a, b)) * kTile;
    if (blockIdx.x == 0 && threadIdx.x < 64) {
      // (the lists are looked at once, by one wave)
      bool good = a.q_start[0] >= 0 && a.kv_start[0] >= 0 && a.q_start[a.B] <= a.T && a.kv_start[a.B] <= a.kv_total;
      for (int k = threadIdx.x; k < a.B; k += 64) {
        const int nq = a.q_start[k + 1] - a.q_start[k], nk = a.kv_start[k + 1] - a.kv_start[k];
        good = good && nq >= 0 && nq <= a.max_q && nk >= nq && nk <= (int64_t)l.max_pages * l.page;
      }
      if (!good && l.status) atomicOr(l.status, MOE_STATUS_BAD_LENGTH);
    }
    if (tok0 < 0 || tok0 >= s.len) return;
    uint32_t lost = 0;
    for (int grp = 0; grp < 4; ++grp) {
      const int tok = tok0 + 16 * grp;
      if (tok >= s.len) break;
      const int page = l.table[b * l.table_stride + tok / l.page];
      if (page < 0 || page >= l.n_pages) {
        lost |= 1u << grp;
        continue;
      }
      const __half* from = l.pages + ((size_t)page * l.page + tok % l.page) * row_halves + DC;
      const int pieces = l.Dr / 8, rows = min(16, s.len - tok);
      for (int e = threadIdx.x; e < rows * pieces; e += 256)
        *reinterpret_cast<U4*>(a.kr + (size_t)(s.first + tok + e / pieces) * l.Dr + 8 * (e % pieces)) =
            ld16(from + (size_t)(e / pieces) * row_halves + 8 * (e % pieces));
    }
    if (threadIdx.x == 0) {
      a.lost[blockIdx.x] = lost;
      if (lost && l.status) atomicOr(l.status, MOE_STATUS_BAD_PAGE);
    }
    return;
  }
  const int tile = blockIdx.x - side, n0 = (tile % col_tiles) * 128, r0 = (tile / col_tiles) * 128;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4, N = l.H * (l.Dn + l.Dv);
  // where the context rows are (a token without a page: the first page's first row, and
  // zeros are stored)
  if (threadIdx.x < 128) {
    const int at = min(r0 + (int)threadIdx.x, a.kv_total - 1);
    const int b = last_at_most(a.B, at, [&](int k) { return a.kv_start[k]; });
    const Span s = context_of(a, b);
    const int tok = at - s.first;
    int page = -1;
    if (tok >= 0 && tok < s.len) page = l.table[b * l.table_stride + tok / l.page];
    where[threadIdx.x] = page >= 0 && page < l.n_pages ? (int64_t)page * l.page + tok % l.page : -1;
  }
  __syncthreads();
  const char *src_c[4], *src_w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 8 * (4 * wave + j) + (lane >> 3), piece = 16 * ((lane & 7) ^ tile_key<8>(r));
    src_c[j] = reinterpret_cast<const char*>(l.pages + max(where[r], (int64_t)0) * row_halves) + piece;
    src_w[j] = reinterpret_cast<const char*>(l.w + (size_t)min(n0 + r, N - 1) * DC) + piece;
  }
  const uint32_t at0 = lds_at(lds);
  auto copy = [&](int k) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      dma16(src_c[j] + 128 * k, at0 + (k & 1) * 32768 + 1024 * (4 * wave + j));
      dma16(src_w[j] + 128 * k, at0 + (k & 1) * 32768 + 16384 + 1024 * (4 * wave + j));
    }
  };
  const int tr = (wave & 1) * 64, tn = (wave >> 1) * 64;
  f4 y[4][4] = {};
  copy(0);
  for (int k = 0; k < DC / 64; ++k) {
    vm_wait<0>();
    lds_barrier();
    if (k + 1 < DC / 64) copy(k + 1);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      h8 w[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int r = tn + 16 * n + c;
        w[n] = ld_h8(lds[k & 1][1] + 128 * r + 16 * ((4 * ks + g) ^ tile_key<8>(r)));
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int r = tr + 16 * m + c;
        const h8 x = ld_h8(lds[k & 1][0] + 128 * r + 16 * ((4 * ks + g) ^ tile_key<8>(r)));
#pragma unroll
        for (int n = 0; n < 4; ++n) y[m][n] = mfma16(w[n], x, y[m][n]);
      }
    }
  }
  const int hd = l.Dn + l.Dv;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int col = n0 + tn + 16 * n + 4 * g;
    if (col >= N) continue;
    const int h = col / hd, in = col % hd;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int r = tr + 16 * m + c, at = r0 + r;
      if (at >= a.kv_total) continue;
      const f4 d = where[r] >= 0 ? y[m][n] : f4{};
      const h4 v = {(_Float16)d[0], (_Float16)d[1], (_Float16)d[2], (_Float16)d[3]};
      __half* to = in < l.Dn ? a.k + ((size_t)h * a.kv_total + at) * l.Dn + in
                             : a.v + ((size_t)h * a.kv_total + at) * l.Dv + in - l.Dn;
      *reinterpret_cast<h4*>(to) = v;
    }
  }
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
  float m[RT], ref[RT], sum[RT];                         // reference (an unscaled score), m unit (or 0), sum
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
    // the reference of a row follows its maximum only where that passes it by kSlack: until
    // then the weights are at most 2^kSlack, and nothing is rescaled
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
        const float mx = fmaxf(m[r], col_max(top[r])), now = mx == -INFINITY ? 0.f : mx * unit;
        const float keep = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[r] - now);
        m[r] = mx;
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
      if (g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = float2{m[r] * unit, total};
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

// The parts of a row's context, joined: four values a thread, Dv / 4 threads a row.
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
    if (ml.x == -INFINITY) continue;                     // (a part without a token of the row)
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

}  // namespace

// Into how many parts the contexts are cut: as fill the CUs, of eight tiles at least on
// average.
int prefill_parts(int max_q, int H, int B, int kv_total) {
  static_assert(kRows == kPartRows, "rows of a partial result");
  const int64_t wholes = (int64_t)((max_q + kRows - 1) / kRows) * H * B;
  const int64_t most = std::max<int64_t>(1, kv_total / ((int64_t)B * kTile * 8));
  return (int)std::max<int64_t>(1, std::min<int64_t>({kPartGroups / wholes, most, 16}));
}

hipError_t launch_latent_prefill(const PrefillArgs& a, hipStream_t st) {
  const LatentArgs& l = a.l;
  const int side = a.kv_total / kTile + a.B, cols = (l.H * (l.Dn + l.Dv) + 127) / 128;
  const dim3 grid(side + (unsigned)cols * ((a.kv_total + 127) / 128)), block(256);
  if (l.Dc == 512)
    hipLaunchKernelGGL(latent_expand_kernel<512>, grid, block, 0, st, a, side, cols);
  else if (l.Dc == 256)
    hipLaunchKernelGGL(latent_expand_kernel<256>, grid, block, 0, st, a, side, cols);
  else
    hipLaunchKernelGGL(latent_expand_kernel<128>, grid, block, 0, st, a, side, cols);
  const hipError_t e = hipGetLastError();
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
  if (max_q < 1 || (int64_t)((max_q + moe::kPartRows - 1) / moe::kPartRows) * spec->heads * B * 512 > (int64_t)UINT32_MAX ||
      (int64_t)(kv_total / 128 + 1) * spec->heads * 2 * 256 + ((int64_t)kv_total / moe::kTile + B) * 256 >
          (int64_t)UINT32_MAX)
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
