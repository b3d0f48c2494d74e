// What the cache's two forms share (moe_latent: fp16 rows, moe_latent4: 4-bit rows): the
// queries' rotation, and of latent attention for single tokens how the tiles of all sequences
// (32 and 64 tokens: STEP) are shared among the workgroups, the ways into and out of the
// latent space, and the joins of partial results.
#pragma once

#include "moe_latent.h"
#include "moe_tile.h"

namespace moe {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kCus = 256;
constexpr int kItemCost = 8;     // (measured: an item costs a workgroup 4 to 9 us, a tile 1 to 1.4; of 4 bits 1.4 to 2.7)

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// ---- cache writes -------------------------------------------------------------
// Part `part` of token t's query, rotated by the (cos, sin) of its position: 8 halves a thread.
__device__ __forceinline__ void rotate_query(const AppendArgs& a, int t, int part, const float2* cs) {
  const LatentArgs& l = a.l;
  const int hd = l.Dn + l.Dr, e = (part * 256 + threadIdx.x) * 8, n = l.H * hd;
  if (e >= n) return;
  const int in_head = e % hd;
  const size_t at = (size_t)t * n + e;
  h8 v = ld_h8(l.q + at);
  if (in_head >= l.Dn) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 r = cs[(in_head - l.Dn) / 2 + k];
      const float x = (float)v[2 * k], y = (float)v[2 * k + 1];
      v[2 * k] = (_Float16)(x * r.x - y * r.y);
      v[2 * k + 1] = (_Float16)(x * r.y + y * r.x);
    }
  }
  *reinterpret_cast<h8*>(a.q_out + at) = v;
}

// ---- the decode call's plan -----------------------------------------------------
__device__ __forceinline__ int clamp_len(const DecodeArgs& a, int n) {
  const int64_t cap = (int64_t)a.l.max_pages * a.l.page;
  return min(max(n, 0), (int)(cap < a.max_len ? cap : a.max_len));
}
template <int STEP>
__device__ __forceinline__ int tiles_of(int len) { return (len + STEP - 1) / STEP; }

// An item takes its tiles and kItemCost places more on the line (nothing without tiles):
// what its query's loads and its partial result cost a workgroup, in tiles.
__device__ __forceinline__ int places(int tiles) { return tiles > 0 ? tiles + kItemCost : 0; }

// Places of the line that a workgroup takes.
__device__ __forceinline__ int share(const DecodeArgs& a) {
  return max(a.p.least, (ld_scalar(a.starts + a.B) + a.p.wgs - 1) / a.p.wgs);
}

struct Item {
  int index, start, tiles;  // order number, first place on the line, tiles
  int row0, rows;           // query rows
  int tok0, last;           // first token, last token that may be read
  const int32_t* pages;
};

template <int STEP>
__device__ __forceinline__ Item prefix_item(const DecodeArgs& a, int chunk, int rb) {
  Item it;
  const int all = tiles_of<STEP>(a.prefix_len), first = chunk * a.p.chunk_tiles;
  it.index = chunk * a.p.row_blocks + rb;
  it.tiles = min(a.p.chunk_tiles, all - first);
  it.start = chunk * a.p.row_blocks * places(a.p.chunk_tiles) + rb * places(it.tiles);
  it.row0 = rb * a.p.rows;
  it.rows = min(a.p.rows, a.B * a.l.H - it.row0);
  it.tok0 = first * STEP;
  it.last = a.prefix_len - 1;
  it.pages = a.prefix;
  return it;
}
template <int STEP>
__device__ __forceinline__ Item own_item(const DecodeArgs& a, int b, int hb, int start, int len) {
  Item it;
  it.index = a.p.chunks * a.p.row_blocks + b * a.p.head_blocks + hb;
  it.tiles = tiles_of<STEP>(len);
  it.start = start + hb * places(it.tiles);
  it.row0 = b * a.l.H + hb * a.p.rows;
  it.rows = min(a.p.rows, a.l.H - hb * a.p.rows);
  it.tok0 = 0;
  it.last = len - 1;
  it.pages = a.l.table + b * a.l.table_stride;
  return it;
}
// A workgroup's tiles of one item after the other: [t, end) of the line. What the next
// sequence's item needs is read while the one at hand is worked on.
template <int STEP>
struct Walk {
  Item it;
  int first, n;             // its tiles of the item
  int t, end;
  int b, s0, s1, s2;        // the sequence at hand, its start, and the next two
  int len0, len1;
  int starts, lens;         // of sequence `lane`, where a wave's lanes hold them all
  __device__ __forceinline__ void begin(const DecodeArgs& a, int wg) {
    b = -1;
    s1 = s2 = 0;
    const int lane = threadIdx.x & 63;
    starts = a.starts[min(lane, a.B)];
    lens = a.kv_len[min(lane, a.B - 1)];
    const int all = ld_scalar(a.starts + a.B), per = share(a);
    t = (int)min((int64_t)all, (int64_t)wg * per);
    end = min(all, t + per);
  }
  __device__ __forceinline__ bool next(const DecodeArgs& a) {
    while (t < end) {
      if (t < a.p.prefix_places) {
        const int chunk = t / (a.p.row_blocks * places(a.p.chunk_tiles));
        const Item one = prefix_item<STEP>(a, chunk, 0);
        it = prefix_item<STEP>(a, chunk, (t - one.start) / places(one.tiles));
      } else {
        sequence_at(a);
        it = own_item<STEP>(a, b, (t - s0) / places(tiles_of<STEP>(len0)), s0, len0);
      }
      const int from = it.start + kItemCost, to = min(end, from + it.tiles);
      first = max(t - from, 0);
      n = to - from - first;
      t = to < end ? from + it.tiles : end;
      if (n > 0) return true;
    }
    return false;
  }

 private:
  // the sequence with starts[b] <= t < starts[b + 1] (sequences without a tile share their
  // start with the next one: the last of equals is the one that has the tile)
  __device__ __forceinline__ void sequence_at(const DecodeArgs& a) {
    if (t < s1) return;
    if (a.B < kWave) {
      const int lane = threadIdx.x & 63;
      b = __popcll(__ballot(lane < a.B && starts <= t)) - 1;
      s0 = __builtin_amdgcn_readlane(starts, b);
      s1 = __builtin_amdgcn_readlane(starts, b + 1);
      len0 = clamp_len(a, __builtin_amdgcn_readlane(lens, b));
      return;
    }
    if (t < s2) {
      ++b;
      s0 = s1;
      s1 = s2;
      len0 = len1;
    } else {
      // 64 starts at a time, each lane one
      int lo = 0, count = a.B;
      while (count > 1) {
        const int step = (count + kWave - 1) / kWave, i = lo + (int)(threadIdx.x & 63) * step;
        const bool below = i < lo + count && a.starts[min(i, a.B)] <= t;
        const int k = __popcll(__ballot(below)) - 1;
        count = min(step, lo + count - (lo + k * step));
        lo += k * step;
      }
      b = lo;
      s0 = ld_scalar(a.starts + b);
      s1 = ld_scalar(a.starts + b + 1);
      len0 = clamp_len(a, ld_scalar(a.kv_len + b));
    }
    s2 = ld_scalar(a.starts + min(b + 2, a.B));
    len1 = clamp_len(a, ld_scalar(a.kv_len + min(b + 1, a.B - 1)));
  }
};

// The runs of tiles of every workgroup, written out (the 4-bit cache: its attention walks the line
// in a short loop then, which the instruction cache and the scalar registers have room for). A
// workgroup's first run stands at its number, the others behind all of those; the whole
// workgroup calls, behind the writes of the starts. held: the first `room` of lds are the starts, the
// next ones the lengths.
__device__ __forceinline__ void list_runs(const DecodeArgs& a, int all, const int* lds, int room, bool held) {
  const int per = max(a.p.least, (all + a.p.wgs - 1) / a.p.wgs);
  for (int wg = threadIdx.x; wg < a.p.wgs; wg += 256) {
    int t = (int)min((int64_t)all, (int64_t)wg * per);
    const int end = min(all, t + per);
    DecodeRun run{};
    DecodeRun* to = a.runs + wg;
    while (t < end) {
      int lo = 0, hi = a.B;                              // (of equal starts the last one has the tile)
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((held ? lds[mid] : a.starts[mid]) <= t)
          lo = mid;
        else
          hi = mid;
      }
      const int s0 = held ? lds[lo] : a.starts[lo], len = held ? lds[room + lo] : clamp_len(a, a.kv_len[lo]);
      const Item it = own_item<64>(a, lo, (t - s0) / places(tiles_of<64>(len)), s0, len);
      const int from = it.start + kItemCost, upto = min(end, from + it.tiles), first = max(t - from, 0), n = upto - from - first;
      t = upto < end ? from + it.tiles : end;
      if (n <= 0) continue;
      const int seg = wg + it.index;
      if (run.n) {
        run.next = a.p.wgs + seg;
        *to = run;
        to = a.runs + a.p.wgs + seg;
      }
      run = DecodeRun{it.row0, it.rows, first, n, it.last, lo, seg, -1};
    }
    *to = run;
  }
}

// ---- q into the latent space ------------------------------------------------------
// qt_h = W_uk,h^T q_n,h for 64 latent columns of one head and 64 sequences a workgroup;
// W_uk,h's columns are staged in LDS and read transposed. qt is rounded to fp16, the
// type of the rows that it meets. The first column block copies q_r beside it; one
// further block adds up the tiles of the sequences for the plan. Bound by latency (weights,
// LDS, products): 48 sequences of 32 heads, 4.2 MB of weights, 5.7 us (7.5 with the queries
// asked for after the weights).
template <int DN, int STEP>
__global__ void __launch_bounds__(256) latent_absorb_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) char wt[DN * 128];
  __shared__ int scan[4];
  const LatentArgs& l = a.l;
  const int h = blockIdx.y, b0 = blockIdx.z * 64, b1 = min(b0 + 64, a.B);
  if ((int)blockIdx.x == l.Dc / 64) {
    if (blockIdx.y || blockIdx.z) return;
    constexpr int kRoom = STEP == 64 ? DN * 16 : 0;       // (as many starts, and lengths, does wt hold)
    int* held = reinterpret_cast<int*>(wt);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = a.p.prefix_places;
    for (int c0 = 0; c0 < a.B; c0 += 256) {
      const int b = c0 + threadIdx.x;
      int n = 0, len = 0;
      if (b < a.B) {
        const int given = a.kv_len[b];
        len = clamp_len(a, given);
        if (len != given && l.status) atomicOr(l.status, MOE_STATUS_BAD_LENGTH);
        n = places(tiles_of<STEP>(len)) * a.p.head_blocks;
      }
      int up = n;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(up, o, kWave);
        if (lane >= o) up += v;
      }
      if (lane == kWave - 1) scan[wave] = up;
      __syncthreads();
      int all = 0;
      for (int w = 0; w < 4; ++w) {
        if (w < wave) up += scan[w];
        all += scan[w];
      }
      if (b < a.B) {
        a.starts[b] = base + up - n;
        if (b < kRoom) {
          held[b] = base + up - n;
          held[kRoom + b] = len;
        }
      }
      base += all;
      __syncthreads();
    }
    if (threadIdx.x == 0) a.starts[a.B] = base;
    if constexpr (STEP == 64) {
      __syncthreads();
      list_runs(a, base, held, kRoom, a.B <= kRoom);
    }
    return;
  }
  const int hd = l.Dn + l.Dr, row = l.Dc + l.Dr, c0 = blockIdx.x * 64;
  const __half* w = l.w + (size_t)h * (l.Dn + l.Dv) * l.Dc + c0;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  // (the weights, the first queries and q_r are asked for together)
  U4 wl[DN / 32];
#pragma unroll
  for (int i = 0; i < DN / 32; ++i) {
    const int e = threadIdx.x + 256 * i;
    wl[i] = ld16(w + (size_t)(e >> 3) * l.Dc + 8 * (e & 7));
  }
  h8 x[DN / 32];
  auto queries = [&](int bt) {
    const __half* q = l.q + ((size_t)min(bt + c, b1 - 1) * l.H + h) * hd + 8 * g;
#pragma unroll
    for (int k = 0; k < DN / 32; ++k) x[k] = ld_h8(q + 32 * k);
  };
  queries(b0);
  if (blockIdx.x == 0) {
    const int pieces = l.Dr / 8;
    for (int e = threadIdx.x; e < (b1 - b0) * pieces; e += 256) {
      const size_t r = (size_t)(b0 + e / pieces) * l.H + h;
      const int p = 8 * (e % pieces);
      const h8 v = ld_h8(l.q + r * hd + l.Dn + p);
      *reinterpret_cast<h8*>(a.ql + r * row + l.Dc + p) = STEP == 64 ? in_code_order(v) : v;
    }
  }
#pragma unroll
  for (int i = 0; i < DN / 32; ++i) {
    const int e = threadIdx.x + 256 * i, n = e >> 3;
    *reinterpret_cast<U4*>(wt + n * 128 + 16 * ((e & 7) ^ tile_key<8>(n))) = wl[i];
  }
  __syncthreads();
  h8 wa[DN / 32];
#pragma unroll
  for (int k = 0; k < DN / 32; ++k) {
    h4 part[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int n = 32 * k + 8 * g + 4 * r + (c >> 2), col = 16 * wave + 4 * (c & 3);
      part[r] = ld_tr(wt + n * 128 + 16 * ((col >> 3) ^ tile_key<8>(n)) + 2 * (col & 7));
    }
    wa[k] = join(part[0], part[1]);
  }
  for (int bt = b0; bt < b1; bt += 16) {
    const size_t r = (size_t)min(bt + c, b1 - 1) * l.H + h;
    f4 d = {};
#pragma unroll
    for (int k = 0; k < DN / 32; ++k) d = mfma16(wa[k], x[k], d);
    if (bt + 16 < b1) queries(bt + 16);
    h4 v = {(_Float16)d[0], (_Float16)d[1], (_Float16)d[2], (_Float16)d[3]};
    if constexpr (STEP == 64) {
      // (the 4-bit cache's products take eight elements in code order, 0, 4, 1, 5, 2, 6, 3, 7: of the two
      // lanes that have them one takes the first four, the other the last)
      typedef uint32_t u2 __attribute__((ext_vector_type(2)));
      const u2 w = __builtin_bit_cast(u2, v);
      const auto both = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
      const uint32_t x = both[0], y = both[1];
      v = __builtin_bit_cast(h4, u2{(x & 0xFFFFu) | y << 16, x >> 16 | (y & 0xFFFF0000u)});
    }
    if (bt + c < b1) *reinterpret_cast<h4*>(a.ql + r * row + c0 + 16 * wave + 4 * g) = v;
  }
}

// ---- joining the partial results --------------------------------------------------
// A query row's partial results are the runs of workgroups that the plan gave its items'
// tiles to. All their (m, l) are read at once, for the weights 2^(m - max) / sum; then the
// thread groups of Dc / 4 (four latent columns a thread) take them in turn. A row without
// any (no tokens) gives zeros. The latents are rounded to fp16 for the product with W_uv,
// which is fp16.
constexpr int kJoinMost = 1024;                          // (partial results of a row: at most the workgroups and its items)

template <int NT>
struct JoinShared {
  int first[16], upto[17];                               // of each item: first partial result, those up to it
  float weight[kJoinMost];
  f4 part[NT];
};
// The joined latents of one of `slices` slices of a row: its 4 i .. 4 i + 3 in threads
// i < Dc / (4 slices); the whole workgroup calls. keep: note the row's reference and 1 / sum,
// so that a token's weight is 2^(score log2(e) - reference) / sum.
template <int NT, int STEP>
__device__ __forceinline__ h4 join_row(const DecodeArgs& a, int row, int slice, int slices, bool keep,
                                       JoinShared<NT>& sh) {
  constexpr int NS = STEP / 16;
  const LatentArgs& l = a.l;
  const int b = row / l.H, h = row % l.H, M = a.p.rows, lane = threadIdx.x & 63;
  const int per = share(a), items = a.p.chunks + 1;
  if (threadIdx.x < kWave) {
    int w0 = 0, n = 0, index = 0;
    if (lane < items) {                                  // (the last item is the sequence's own)
      const Item it = lane == a.p.chunks ? own_item<STEP>(a, b, h / M, a.starts[b], clamp_len(a, a.kv_len[b]))
                                         : prefix_item<STEP>(a, lane, row / M);
      index = it.index;
      if (it.tiles > 0) {
        const int from = it.start + kItemCost;
        w0 = from / per;
        n = (from + it.tiles - 1) / per - w0 + 1;
      }
    }
    int up = n;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int v = __shfl_up(up, o, kWave);
      if (lane >= o) up += v;
    }
    if (lane < items) {
      sh.first[lane] = w0 + index;
      sh.upto[lane + 1] = up;
    }
    if (lane == 0) sh.upto[0] = 0;
  }
  __syncthreads();
  const int parts = sh.upto[items];
  auto seg_of = [&](int i, int& r) {                     // the i-th partial result: where it is, and its row there
    int k = 0;
    while (i >= sh.upto[k + 1]) ++k;
    r = k == items - 1 ? h % M : row % M;
    return (size_t)(sh.first[k] + i - sh.upto[k]);
  };
  // every wave forms the maximum and the sum for itself
  float top = -INFINITY, sum = 0.f;
  for (int i = lane; i < parts; i += kWave) {
    int r;
    const size_t seg = seg_of(i, r);
    top = fmaxf(top, a.part_ml[(seg * NS * M + r) * 2]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  for (int i = lane; i < parts; i += kWave) {
    int r;
    const size_t seg = seg_of(i, r);
    const float2 a0 = *reinterpret_cast<const float2*>(a.part_ml + (seg * NS * M + r) * 2);
    float l_of = a0.y;
#pragma unroll
    for (int k = 1; k < NS; ++k) l_of += a.part_ml[((seg * NS + k) * M + r) * 2 + 1];
    // (-inf: no score of it is above that, and its sum is 0, or NaN, which a weight of 0 keeps)
    const float w = a0.x == -INFINITY ? 0.f : exp2_fast(a0.x - top);
    sum += w * l_of;
    if (threadIdx.x < kWave) sh.weight[i] = w;
  }
  sum = wave_sum(sum);
  __syncthreads();
  const int cols = l.Dc / 4 / slices, groups = NT / cols, grp = threadIdx.x / cols;
  const int col = 4 * (slice * cols + threadIdx.x % cols);
  f4 o = {};
#pragma unroll 4
  for (int i = grp; i < parts; i += groups) {
    int r;
    const size_t seg = seg_of(i, r);
    const float w = sh.weight[i];
    if (w != 0.f) o += *reinterpret_cast<const f4*>(a.part_o + (seg * M + r) * l.Dc + col) * w;
  }
  sh.part[threadIdx.x] = o;
  __syncthreads();
  if (grp == 0)
    for (int k = 1; k < groups; ++k) o += sh.part[k * cols + threadIdx.x];
  const float inv = sum > 0.f ? 1.f / sum : sum != sum ? sum : 0.f;
  if (keep && threadIdx.x == 0)
    *reinterpret_cast<float2*>(a.row_ml + 2 * (size_t)row) = float2{top == -INFINITY ? INFINITY : top - kRaise, inv};
  return h4{(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
}

// With few rows 512 threads share a row's partial results, and its columns are cut into
// slices that are workgroups of their own (16 heads over 16,000 tokens, 250 partial results
// a row: the whole call in 34 us with four slices, 55 without); with many 128 do, so that
// more rows are on a CU at once (2048 rows: 13.4 us against 21; 32 rows: 14.6 against 5.9).
// Bound by the partial results' reads, which the decode launch has just left in the L2s.
template <int NT, int STEP>
__global__ void __launch_bounds__(NT) latent_join_kernel(DecodeArgs a) {
  __shared__ JoinShared<NT> sh;
  const int cols = a.l.Dc / 4 / gridDim.y, i = blockIdx.y * cols + threadIdx.x;
  const h4 v = join_row<NT, STEP>(a, blockIdx.x, blockIdx.y, gridDim.y, a.row_ml && blockIdx.y == 0, sh);
  if ((int)threadIdx.x < cols) *reinterpret_cast<h4*>(a.lat + (size_t)blockIdx.x * a.l.Dc + 4 * i) = v;
}

// ---- out of the latent space --------------------------------------------------------
// o_h = W_uv,h lat_h (48 sequences of 32 heads: 5.3 us, bound by latency as the way in is):
// 16 values of one head a workgroup, whose four waves split the
// latent columns and keep their weights in registers for all sequences. For one short
// sequence it joins its head's row itself (JOIN; the workgroups of a head do that over
// again): a launch less (16 heads over 100 tokens: the call in 15.6 us against 18.1; 500
// tokens: 17.3, 18.4; 1,000 tokens: 19.7, 18.6; two sequences of 500: 21.6, 18.4).
constexpr int kFusedTokens = 768;

template <int DC, bool JOIN, int STEP>
__device__ __forceinline__ void latent_up(const DecodeArgs& a, int tile, int h, int block) {
  constexpr int NT = 256, KS = DC / 128;
  __shared__ f4 red[4][kWave];
  __shared__ JoinShared<JOIN ? NT : 1> sh;
  __shared__ __attribute__((aligned(16))) _Float16 joined[JOIN ? DC : 8];
  const LatentArgs& l = a.l;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int v0 = tile * 16, b0 = block * 128, b1 = min(b0 + 128, a.B);
  h8 w[KS];
  const __half* wv = l.w + ((size_t)h * (l.Dn + l.Dv) + l.Dn + v0 + c) * DC + wave * (DC / 4) + 8 * g;
#pragma unroll
  for (int k = 0; k < KS; ++k) w[k] = ld_h8(wv + 32 * k);
  if constexpr (JOIN) {
    const h4 v = join_row<NT, STEP>(a, h, 0, 1, a.row_ml && tile == 0, sh);
    if (threadIdx.x < DC / 4) *reinterpret_cast<h4*>(&joined[4 * threadIdx.x]) = v;
    __syncthreads();
  }
  h8 x[KS];                                              // (the next 16 sequences' are asked for early)
  auto latents = [&](int bt) {
    const void* lat = a.lat + ((size_t)min(bt + c, b1 - 1) * l.H + h) * DC;
    if constexpr (JOIN) lat = joined;
#pragma unroll
    for (int k = 0; k < KS; ++k) x[k] = ld_h8(static_cast<const _Float16*>(lat) + wave * (DC / 4) + 32 * k + 8 * g);
  };
  latents(b0);
  for (int bt = b0; bt < b1; bt += 16) {
    const size_t r = (size_t)min(bt + c, b1 - 1) * l.H + h;
    f4 d = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) d = mfma16(w[k], x[k], d);
    if (bt + 16 < b1) latents(bt + 16);
    red[wave][lane] = d;
    __syncthreads();
    if (wave == 0 && bt + c < b1) {
      const f4 s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
      const h4 v = {(_Float16)s[0], (_Float16)s[1], (_Float16)s[2], (_Float16)s[3]};
      *reinterpret_cast<h4*>(l.out + r * l.Dv + v0 + 4 * g) = v;
    }
    __syncthreads();
  }
}

template <int DC, bool JOIN, int STEP>
__global__ void __launch_bounds__(256) latent_up_kernel(DecodeArgs a) {
  latent_up<DC, JOIN, STEP>(a, blockIdx.x, blockIdx.y, blockIdx.z);
}

inline bool joins_itself(const DecodeArgs& a) { return a.B == 1 && a.prefix_len == 0 && a.max_len <= kFusedTokens; }
inline dim3 up_grid(const DecodeArgs& a) { return dim3(a.l.Dv / 16, a.l.H, (a.B + 127) / 128); }

template <int STEP>
hipError_t launch_join(const DecodeArgs& a, hipStream_t st) {
  const int rows = a.B * a.l.H;
  if (rows > 2 * kCus)
    hipLaunchKernelGGL((latent_join_kernel<128, STEP>), dim3(rows), dim3(128), 0, st, a);
  else {
    // (the 4-bit cache's attention takes half the time, so the join's share counts: 16 rows of 250
    // partial results 9.8 us with eight slices, 11.3 with four; 32 rows of 47 6.4 with either)
    const int slices = STEP == 64 && rows <= kCus / 8 && a.l.Dc >= 256 ? 8 : rows <= kCus / 2 ? 4 : rows <= kCus ? 2 : 1;
    hipLaunchKernelGGL((latent_join_kernel<512, STEP>), dim3(rows, slices), dim3(512), 0, st, a);
  }
  return hipGetLastError();
}
template <int DC, int STEP>
hipError_t launch_up(const DecodeArgs& a, hipStream_t st) {
  const bool joins = joins_itself(a);
  if (!joins) {
    const hipError_t e = launch_join<STEP>(a, st);
    if (e != hipSuccess) return e;
  }
  auto kernel = joins ? latent_up_kernel<DC, true, STEP> : latent_up_kernel<DC, false, STEP>;
  hipLaunchKernelGGL(kernel, up_grid(a), dim3(256), 0, st, a);
  return hipGetLastError();
}

inline size_t round256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace
}  // namespace moe
