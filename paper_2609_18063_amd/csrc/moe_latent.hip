// Latent attention for single tokens, in its absorbed form, and the writes of the
// paged latent cache. Each cached token is one row (c, k_r): a latent c [Dc], from
// which every head's keys W_uk,h c and values W_uv,h c come, and one rotated key k_r
// [Dr] that all heads share. For a query (q_n, q_r) of head h
//   s_j = scale (q_n . W_uk,h c_j + q_r . k_r,j) = scale ((W_uk,h^T q_n) . c_j + q_r . k_r,j)
//   o   = sum_j p_j W_uv,h c_j                   = W_uv,h sum_j p_j c_j,   p = softmax(s)
// so with the query taken into the latent space once, all heads read the same row: the
// cache is read once for all of them, (Dc + Dr) 2 bytes a token.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "moe_decode.h"

namespace moe {
namespace {

constexpr int kChunks = 15;

// ---- cache writes -------------------------------------------------------------
// Block (t, 0) normalizes and rotates token t's row into its page; blocks (t, 1 ..)
// rotate the query, 8 halves a thread. One pass; bound by the bytes read and written (3,100
// tokens of 32 heads: 87 MB in 19 us, 4.6 TB/s; 16 tokens: 3.5 us, latency).
__global__ void __launch_bounds__(256) latent_append_kernel(AppendArgs a) {
  const LatentArgs& l = a.l;
  const int t = blockIdx.x, seq = a.seq[t], pos = a.pos[t], row = l.Dc + l.Dr;
  if (seq < 0) return;                                   // a padding row
  int32_t page = -1;
  const bool in = seq < l.n_seqs && pos >= 0 && pos < a.max_pos && pos / l.page < l.max_pages;
  if (in) page = l.table[seq * l.table_stride + pos / l.page];
  if (page < 0 || page >= l.n_pages) {
    if (blockIdx.y == 0 && threadIdx.x == 0 && l.status)
      atomicOr(l.status, in ? MOE_STATUS_BAD_PAGE : MOE_STATUS_BAD_INDEX);
    return;
  }
  const float2* cs = reinterpret_cast<const float2*>(a.rope) + (size_t)pos * (l.Dr / 2);
  if (blockIdx.y > 0) {
    rotate_query(a, t, blockIdx.y - 1, cs);
    return;
  }
  __shared__ float red[4];
  const float* kv = a.kv + (size_t)t * row;
  __half* to = a.pages + ((size_t)page * l.page + pos % l.page) * row;
  float2 v = {0.f, 0.f};                                 // two of Dc <= 512 a thread
  const int e = 2 * threadIdx.x;
  if (e < l.Dc) v = *reinterpret_cast<const float2*>(kv + e);
  const float s = wave_sum(fmaf(v.x, v.x, v.y * v.y));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  const float inv = 1.f / sqrtf((red[0] + red[1] + red[2] + red[3]) / (float)l.Dc + 1e-6f);
  if (e < l.Dc) {
    const float2 gm = __half22float2(*reinterpret_cast<const __half2*>(a.gamma + e));
    *reinterpret_cast<__half2*>(to + e) = __floats2half2_rn(v.x * inv * gm.x, v.y * inv * gm.y);
  }
  if (e < l.Dr) {
    const float2 x = *reinterpret_cast<const float2*>(kv + l.Dc + e), r = cs[threadIdx.x];
    *reinterpret_cast<__half2*>(to + l.Dc + e) =
        __floats2half2_rn(x.x * r.x - x.y * r.y, x.x * r.y + x.y * r.x);
  }
}

// ---- attention over the cache -------------------------------------------------------
// A workgroup takes its share of the line of tiles (32 tokens each), item by item. Half
// of its waves form the scores, transposed (tokens x query rows, a wave 16 of the tokens
// and, of four, half of the rows, with the query in registers), and the weights; the
// other half add up the weighted latents of the tile before, each its share of the latent
// columns, read transposed from the same LDS copy, and make the copies, two tiles ahead in
// four buffers. So the products of one tile run beside the exponentials of the next, with
// one barrier a tile. With few heads HBM bounds it (32 heads, 48 sequences, 378,000 tokens:
// 445 MB in 88 us, 5.05 TB/s), with many, or a shared prefix, the scores' chain of one wave
// (its products, exponentials and the barrier): 32 sequences of 64 heads on 12,000 shared
// tokens in 88 us, 0.62 PFLOP/s.
// The weights are taken against a reference per row (see kSlack), and rounded to fp16 for
// the product with the latents, which are fp16.
template <int DC, int DR, int MT>
struct DecodeShape {
  static constexpr int M = 16 * MT;
  static constexpr int WR = MT == 1 ? 1 : 2, RT = MT / WR;     // row blocks, 16-row tiles of a score wave
  static constexpr int NS = 2 * WR, NW = 2 * NS;               // score waves (as many add up), waves
  static constexpr int OWN = kStep / NS;                       // token rows that a wave of the others copies
  static constexpr int KS = (DC + DR) / 32, CT = DC / (16 * NS);
  static constexpr int LAT = kStep * DC * 2, BUF = LAT + kStep * DR * 2;
  static constexpr int PT = M * 64;                            // the weights of a tile
  static constexpr int LDS = 4 * BUF + 2 * PT + 3 * M * 4 + 32;
  // copies of a tile by one wave: latent rows LR at a time, rotated keys RR at a time
  static constexpr int LP = DC / 8, LR = kWave / LP, RP = DR / 8, RR = kWave / RP;
  static constexpr int LN = OWN / LR, RN = RR <= OWN ? OWN / RR : 1;
  static_assert(OWN % LR == 0 && OWN <= 16, "rows of a wave's copies lie in one group");
};

template <int DC, int DR, int MT>
__global__ void __launch_bounds__((64 * DecodeShape<DC, DR, MT>::NW)) latent_decode_kernel(DecodeArgs a) {
  using S = DecodeShape<DC, DR, MT>;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  char* pt = lds + 4 * S::BUF;                                  // weights [2][M][32] halves
  float* smax = reinterpret_cast<float*>(pt + 2 * S::PT);       // [2][M], by token half
  float* skeep = smax + 2 * S::M;                               // [M]
  int* passed = reinterpret_cast<int*>(skeep + S::M);           // [2]: the last step with a row past its reference
  const LatentArgs& l = a.l;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4;
  const int wt = wave % 2, wr = wave / 2, wo = wave - S::NS;    // token half, row block; share of the columns
  // neighbours on the line share a chiplet and its L2
  const int wg = (blockIdx.x % 8) * (a.p.wgs / 8) + blockIdx.x / 8;
  Walk<kStep> at;
  at.begin(a, wg);
  const float unit = l.scale * kLog2e;
  const int shift = 31 - __clz(l.page);
  // 16-token group `grp` (0 or 1) of a tile, from its first token (past the end: the last group)
  auto group = [&](const Item& it, int tile, int grp) { return min(it.tok0 + tile * kStep + 16 * grp, it.last & ~15); };
  auto page_of = [&](const Item& it, int tile, int grp) { return ld_scalar(it.pages + (group(it, tile, grp) >> shift)); };
  auto known = [&](int page) { return page >= 0 && page < l.n_pages; };
  if (threadIdx.x < 2) passed[threadIdx.x] = -1;

  if (wave < S::NS) {
    __builtin_amdgcn_s_setprio(2);
    bool more = at.next(a);
    h8 q[S::RT][S::KS];
    auto queries = [&]() {
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        const size_t row = at.it.row0 + min((wr * S::RT + r) * 16 + c, at.it.rows - 1);
#pragma unroll
        for (int k = 0; k < S::KS; ++k) q[r][k] = ld_h8(a.ql + row * (DC + DR) + 32 * k + 8 * g);
      }
    };
    float sum[S::RT], m[S::RT], ref[S::RT];                     // m: the reference, unscaled; ref: m unit - kRaise, or 0
    auto start = [&]() {
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        m[r] = -INFINITY;
        sum[r] = ref[r] = 0.f;
      }
    };
    int page = 0;
    if (more) {
      queries();
      page = page_of(at.it, at.first, wt);
    }
    start();
    vm_drain();
    lds_barrier();
    // step u: the scores of tile u, the k-th of its item
    for (int u = 0, k = 0; more; ++u) {
      const char* buf = lds + (u & 3) * S::BUF;
      f4 x[S::RT] = {};
      const int tok = wt * 16 + c;
#pragma unroll
      for (int k = 0; k < S::KS; ++k) {
        const char* p = k < DC / 32
                            ? buf + tok * DC * 2 + 256 * (k >> 2) + 16 * ((4 * (k & 3) + g) ^ tile_key<S::LP>(c))
                            : buf + S::LAT + tok * DR * 2 + 16 * ((4 * (k - DC / 32) + g) ^ tile_key<S::RP>(c));
        const h8 kk = ld_h8(p);
#pragma unroll
        for (int r = 0; r < S::RT; ++r) x[r] = mfma16(kk, q[r][k], x[r]);
      }
      const bool lost = !known(page);
      const int left = at.it.last - (at.it.tok0 + (at.first + k) * kStep + 16 * wt);  // tokens of the group, less one
      const size_t seg = (size_t)wg + at.it.index;
      // (the next item's query is asked for while this step's weights are formed)
      const bool ends = ++k == at.n;
      if (ends) {
        k = 0;
        more = at.next(a);
        if (more) queries();
      }
      if (more) page = page_of(at.it, at.first + k, wt);
      if (lost || left < 15) {
        const int most = lost ? -1 : left - 4 * g;
#pragma unroll
        for (int r = 0; r < S::RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e > most) x[r][e] = -INFINITY;
      }
      // the weights, where the latents are read in the same order: of the tile's tokens,
      // 16 v + 4 g .. + 3 at 8 g + 4 v
      float add[S::RT];
      auto weights = [&]() {
#pragma unroll
        for (int r = 0; r < S::RT; ++r) {
          h4 p;
          add[r] = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = exp2_fast(fmaf(x[r][e], unit, -ref[r]));
            add[r] += v;
            p[e] = (_Float16)v;
          }
          *reinterpret_cast<h4*>(pt + (u & 1) * S::PT + ((wr * S::RT + r) * 16 + c) * 64 + 16 * (g ^ tile_key<4>(c)) +
                                 8 * wt) = p;
        }
      };
      weights();
      bool far = false;
      float top[S::RT];
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        top[r] = fmaxf(fmaxf(x[r][0], x[r][1]), fmaxf(x[r][2], x[r][3]));
        far = far || (top[r] - m[r]) * unit > kSlack;           // (no token so far: any score is)
      }
      if (__any(far) && lane == 0) passed[u & 1] = u;
      lds_barrier();
      if (__builtin_amdgcn_readfirstlane(passed[u & 1]) == u) {
        // every row that is past its reference takes its largest score as the new one (the others
        // keep theirs: a row's roundings are its own)
#pragma unroll
        for (int r = 0; r < S::RT; ++r) {
          top[r] = col_max(top[r]);
          if (g == 0) smax[wt * S::M + (wr * S::RT + r) * 16 + c] = top[r];
        }
        lds_barrier();
#pragma unroll
        for (int r = 0; r < S::RT; ++r) {
          const int row = (wr * S::RT + r) * 16 + c;
          const float most = max3(m[r], top[r], smax[(1 - wt) * S::M + row]);
          float keep = 1.f;
          if ((most - m[r]) * unit > kSlack) {
            const float now = most * unit - kRaise;
            keep = m[r] == -INFINITY ? 0.f : exp2_fast(ref[r] - now);
            m[r] = most;
            sum[r] *= keep;
            ref[r] = now;
          }
          if (g == 0 && wt == 0) skeep[row] = keep;
        }
        weights();
        lds_barrier();
      }
#pragma unroll
      for (int r = 0; r < S::RT; ++r) sum[r] += add[r];
      if (ends) {
#pragma unroll
        for (int r = 0; r < S::RT; ++r) {
          sum[r] = col_sum(sum[r]);
          if (g == 0)
            *reinterpret_cast<float2*>(a.part_ml + ((seg * 2 + wt) * S::M + (wr * S::RT + r) * 16 + c) * 2) =
                float2{m[r] * unit, sum[r]};
        }
        start();
      }
    }
    return;
  }

  // this wave copies rows own0 .. own0 + OWN - 1 of a tile and its part of the rotated keys
  // (where a copy of those is several waves' rows, one of them takes it)
  const int own0 = S::OWN * wo, grp = own0 / 16;
  const bool ropes = S::RR <= S::OWN || own0 % S::RR == 0;
  const uint32_t at0 = lds_at(lds);
  auto copy = [&](const Item& it, int tile, int buf, int page) {
    const int base = group(it, tile, grp);
    if (!known(page)) {
      // (zeros, whose scores are masked; the waits for copies find fewer than they allow)
      if (lane == 0 && l.status) atomicOr(l.status, MOE_STATUS_BAD_PAGE);
      char* lat = lds + buf * S::BUF;
      for (int e = lane; e < S::OWN * DC / 8; e += kWave) *reinterpret_cast<U4*>(lat + own0 * DC * 2 + 16 * e) = U4{};
      for (int e = lane; e < S::OWN * DR / 8; e += kWave)
        *reinterpret_cast<U4*>(lat + S::LAT + own0 * DR * 2 + 16 * e) = U4{};
      vm_wait<0>();
      return;
    }
    const uint32_t lat = at0 + buf * S::BUF, rope = lat + S::LAT;
    const char* from = reinterpret_cast<const char*>(l.pages) +
                       ((size_t)page * l.page + (base & (l.page - 1))) * (DC + DR) * 2;
    int ln = lane;                                              // (offsets formed here, not held in registers)
    asm volatile("" : "+v"(ln));
    auto rows = [&](auto at_most) {
#pragma unroll
      for (int j = 0; j < S::LN; ++j) {
        const int r0 = j * S::LR, r = S::LR == 1 ? r0 : r0 + ln / S::LP;
        dma16(from, at_most((own0 & 15) + r) * ((DC + DR) * 2) + 16 * ((ln % S::LP) ^ tile_key<S::LP>(own0 + r)),
              lat + (own0 + r0) * DC * 2);
      }
      if (ropes)
#pragma unroll
        for (int j = 0; j < S::RN; ++j) {
          const int r0 = j * S::RR, r = r0 + ln / S::RP;
          dma16(from + DC * 2,
                at_most((own0 & 15) + r) * ((DC + DR) * 2) + 16 * ((ln % S::RP) ^ tile_key<S::RP>(own0 + r)),
                rope + (own0 + r0) * DR * 2);
        }
    };
    const int most = it.last - base;                            // rows past the end repeat the last one
    if (most >= 15)
      rows([](int r) { return r; });
    else
      rows([most](int r) { return min(r, most); });
  };
  // the tiles asked for so far, and the next one
  Walk<kStep> ask = at;
  int asked = 0, k = 0;
  bool more = ask.next(a);
  int page = more ? page_of(ask.it, ask.first, grp) : 0;
  auto ask_next = [&]() {
    if (!more) return false;
    copy(ask.it, ask.first + k, asked & 3, page);
    ++asked;
    if (++k == ask.n) {
      k = 0;
      more = ask.next(a);
    }
    if (more) page = page_of(ask.it, ask.first + k, grp);
    return true;
  };
  ask_next();
  ask_next();
  f4 o[S::CT][MT] = {};
  vm_drain();
  lds_barrier();
  int left = 0;                                                 // tiles of the item that are not added up yet
  // step u: the latents of tile u - 1, and tile u + 2 is asked for; the last step has no scores beside it
  for (int u = 0;; ++u) {
    const bool newer = ask_next();
    bool stored = false;
    if (u > 0) {
      if (left == 0) {
        at.next(a);
        left = at.n;
      }
      const char* buf = lds + ((u - 1) & 3) * S::BUF;
      h8 p[MT];
#pragma unroll
      for (int r = 0; r < MT; ++r)
        p[r] = ld_h8(pt + ((u - 1) & 1) * S::PT + (16 * r + c) * 64 + 16 * (g ^ tile_key<4>(c)));
#pragma unroll
      for (int k = 0; k < S::CT; ++k) {
        h4 part[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int t0 = 4 * g + (c >> 2), col = 16 * (wo * S::CT + k) + 4 * (c & 3);
          part[v] = ld_tr(buf + (16 * v + t0) * DC * 2 + 16 * ((col >> 3) ^ tile_key<S::LP>(t0)) + 2 * (col & 7));
        }
        const h8 v = join(part[0], part[1]);
#pragma unroll
        for (int r = 0; r < MT; ++r) o[k][r] = mfma16(v, p[r], o[k][r]);
      }
      if (--left == 0) {
        const size_t seg = (size_t)wg + at.it.index;
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
          for (int k = 0; k < S::CT; ++k) {
            *reinterpret_cast<f4*>(a.part_o + (seg * S::M + 16 * r + c) * DC + 16 * (wo * S::CT + k) + 4 * g) = o[k][r];
            o[k][r] = f4{};
          }
        stored = true;
      }
    }
    if (u >= asked) break;
    // tile u + 1 is there: all but this step's copies and, behind them, the stores (16 bytes
    // a lane each: no fewer than these)
    constexpr int ST = S::CT * MT;
    if (!newer)
      vm_wait<0>();
    else if (ropes && stored)
      vm_wait<S::LN + S::RN + ST>();
    else if (ropes)
      vm_wait<S::LN + S::RN>();
    else if (stored)
      vm_wait<S::LN + ST>();
    else
      vm_wait<S::LN>();
    lds_barrier();
    if (__builtin_amdgcn_readfirstlane(passed[u & 1]) == u) {
      lds_barrier();
      lds_barrier();
#pragma unroll
      for (int r = 0; r < MT; ++r) {
        const float keep = skeep[16 * r + c];
#pragma unroll
        for (int k = 0; k < S::CT; ++k) o[k][r] *= keep;
      }
    }
  }
}

int tiles_host(int len) { return (len + kStep - 1) / kStep; }

template <int DC, int DR, int MT>
hipError_t launch_attention(const DecodeArgs& a, hipStream_t st) {
  constexpr int lds = DecodeShape<DC, DR, MT>::LDS;
  static_assert(lds <= 160 * 1024, "LDS of a CU");
  auto kernel = latent_decode_kernel<DC, DR, MT>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(a.p.wgs), dim3(64 * DecodeShape<DC, DR, MT>::NW), lds, st, a);
  return hipGetLastError();
}
template <int DC, int DR>
hipError_t launch_attention(const DecodeArgs& a, hipStream_t st) {
  if (a.p.rows == 16) return launch_attention<DC, DR, 1>(a, st);
  if (a.p.rows == 32) return launch_attention<DC, DR, 2>(a, st);
  return launch_attention<DC, DR, 4>(a, st);
}
template <int DC>
hipError_t launch_attention(const DecodeArgs& a, hipStream_t st) {
  return a.l.Dr == 64 ? launch_attention<DC, 64>(a, st) : launch_attention<DC, 32>(a, st);
}

}  // namespace

DecodePlan decode_plan(int H, int Dc, int Dr, int B, int max_len, int prefix_len) {
  DecodePlan p{};
  const int pt = tiles_host(prefix_len);
  // The fewest rows that hold a sequence's heads (more would be idle in its own tiles), and
  // with a prefix as many more as keep its tiles, which all sequences' rows share, under 12 a
  // CU (16 heads, 8 sequences, 4,000 shared tokens: 29.8 us with 16 rows, 40.8 with 64; 32
  // sequences, 12,000 tokens: 99.7, 52.6; 32 heads, 16 sequences, 8,000: 47.3 with 32, 45.4).
  p.rows = H <= 16 ? 16 : H <= 32 ? 32 : 64;
  while (p.rows < 64 && (int64_t)pt * ((B * H + p.rows - 1) / p.rows) > 12 * kCus) p.rows *= 2;
  p.head_blocks = (H + p.rows - 1) / p.rows;
  p.row_blocks = prefix_len > 0 ? (B * H + p.rows - 1) / p.rows : 0;
  // (one workgroup a CU has the whole LDS and fewer partial results; two pay for the small
  // tiles of 128 latents: 64 sequences of 4,000 tokens 40.1 us against 44.9, with 256 latents,
  // 32 heads, 32 of 6,000 47.7 against 40.9)
  const int wgs = kCus * (Dc <= 128 ? 2 : 1);
  const long long own = (long long)B * p.head_blocks * (max_len > 0 ? tiles_host(max_len) + kItemCost : 0);
  // A share of fewer tiles leaves more partial results than it saves time: about
  // sqrt(tiles) / 6 of a sequence (one of 16,000 tokens, 16 heads: 34 us with 2, 29.6 with 4,
  // 30.5 with 6; of 3,000: 20.4 with 2, 21.7 with 4).
  p.least = std::max(1, (int)(0.18 * std::sqrt((double)tiles_host(max_len)) + 0.5));
  if (prefix_len > 0) {
    // Token chunks of the prefix such that a row block of a chunk is just one workgroup's
    // share: as many as leave workgroups enough for the sequences' own tiles. Then no
    // workgroup has two partial results of the prefix, and the workgroups of a chiplet read
    // the same tokens, which its L2 holds.
    p.chunks = 1;
    for (int c = kChunks; c > 1; --c) {
      const int item = (pt + c - 1) / c + kItemCost;
      if (c <= pt && (long long)c * p.row_blocks + (own + item - 1) / item <= wgs && c * p.row_blocks * 2 >= wgs) {
        p.chunks = c;
        p.least = item;
        break;
      }
    }
    p.chunk_tiles = (pt + p.chunks - 1) / p.chunks;
    p.chunks = (pt + p.chunk_tiles - 1) / p.chunk_tiles;
  }
  p.prefix_places = (pt + p.chunks * kItemCost) * p.row_blocks;
  const long long tiles = (long long)pt * p.row_blocks + (long long)B * p.head_blocks * tiles_host(max_len);
  p.wgs = (int)std::min<long long>(wgs, (std::max<long long>(tiles, 1) + 7) / 8 * 8);
  const size_t rows = (size_t)B * H, parts = (size_t)p.wgs + (size_t)p.chunks * p.row_blocks + (size_t)B * p.head_blocks;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += round256(bytes);
    return o;
  };
  p.ql = take(rows * (Dc + Dr) * 2);
  p.lat = take(rows * Dc * 2);
  p.starts = take(((size_t)B + 1) * 4);
  p.part_o = take(parts * p.rows * Dc * 4);
  p.part_ml = take(parts * p.rows * 16);
  p.total = off;
  return p;
}

hipError_t launch_latent_append(const AppendArgs& a, hipStream_t st) {
  const int n = a.l.q ? a.l.H * (a.l.Dn + a.l.Dr) : 0;
  hipLaunchKernelGGL(latent_append_kernel, dim3(a.T, 1 + (n + 2047) / 2048), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_latent_decode(const DecodeArgs& a, hipStream_t st) {
  const LatentArgs& l = a.l;
  const dim3 ga(l.Dc / 64 + 1, l.H, (a.B + 63) / 64);
  if (l.Dn == 128)
    hipLaunchKernelGGL((latent_absorb_kernel<128, kStep>), ga, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((latent_absorb_kernel<64, kStep>), ga, dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = l.Dc == 512 ? launch_attention<512>(a, st) : l.Dc == 256 ? launch_attention<256>(a, st) : launch_attention<128>(a, st);
  if (e != hipSuccess) return e;
  return l.Dc == 512 ? launch_up<512, kStep>(a, st) : l.Dc == 256 ? launch_up<256, kStep>(a, st) : launch_up<128, kStep>(a, st);
}

// ---- arguments of the calls --------------------------------------------------------

int latent_cache_check(const moe_latent_spec* s, const moe_latent_cache* c) {
  const int rc = moe_latent_spec_check(s);
  if (rc != MOE_OK) return rc;
  if (!c || !c->pages || c->n_pages < 1 || c->n_seqs < 1 || !c->table || c->max_pages < 1 ||
      c->table_stride < c->max_pages || c->reserved != 0 ||
      (int64_t)c->max_pages * s->page_tokens > (int64_t(1) << 30))
    return MOE_EINVAL;
  if ((reinterpret_cast<uintptr_t>(c->pages) & 15) || (reinterpret_cast<uintptr_t>(c->table) & 3)) return MOE_EALIGN;
  return MOE_OK;
}

LatentArgs latent_args(const moe_latent_spec* s, const moe_latent_cache* c) {
  LatentArgs l{};
  l.H = s->heads;
  l.Dc = s->d_latent;
  l.Dr = s->d_rope;
  l.Dn = s->d_nope;
  l.Dv = s->d_v;
  l.page = s->page_tokens;
  l.scale = s->scale;
  l.pages = static_cast<const __half*>(c->pages);
  l.n_pages = c->n_pages;
  l.n_seqs = c->n_seqs;
  l.max_pages = c->max_pages;
  l.table = c->table;
  l.table_stride = c->table_stride;
  return l;
}

}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int kMaxLen = 1 << 26, kMaxBatch = 1 << 16;

bool decode_shape_ok(const moe_latent_spec* s, int B, int max_len, int prefix_len) {
  if (moe_latent_spec_check(s) != MOE_OK || B < 0 || B > kMaxBatch || max_len < 0 || max_len > kMaxLen ||
      prefix_len < 0 || prefix_len > kMaxLen)
    return false;
  // tiles on the plan's line, with their row blocks (16 query rows and 32 tokens the smallest)
  const int64_t rows = ((int64_t)B * s->heads + 15) / 16 + B;
  return rows * (((int64_t)max_len + prefix_len + 31) / 32 + 32) < (int64_t(1) << 30);
}

}  // namespace

extern "C" {

int moe_latent_spec_check(const moe_latent_spec* s) {
  if (!s) return MOE_EINVAL;
  if (s->heads < 1 || s->heads > 128) return MOE_EINVAL;
  if (s->d_latent != 128 && s->d_latent != 256 && s->d_latent != 512) return MOE_EINVAL;
  if (s->d_rope != 32 && s->d_rope != 64) return MOE_EINVAL;
  if ((s->d_nope != 64 && s->d_nope != 128) || (s->d_v != 64 && s->d_v != 128)) return MOE_EINVAL;
  const int p = s->page_tokens;
  if (p < 16 || p > 1024 || (p & (p - 1))) return MOE_EINVAL;
  if (!(s->scale > 0.f) || s->scale > 1e4f) return MOE_EINVAL;
  return s->reserved[0] == 0 && s->reserved[1] == 0 ? MOE_OK : MOE_EINVAL;
}

int moe_latent_append(const moe_latent_spec* spec, const moe_latent_cache* cache, const float* kv, const void* gamma_f16,
                      const float* rope, int max_pos, const int32_t* seq, const int32_t* pos, int T, const void* q_f16,
                      void* q_out_f16, uint32_t* status, void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (T < 0 || T > (1 << 22) || max_pos < 1 || (!q_f16) != (!q_out_f16)) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!kv || !gamma_f16 || !rope || !seq || !pos) return MOE_EINVAL;
  if (misaligned(kv, 16) || misaligned(gamma_f16, 16) || misaligned(rope, 16) || misaligned(seq, 4) ||
      misaligned(pos, 4) || misaligned(q_f16, 16) || misaligned(q_out_f16, 16) || misaligned(status, 4))
    return MOE_EALIGN;
  moe::AppendArgs a{};
  a.l = moe::latent_args(spec, cache);
  a.l.q = static_cast<const __half*>(q_f16);
  a.l.status = status;
  a.kv = kv;
  a.gamma = static_cast<const __half*>(gamma_f16);
  a.rope = rope;
  a.max_pos = max_pos;
  a.T = T;
  a.seq = seq;
  a.pos = pos;
  a.pages = static_cast<__half*>(cache->pages);
  a.q_out = static_cast<__half*>(q_out_f16);
  return moe::launch_latent_append(a, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

size_t moe_latent_decode_workspace_bytes(const moe_latent_spec* s, int B, int max_len, int prefix_len) {
  if (!decode_shape_ok(s, B, max_len, prefix_len)) return 0;
  return moe::decode_plan(s->heads, s->d_latent, s->d_rope, B < 1 ? 1 : B, max_len, prefix_len).total;
}

int moe_latent_decode(const moe_latent_spec* spec, const moe_latent_cache* cache, const void* w_kvb_f16,
                      const void* q_f16, int B, const int32_t* kv_len, int max_len, const int32_t* prefix_pages,
                      int prefix_len, void* out_f16, uint32_t* status, void* workspace, size_t workspace_bytes,
                      void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (!decode_shape_ok(spec, B, max_len, prefix_len) || B > cache->n_seqs) return MOE_EINVAL;
  if (B == 0) return MOE_OK;
  if (!w_kvb_f16 || !q_f16 || !kv_len || !out_f16 || !workspace || (prefix_len > 0 && !prefix_pages)) return MOE_EINVAL;
  if (misaligned(w_kvb_f16, 16) || misaligned(q_f16, 16) || misaligned(kv_len, 4) || misaligned(prefix_pages, 4) ||
      misaligned(out_f16, 16) || misaligned(status, 4) || misaligned(workspace, 16))
    return MOE_EALIGN;
  moe::DecodeArgs a{};
  a.l = moe::latent_args(spec, cache);
  a.l.w = static_cast<const __half*>(w_kvb_f16);
  a.l.q = static_cast<const __half*>(q_f16);
  a.l.out = static_cast<__half*>(out_f16);
  a.l.status = status;
  a.B = B;
  a.max_len = max_len;
  a.prefix_len = prefix_len;
  a.kv_len = kv_len;
  a.prefix = prefix_len > 0 ? prefix_pages : nullptr;
  a.p = moe::decode_plan(a.l.H, a.l.Dc, a.l.Dr, B, max_len, prefix_len);
  if (workspace_bytes < a.p.total) return MOE_ENOMEM;
  char* ws = static_cast<char*>(workspace);
  a.ql = reinterpret_cast<__half*>(ws + a.p.ql);
  a.lat = reinterpret_cast<__half*>(ws + a.p.lat);
  a.starts = reinterpret_cast<int32_t*>(ws + a.p.starts);
  a.part_o = reinterpret_cast<float*>(ws + a.p.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + a.p.part_ml);
  return moe::launch_latent_decode(a, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
