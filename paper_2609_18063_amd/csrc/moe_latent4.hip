// Latent attention for single tokens over a cache held in 4 bits (moe_latent4.h), the
// writes of that cache, and rows read back from it. The formulas are moe_latent.hip's; a
// cached row is (Dc + Dr) / 2 + 4 (Dc / 64 + 1) bytes instead of 2 (Dc + Dr), 324 instead of
// 1152 for 512 + 64.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "moe_decode.h"
#include "moe_latent4.h"

namespace moe {
namespace {

// ---- cache writes -------------------------------------------------------------
// Of a group: s = fp16((hi - lo) / 15), z = fp16(lo + 8 s), q = rint((v - z) / s) + 8. The
// values are formed in 64 bits, as a code beside a border goes one way or the other by the
// last bit: so a row's codes are those of its definition, but for exact ties.
struct Append4Args {
  AppendArgs a;                  // (a.pos: the angle's position)
  const int32_t* slot;           // [T]: the place in the sequence
  char* pages;
};

// op over 8 or 64 lanes, by lane moves (a trip through LDS for each of a double's halves costs
// more than the sums); every lane has the result.
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  return __hiloint2double(dpp_i<CTRL>(0, __double2hiint(v)), dpp_i<CTRL>(0, __double2loint(v)));
}
template <int LANES, typename Op>
__device__ __forceinline__ double over_lanes(double v, Op op) {
  v = op(v, dpp_d<0xB1>(v));
  v = op(v, dpp_d<0x4E>(v));
  v = op(v, dpp_d<0x141>(v));
  if constexpr (LANES == 64) {
    auto both = [&](auto lo, auto hi) { return op(__hiloint2double(hi[0], lo[0]), __hiloint2double(hi[1], lo[1])); };
    v = op(v, dpp_d<0x140>(v));
    uint32_t lo = __double2loint(v), hi = __double2hiint(v);
    v = both(__builtin_amdgcn_permlane16_swap(lo, lo, false, false), __builtin_amdgcn_permlane16_swap(hi, hi, false, false));
    lo = __double2loint(v), hi = __double2hiint(v);
    v = both(__builtin_amdgcn_permlane32_swap(lo, lo, false, false), __builtin_amdgcn_permlane32_swap(hi, hi, false, false));
  }
  return v;
}

// Eight neighbouring values of a group a lane, eight lanes a group; the codes of the lane's.
__device__ __forceinline__ uint32_t group_codes(const double (&v)[8], __half& s, __half& z) {
  auto lower = [](double v, double o) { return o < v ? o : v; };
  auto upper = [](double v, double o) { return o > v ? o : v; };
  double lo = v[0], hi = v[0];
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = lower(lo, v[i]);
    hi = upper(hi, v[i]);
    odd = odd || !isfinite(v[i]);
  }
  lo = over_lanes<8>(lo, lower);
  hi = over_lanes<8>(hi, upper);
  odd = __ballot(odd) >> (threadIdx.x & 56) & 0xFF;
  // (rounded by way of fp32, as defined: the compiler would make one rounding of the two)
  auto half = [](double v) {
    float f = (float)v;
    asm("" : "+v"(f));
    return __float2half_rn(f);
  };
  s = half((hi - lo) / 15.0);
  const double step = (double)__half2float(s);
  z = half(lo + 8.0 * step);
  // (a value that is not finite, or beyond fp16, makes NaN of its group)
  if (odd || !isfinite(__half2float(s)) || !isfinite(__half2float(z))) s = z = __ushort_as_half(0x7E00);
  const double base = (double)__half2float(z), div = step == 0.0 ? 1.0 : step, inv = 1.0 / div;
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double n = (v[i] - base) * inv, r = rint(n);
    if (fabs(fabs(n - r) - 0.5) < 1e-9) r = rint((v[i] - base) / div);  // (beside a border: as defined)
    codes |= (uint32_t)(int)fmin(fmax(r + 8.0, 0.0), 15.0) << 4 * i;
  }
  return codes;
}

// Blocks (., 0) normalize, rotate and quantize rows into their pages, a wave a token's: of its groups
// eight lanes one, eight values a lane (with two a thread, 256 threads a token, the reductions and
// quotients were four times as many: 3,100 tokens in 24.0 us). Blocks (t, 1 ..) rotate token t's query; the
// grid is theirs, so that of the blocks (., 0) three in four find no token. What a row's wave reads is asked
// for before the page is known. Most of the bytes are the queries' (3,100 tokens of 32 heads: 84 MB in 21.5 us, 3.9
// of a copy's 5.15 TB/s; 16 tokens: 4.8 us, latency and the 64-bit quotients).
__global__ void __launch_bounds__(256) latent4_append_kernel(Append4Args b) {
  const AppendArgs& a = b.a;
  const LatentArgs& l = a.l;
  const int lane = threadIdx.x & 63, t = blockIdx.y ? blockIdx.x : blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.T) return;
  const int seq = a.seq[t], pos = a.pos[t], slot = b.slot[t];
  const int G = l.Dc / 64 + 1, grp = lane >> 3, e = 8 * lane;
  const float* kv = a.kv + (size_t)t * (l.Dc + l.Dr);
  float x[8] = {}, y[8] = {};                            // of a latent group, or the key's
  h8 gm = {};
  const int key = 8 * (lane & 7) & (l.Dr - 1);           // (32 values: lanes 4 .. 7 have them again)
  if (blockIdx.y == 0) {
    auto read = [](float (&to)[8], const float* from) {
      const f4 p = *reinterpret_cast<const f4*>(from), q = *reinterpret_cast<const f4*>(from + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        to[i] = p[i];
        to[4 + i] = q[i];
      }
    };
    if (e < l.Dc) {
      read(x, kv + e);
      gm = ld_h8(a.gamma + e);
    }
    read(y, kv + l.Dc + key);
  }
  if (seq < 0) return;                                   // a padding row
  int32_t page = -1;
  const bool in = seq < l.n_seqs && pos >= 0 && pos < a.max_pos && slot >= 0 && slot / l.page < l.max_pages;
  if (in) page = l.table[seq * l.table_stride + slot / l.page];
  if (page < 0 || page >= l.n_pages) {
    if (blockIdx.y == 0 && lane == 0 && l.status) atomicOr(l.status, in ? MOE_STATUS_BAD_PAGE : MOE_STATUS_BAD_INDEX);
    return;
  }
  const float2* cs = reinterpret_cast<const float2*>(a.rope) + (size_t)pos * (l.Dr / 2);
  if (blockIdx.y > 0) {
    rotate_query(a, t, blockIdx.y - 1, cs);
    return;
  }
  const Page4 p4 = page4(l.Dc, l.Dr, l.page);
  char* to = b.pages + (size_t)page * p4.bytes;
  const int at = slot & (l.page - 1);
  __half* s_to = reinterpret_cast<__half*>(to + p4.steps) + at;
  float2 r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = cs[key / 2 + i];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += (double)x[i] * x[i];
  sum = over_lanes<64>(sum, [](double p, double q) { return p + q; });
  const double inv = 1.0 / sqrt(sum / (double)l.Dc + 1e-6);
  double v[8];
  auto store = [&](int group, bool holds) {
    __half s, z;
    const uint32_t codes = group_codes(v, s, z);
    if (!holds) return;
    *reinterpret_cast<uint32_t*>(group < G - 1 ? to + at * (l.Dc / 2) + e / 2 : to + p4.keys + at * (l.Dr / 2) + key / 2) = codes;
    if ((lane & 7) == 0) {
      s_to[group * l.page] = s;
      s_to[(G + group) * l.page] = z;
    }
  };
  auto turned = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = (double)y[2 * i] * r[i].x - (double)y[2 * i + 1] * r[i].y;
      v[2 * i + 1] = (double)y[2 * i] * r[i].y + (double)y[2 * i + 1] * r[i].x;
    }
  };
  // (up to 256 latents the key's lanes are the ones behind the latents', else the first ones again)
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = x[i] * inv * (double)gm[i];
  const bool keyed = 8 * (lane & 7) < l.Dr;
  if (grp == G - 1) turned();
  store(min(grp, G - 1), grp < G - 1 || (grp == G - 1 && keyed));
  if (G - 1 >= 8) {
    turned();
    store(G - 1, grp == 0 && keyed);
  }
}

// Rows as fp16, each value rounded once; eight a thread. Bound by latency (16 rows 3.1 us, 3,100 4.2).
__global__ void __launch_bounds__(256) latent4_read_kernel(LatentArgs l, const int32_t* seq, const int32_t* slot, int T,
                                                           __half* rows) {
  const int row = l.Dc + l.Dr, per = row / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(i / per), e = 8 * (int)(i % per);
  if (t >= T) return;
  const int b = seq[t], at = slot[t];
  if (b < 0) return;
  int32_t page = -1;
  const bool in = b < l.n_seqs && at >= 0 && at / l.page < l.max_pages;
  if (in) page = l.table[b * l.table_stride + at / l.page];
  if (page < 0 || page >= l.n_pages) {
    if (e == 0 && l.status) atomicOr(l.status, in ? MOE_STATUS_BAD_PAGE : MOE_STATUS_BAD_INDEX);
    return;
  }
  const Page4 p4 = page4(l.Dc, l.Dr, l.page);
  const char* from = reinterpret_cast<const char*>(l.pages) + (size_t)page * p4.bytes;
  const int k = at & (l.page - 1), G = l.Dc / 64 + 1, grp = min(e / 64, G - 1);
  const char* code = e < l.Dc ? from + k * (l.Dc / 2) + e / 2 : from + p4.keys + k * (l.Dr / 2) + (e - l.Dc) / 2;
  const _Float16* s = reinterpret_cast<const _Float16*>(from + p4.steps) + (size_t)grp * l.page + k;
  const h8 v = values8(*reinterpret_cast<const uint32_t*>(code), splat8(s[0]), splat8(s[(size_t)G * l.page]), code_bits());
  *reinterpret_cast<h8*>(rows + (size_t)t * row + e) = in_value_order(v);
}

// ---- attention over the cache ---------------------------------------------------
// A workgroup takes its runs of tiles (64 tokens each) one after the other. The schedule is
// moe_latent.hip's: of eight waves four form the scores, transposed (tokens x query rows), and
// the weights of a tile, the other four add up the weighted latents of the tile before, each a
// quarter of the latent columns, and make the copies, two tiles ahead in four buffers. The codes
// stay codes in LDS: a wave takes those it needs out of it, along a token for the scores and
// across 16 tokens (the 4-bit transposing read) for the sums, and forms the values in registers,
// so that LDS and HBM carry 4 bits a value. The values are rounded to fp16, the type of the products (held as
// two halves each they would double the products and the forming); a weight too, as in moe_latent.h.
// Of a tile's 550 vector instructions a SIMD 440 are that forming, 13 for eight values and either use,
// beside 68 products. On a long line no unit is full: of about 4,100 clocks a tile (32 heads) vector
// instructions take 2,200 and products 1,100, with two waves a SIMD in step by a barrier a tile, and what the
// others go to has not been told apart. 512 latents, us a tile and workgroup: 16 heads
// 1.4, 32 1.7, 64 2.7; its copies alone take 1.1. 48 sequences of 32 heads, 378,000 tokens, 122 MB:
// 58 us, 2.1 TB/s (the fp16 cache's 445 MB: 88); 700 tokens of one: 12, of which a tile is 1.7 and the trips to memory
// before it (run, page, codes) are part. Measured and left: sixteen waves, each with half of a token's elements and the partial scores
// added by way of LDS (1.5 and 1.75 us a tile: the instructions are the same); codes by loads to
// registers, a lane a token's (64 separate pieces an instruction: 1.8).
template <int DC, int DR, int MT>
struct Decode4Shape {
  static constexpr int M = 16 * MT, G = DC / 64 + 1;
  static constexpr int NS = 4, NW = 2 * NS;                    // score waves (as many add up), waves
  static constexpr int WR = MT == 4 ? 2 : 1, TW = NS / WR;     // row blocks by token shares of the score waves
  static constexpr int RT = MT / WR, TT = 4 / TW;              // 16-row and 16-token tiles of one
  static constexpr int NJ = DC / 128, KW = DR / 32;            // 16-byte pieces of a token's codes a lane has, words of its key
  static constexpr int KS = 4 * NJ + KW, CT = DC / 64;         // products of a score, 16-column tiles of an adding wave
  // a group of 16 tokens: latents' codes, keys' codes, s and z
  static constexpr int LAT = 8 * DC, KEY = 8 * DR, TAIL = (KEY + 64 * G + 1023) / 1024 * 1024, GRP = LAT + TAIL;
  static constexpr int BUF = 4 * GRP, LN = LAT / 1024, CN = GRP / 1024;  // copies of a wave
  static constexpr int PT = M * 128;                           // the weights of a tile
  static constexpr int LDS = 4 * BUF + 2 * PT + (TW + 1) * M * 4 + 32;
  static constexpr int PC = DC / 32;                           // 16-byte pieces of a row of codes
};
// XOR key of a row's pieces: 16 rows at one piece lie on all banks.
template <int PC>
__device__ __forceinline__ int code_key(int row) { return row * PC / 16; }

// For the scheduler: N products behind the 13 instructions that form the next ones' values.
template <int N>
__device__ __forceinline__ void pace() {
  __builtin_amdgcn_sched_group_barrier(0x2, 13, 0);
  __builtin_amdgcn_sched_group_barrier(0x8, N, 0);
}

struct Decode4Args {
  DecodeArgs d;
  float* sums;                   // [B][sums_stride], or null
  int64_t sums_stride;
};

// (through the scalar unit, as one load)
__device__ __forceinline__ DecodeRun ld_run(const DecodeRun* p) {
  const int32_t* q = reinterpret_cast<const int32_t*>(p);
  return DecodeRun{ld_scalar(q),     ld_scalar(q + 1), ld_scalar(q + 2), ld_scalar(q + 3),
                   ld_scalar(q + 4), ld_scalar(q + 5), ld_scalar(q + 6), ld_scalar(q + 7)};
}

template <int DC, int DR, int MT>
__global__ void __launch_bounds__((64 * Decode4Shape<DC, DR, MT>::NW)) latent4_decode_kernel(DecodeArgs a) {
  using S = Decode4Shape<DC, DR, MT>;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  char* pt = lds + 4 * S::BUF;                                  // weights [2][M][64] halves
  float* smax = reinterpret_cast<float*>(pt + 2 * S::PT);       // [TW][M], by token share
  float* skeep = smax + S::TW * S::M;                           // [M]
  int* passed = reinterpret_cast<int*>(skeep + S::M);           // [2]: the last step with a row past its reference
  const LatentArgs& l = a.l;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4;
  const int wt = wave % S::TW, wr = wave / S::TW, wo = wave - S::NS;  // token share, row block; share of the columns
  // neighbours on the line share a chiplet and its L2
  const int wg = (blockIdx.x % 8) * (a.p.wgs / 8) + blockIdx.x / 8;
  DecodeRun at = ld_run(a.runs + wg);
  const float unit = l.scale * kLog2e;
  const int shift = 31 - __clz(l.page);
  // 16-token group `grp` (0 .. 3) of a tile, from its first token (past the end: the last group)
  auto group = [&](const DecodeRun& run, int tile, int grp) { return min(tile * kStep4 + 16 * grp, run.last & ~15); };
  auto page_of = [&](const DecodeRun& run, int tile, int grp) {
    return ld_scalar(l.table + run.seq * l.table_stride + (group(run, tile, grp) >> shift));
  };
  auto known = [&](int page) { return page >= 0 && page < l.n_pages; };
  if (threadIdx.x < 2) passed[threadIdx.x] = -1;
  const CodeBits bits = code_bits();

  if (wave < S::NS) {
    bool more = at.n > 0;
    h8 q[S::RT][S::KS];
    // (a product's k: the eight codes of a word, of which a lane has 32 latents' of 128, 128 j + 32 g .. + 31,
    // all of one group, and of the key 8 KW)
    auto queries = [&]() {
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        const size_t row = at.row0 + min((wr * S::RT + r) * 16 + c, at.rows - 1);
#pragma unroll
        for (int k = 0; k < S::KS; ++k) {
          const int e = k < 4 * S::NJ ? 128 * (k / 4) + 32 * g + 8 * (k % 4) : DC + 8 * S::KW * g + 8 * (k - 4 * S::NJ);
          q[r][k] = ld_h8(a.ql + row * (DC + DR) + e);
        }
      }
    };
    float sum[S::TT][S::RT], m[S::RT], ref[S::RT];              // m: the reference, unscaled; ref: m unit - kRaise, or 0
    auto start = [&]() {
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        m[r] = -INFINITY;
        ref[r] = 0.f;
#pragma unroll
        for (int t = 0; t < S::TT; ++t) sum[t][r] = 0.f;
      }
    };
    int page[S::TT] = {};
    auto pages = [&](int tile) {
#pragma unroll
      for (int t = 0; t < S::TT; ++t) page[t] = page_of(at, tile, wt * S::TT + t);
    };
    if (more) {
      queries();
      pages(at.first);
    }
    start();
    vm_drain();
    lds_barrier();
    // step u: the scores of tile u, the k-th of its item
    for (int u = 0, k = 0; more; ++u) {
      const char* buf = lds + (u & 3) * S::BUF + wt * S::TT * S::GRP;
      f4 x[S::TT][S::RT] = {};
#pragma unroll
      for (int t = 0; t < S::TT; ++t) {
        const char* lat = buf + t * S::GRP + c * (DC / 2);
        const char* key = buf + t * S::GRP + S::LAT + c * (DR / 2) + 4 * S::KW * g;
        const _Float16* sz = reinterpret_cast<const _Float16*>(buf + t * S::GRP + S::LAT + S::KEY) + c;
        u4 w[S::NJ];
        uint32_t kw[S::KW];
        _Float16 s[S::NJ + 1], z[S::NJ + 1];
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) w[j] = *reinterpret_cast<const u4*>(lat + 16 * ((4 * j + g) ^ code_key<S::PC>(c)));
#pragma unroll
        for (int j = 0; j <= S::NJ; ++j) {
          const int n = j < S::NJ ? 2 * j + (g >> 1) : S::G - 1;
          s[j] = sz[16 * n];
          z[j] = sz[16 * (S::G + n)];
        }
        if constexpr (S::KW == 2) {
          const u2 v = *reinterpret_cast<const u2*>(key);
          kw[0] = v[0];
          kw[1] = v[1];
        } else {
          kw[0] = *reinterpret_cast<const uint32_t*>(key);
        }
        // (a product's values are formed beside the product before it)
        h8 v[2];
        auto form = [&](int k) {
          const int j = k < 4 * S::NJ ? k / 4 : S::NJ;
          v[k & 1] = values8(k < 4 * S::NJ ? w[k / 4][k % 4] : kw[k - 4 * S::NJ], splat8(s[j]), splat8(z[j]), bits);
        };
        form(0);
#pragma unroll
        for (int k = 0; k < S::KS; ++k) {
          if (k + 1 < S::KS) form(k + 1);
#pragma unroll
          for (int r = 0; r < S::RT; ++r) x[t][r] = mfma16(v[k & 1], q[r][k], x[t][r]);
          pace<S::RT>();
        }
      }
      bool lost[S::TT];
      int left[S::TT];                                          // tokens of the group, less one
#pragma unroll
      for (int t = 0; t < S::TT; ++t) {
        lost[t] = !known(page[t]);
        left[t] = at.last - ((at.first + k) * kStep4 + 16 * (wt * S::TT + t));
      }
      const size_t seg = at.seg;
      // (the next run's query is asked for while this step's weights are formed)
      const bool ends = ++k == at.n;
      if (ends) {
        k = 0;
        more = at.next >= 0;
        if (more) {
          at = ld_run(a.runs + at.next);
          queries();
        }
      }
      if (more) pages(at.first + k);
#pragma unroll
      for (int t = 0; t < S::TT; ++t)
        if (lost[t] || left[t] < 15) {
          const int most = lost[t] ? -1 : left[t];
#pragma unroll
          for (int r = 0; r < S::RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (4 * g + e > most) x[t][r][e] = -INFINITY;
        }
      // the weights, in the tokens' order
      float add[S::TT][S::RT];
      auto weights = [&]() {
#pragma unroll
        for (int t = 0; t < S::TT; ++t)
#pragma unroll
          for (int r = 0; r < S::RT; ++r) {
            h4 p;
            add[t][r] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = exp2_fast(fmaf(x[t][r][e], unit, -ref[r]));
              add[t][r] += v;
              p[e] = (_Float16)v;
            }
            *reinterpret_cast<h4*>(pt + (u & 1) * S::PT + ((wr * S::RT + r) * 16 + c) * 128 +
                                   16 * ((2 * (wt * S::TT + t) + (g >> 1)) ^ tile_key<8>(c)) + 8 * (g & 1)) = p;
          }
      };
      weights();
      bool far = false;
      float top[S::RT];
#pragma unroll
      for (int r = 0; r < S::RT; ++r) {
        top[r] = -INFINITY;
#pragma unroll
        for (int t = 0; t < S::TT; ++t) top[r] = max3(max3(top[r], x[t][r][0], x[t][r][1]), x[t][r][2], x[t][r][3]);
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
          float most = m[r];
#pragma unroll
          for (int t = 0; t < S::TW; ++t) most = fmaxf(most, smax[t * S::M + row]);
          float keep = 1.f;
          if ((most - m[r]) * unit > kSlack) {
            const float now = most * unit - kRaise;
            keep = m[r] == -INFINITY ? 0.f : exp2_fast(ref[r] - now);
            m[r] = most;
#pragma unroll
            for (int t = 0; t < S::TT; ++t) sum[t][r] *= keep;
            ref[r] = now;
          }
          if (g == 0 && wt == 0) skeep[row] = keep;
        }
        weights();
        lds_barrier();
      }
#pragma unroll
      for (int t = 0; t < S::TT; ++t)
#pragma unroll
        for (int r = 0; r < S::RT; ++r) sum[t][r] += add[t][r];
      if (ends) {
#pragma unroll
        for (int r = 0; r < S::RT; ++r)
#pragma unroll
          for (int t = 0; t < S::TT; ++t) {
            const float all = col_sum(sum[t][r]);
            if (g == 0)
              *reinterpret_cast<float2*>(a.part_ml + ((seg * 4 + wt * S::TT + t) * S::M + (wr * S::RT + r) * 16 + c) * 2) =
                  float2{m[r] * unit, all};
          }
        start();
      }
    }
    return;
  }

  // this wave copies 16-token group wo of a tile
  const uint32_t at0 = lds_at(lds);
  const Page4 p4 = page4(DC, DR, l.page);
  // a lane's offsets: latents' codes in pieces whose places are keyed, then the keys' codes in one
  // run and 32 bytes of each s and z (past the last: it again)
  uint32_t lat_off[S::LN], tail_off[S::CN - S::LN], tail_step[S::CN - S::LN];
#pragma unroll
  for (int j = 0; j < S::LN; ++j) {
    const int n = 64 * j + lane, row = n / S::PC;
    lat_off[j] = row * (DC / 2) + 16 * ((n % S::PC) ^ code_key<S::PC>(row));
  }
#pragma unroll
  for (int j = 0; j < S::CN - S::LN; ++j) {
    const int n = 64 * j + lane, k = min(n - DR / 2, 4 * S::G - 1);
    tail_off[j] = n < DR / 2 ? p4.keys + 16 * n : p4.steps + (k >> 1) * 2 * l.page + 16 * (k & 1);
    tail_step[j] = n < DR / 2 ? DR / 2 : 2;
  }
  auto copy = [&](const DecodeRun& run, int tile, int buf, int page) {
    if (!known(page)) {
      // (zeros, whose scores are masked; the waits for copies find fewer than they allow)
      if (lane == 0 && l.status) atomicOr(l.status, MOE_STATUS_BAD_PAGE);
      char* to = lds + buf * S::BUF + wo * S::GRP;
      for (int e = lane; e < S::GRP / 16; e += kWave) *reinterpret_cast<U4*>(to + 16 * e) = U4{};
      vm_wait<0>();
      return;
    }
    const uint32_t to = at0 + buf * S::BUF + wo * S::GRP, in = group(run, tile, wo) & (l.page - 1);
    const char* from = reinterpret_cast<const char*>(l.pages) + (size_t)page * p4.bytes;
#pragma unroll
    for (int j = 0; j < S::LN; ++j) dma16(from + in * (DC / 2), lat_off[j], to + 1024 * j);
#pragma unroll
    for (int j = 0; j < S::CN - S::LN; ++j) dma16(from, tail_off[j] + in * tail_step[j], to + S::LAT + 1024 * j);
  };
  // the tiles asked for so far, and the next one
  DecodeRun ask = at;
  int asked = 0, k = 0;
  bool more = ask.n > 0;
  int page = more ? page_of(ask, ask.first, wo) : 0;
  auto ask_next = [&]() {
    if (!more) return false;
    copy(ask, ask.first + k, asked & 3, page);
    ++asked;
    if (++k == ask.n) {
      k = 0;
      more = ask.next >= 0;
      if (more) ask = ld_run(a.runs + ask.next);
    }
    if (more) page = page_of(ask, ask.first + k, wo);
    return true;
  };
  ask_next();
  ask_next();
  // (a lane's address is a token's; the one of lane i is that of the i-th code of a word, so that
  // the codes, which come out in code order, are in the tokens' order)
  const int row = 8 * (c >> 3) + 2 * (c & 3) + (c >> 2 & 1);
  f4 o[S::CT][MT] = {};
  vm_drain();
  lds_barrier();
  int left = at.n;                                              // tiles of the run that are not added up yet
  // step u: the latents of tile u - 1, and tile u + 2 is asked for; the last step has no scores beside it
  for (int u = 0;; ++u) {
    const bool newer = ask_next();
    bool stored = false;
    if (u > 0) {
      const char* blk = lds + ((u - 1) & 3) * S::BUF + g * S::GRP;
      h8 p[MT][2];
#pragma unroll
      for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          p[r][i] = ld_h8(pt + ((u - 1) & 1) * S::PT + (16 * r + c) * 128 + 16 * ((2 * g + i) ^ tile_key<8>(c)));
      // (past the sequence's end s and z are zeros: whatever is there takes no part)
      const int most = at.last - (at.first + at.n - left) * kStep4;
      // (the codes of KR column tiles, all of one group, are asked for before the products of the KR before them)
      typedef int i2 __attribute__((ext_vector_type(2)));
      constexpr int KR = S::CT < 4 ? S::CT : 4;
      i2 w[2][KR];
      h8 s[2][2], z[2][2];
      auto read = [&](int n) {
        const char* sz = blk + S::LAT + S::KEY + ((wo * S::CT + n) / 4) * 32;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          s[n / KR & 1][i] = ld_h8(sz + 16 * i);
          z[n / KR & 1][i] = ld_h8(sz + 32 * S::G + 16 * i);
        }
#pragma unroll
        for (int k = 0; k < KR; ++k) {
          const int col = wo * S::CT + n + k;
          const char* from = blk + row * (DC / 2) + 16 * ((col >> 1) ^ code_key<S::PC>(row)) + 8 * (col & 1);
          w[n / KR & 1][k] = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
              (__attribute__((address_space(3))) i2*)(__attribute__((address_space(3))) char*)from);
        }
      };
      read(0);
#pragma unroll
      for (int n = 0; n < S::CT; n += KR) {
        if (n + KR < S::CT) read(n + KR);
        __builtin_amdgcn_sched_barrier(0);
        h8(&sn)[2] = s[n / KR & 1], (&zn)[2] = z[n / KR & 1];
        if (most < kStep4 - 1) {
          asm volatile("");                                     // (a branch: as selects they would cost every tile)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (16 * g + 8 * i + j > most) sn[i][j] = zn[i][j] = (_Float16)0.f;
        }
        h8 v[2];
        auto form = [&](int k) { v[k & 1] = values8((uint32_t)w[n / KR & 1][k / 2][k % 2], sn[k % 2], zn[k % 2], bits); };
        form(0);
#pragma unroll
        for (int k = 0; k < 2 * KR; ++k) {
          if (k + 1 < 2 * KR) form(k + 1);
#pragma unroll
          for (int r = 0; r < MT; ++r) o[n + k / 2][r] = mfma16(v[k & 1], p[r][k % 2], o[n + k / 2][r]);
          pace<MT>();
        }
      }
      if (--left == 0) {
        const size_t seg = at.seg;
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
          for (int k = 0; k < S::CT; ++k) {
            *reinterpret_cast<f4*>(a.part_o + (seg * S::M + 16 * r + c) * DC + 16 * (wo * S::CT + k) + 4 * g) = o[k][r];
            o[k][r] = f4{};
          }
        stored = true;
        if (at.next >= 0) {
          at = ld_run(a.runs + at.next);
          left = at.n;
        }
      }
    }
    if (u >= asked) break;
    // tile u + 1 is there: all but this step's copies and, behind them, the stores (16 bytes
    // a lane each: no fewer than these)
    constexpr int ST = S::CT * MT;
    if (!newer)
      vm_wait<0>();
    else if (stored)
      vm_wait<S::CN + ST>();
    else
      vm_wait<S::CN>();
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

// ---- the tokens' weights -----------------------------------------------------------
// sums[b][j] += sum_h softmax_h(j), once the rows' references and sums are known: the scores
// again, 16 RT heads a wave (RB such blocks beside each other), 16 tokens a product. A token's
// weights are added up in one order: heads by rows, lanes, then blocks. The codes go from memory
// to registers, 16 bytes a lane, as each is used once, and the next 16 tokens' are asked for
// before these are used. Bound by latency where a wave has a step or two, then mostly by the values'
// forming (512 latents: 40,000 tokens of 16 heads 10 us, 320,000 of 32 heads 35).
// Workgroups at most, while a sequence has one (what is on the chip at once: with 256 and 1024
// 320,000 tokens take 42 us; 60,000 of 32 heads 13, 15 and 22 with 256, 512 and 1024). A workgroup's
// tokens are cut by the bound max_len, and all of these are with the longest length for it: 20 sequences of up to
// 3,001 tokens, the call 28 us, take 42 under a bound of 32,768 and 73 under 131,072, where
// a sequence's tokens are one workgroup's; 48 of up to 16,384 tokens 126 us, and 352 under 131,072.
constexpr int kSumGroups = 512;

template <int DC, int DR, int RT, int RB>
__device__ __forceinline__ void sum_weights(const Decode4Args& b, int tokens, int block) {
  constexpr int G = DC / 64 + 1, NJ = DC / 128, KW = DR / 32, KS = 4 * NJ + KW, TG = 4 / RB;
  __shared__ float part[2][4][16];
  const DecodeArgs& a = b.d;
  const LatentArgs& l = a.l;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int rb = wave % RB, tw = wave / RB, seq = block % a.B, tok0 = block / a.B * tokens;
  const int shift = 31 - __clz(l.page);
  const Page4 p4 = page4(DC, DR, l.page);
  struct Raw {                                               // what a lane has of 16 tokens' codes
    u4 w[NJ];
    uint32_t kw[KW];
    _Float16 s[NJ + 1], z[NJ + 1];
    int page;
  };
  auto page_of = [&](int t) { return ld_scalar(l.table + seq * l.table_stride + min(t >> shift, l.max_pages - 1)); };
  auto known = [&](int page) { return page >= 0 && page < l.n_pages; };
  auto load = [&](Raw& raw, int t, int page) {
    raw.page = page;
    if (!known(page)) return;
    const char* from = reinterpret_cast<const char*>(l.pages) + (size_t)page * p4.bytes;
    const int in = (t & (l.page - 1)) + c;
    const char* lat = from + in * (DC / 2) + 16 * g;
    const char* key = from + p4.keys + in * (DR / 2) + 4 * KW * g;
    const _Float16* sz = reinterpret_cast<const _Float16*>(from + p4.steps) + in;
#pragma unroll
    for (int j = 0; j < NJ; ++j) raw.w[j] = *reinterpret_cast<const u4*>(lat + 64 * j);
#pragma unroll
    for (int i = 0; i < KW; ++i) raw.kw[i] = *reinterpret_cast<const uint32_t*>(key + 4 * i);
#pragma unroll
    for (int j = 0; j <= NJ; ++j) {
      const int n = j < NJ ? 2 * j + (g >> 1) : G - 1;
      raw.s[j] = sz[n * l.page];
      raw.z[j] = sz[(G + n) * l.page];
    }
  };
  Raw now;
  load(now, tok0 + 16 * tw, page_of(tok0 + 16 * tw));
  h8 q[RT][KS];
  float ref[RT][4], inv[RT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int h0 = 16 * (RT * rb + r);
    const __half* from = a.ql + ((size_t)seq * l.H + min(h0 + c, l.H - 1)) * (DC + DR);
#pragma unroll
    for (int k = 0; k < KS; ++k)
      q[r][k] = ld_h8(from + (k < 4 * NJ ? 128 * (k / 4) + 32 * g + 8 * (k % 4) : DC + 8 * (KW * g + k - 4 * NJ)));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int h = h0 + 4 * g + e;
      const float2 ml = *reinterpret_cast<const float2*>(a.row_ml + 2 * ((size_t)seq * l.H + min(h, l.H - 1)));
      ref[r][e] = h < l.H ? ml.x : INFINITY;                 // (a head that is not there: weight 0)
      inv[r][e] = h < l.H ? ml.y : 0.f;
    }
  }
  const int end = min(clamp_len(a, a.kv_len[seq]), tok0 + tokens);
  const float unit = l.scale * kLog2e;
  const CodeBits bits = code_bits();
  int it = 0;
  for (int t0 = tok0; t0 < end; t0 += 16 * TG, ++it) {
    const int t = t0 + 16 * tw;
    const bool there = t < end && known(now.page);
    const Raw raw = now;
    if (t0 + 16 * TG < end) load(now, t + 16 * TG, page_of(t + 16 * TG));
    f4 x[RT] = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int j = k < 4 * NJ ? k / 4 : NJ;
      const h8 v = values8(k < 4 * NJ ? raw.w[k / 4][k % 4] : raw.kw[k - 4 * NJ], splat8(raw.s[j]), splat8(raw.z[j]), bits);
#pragma unroll
      for (int r = 0; r < RT; ++r) x[r] = mfma16(q[r][k], v, x[r]);
    }
    float w = 0.f;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) w += exp2_fast(fmaf(x[r][e], unit, -ref[r][e])) * inv[r][e];
    w = there ? col_sum(w) : 0.f;
    if constexpr (RB > 1) {
      if (g == 0) part[it & 1][wave][c] = w;
      __syncthreads();
      w = 0.f;
#pragma unroll
      for (int k = 0; k < RB; ++k) w += part[it & 1][tw * RB + k][c];
    }
    if (there && rb == 0 && g == 0 && t + c < end) b.sums[seq * b.sums_stride + t + c] += w;
  }
}

template <int DC, int DR, int MT>
hipError_t launch_attention(const DecodeArgs& a, hipStream_t st) {
  constexpr int lds = Decode4Shape<DC, DR, MT>::LDS;
  static_assert(lds <= 160 * 1024, "LDS of a CU");
  auto kernel = latent4_decode_kernel<DC, DR, MT>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(a.p.wgs), dim3(64 * Decode4Shape<DC, DR, MT>::NW), lds, st, a);
  return hipGetLastError();
}
// The first `groups` workgroups form the sums, those behind them the way out of the latent space, which has
// as little to wait for (a launch less: 20 heads over 27,000 tokens of 20 sequences, the call 27 us against 30).
template <int DC, int DR, int RT, int RB>
__global__ void __launch_bounds__(256) latent4_sums_kernel(Decode4Args b, int tokens, int groups) {
  if ((int)blockIdx.x < groups) {
    sum_weights<DC, DR, RT, RB>(b, tokens, blockIdx.x);
  } else {
    const int i = blockIdx.x - groups, tiles = b.d.l.Dv / 16, rest = i / tiles;
    latent_up<DC, false, kStep4>(b.d, i % tiles, rest % b.d.l.H, rest / b.d.l.H);
  }
}

template <int DC, int DR, int RT, int RB>
hipError_t launch_sums(const Decode4Args& b, hipStream_t st) {
  const DecodeArgs& a = b.d;
  constexpr int step = 64 / RB;                              // tokens of a workgroup's step
  const int64_t steps = (a.max_len + step - 1) / step, most = (kSumGroups + a.B - 1) / a.B;
  const int each = (int)((steps + most - 1) / most);
  const unsigned groups = (unsigned)((steps + each - 1) / each) * a.B;
  const dim3 up = up_grid(a);
  hipLaunchKernelGGL((latent4_sums_kernel<DC, DR, RT, RB>), dim3(groups + (joins_itself(a) ? 0 : up.x * up.y * up.z)), dim3(256), 0,
                     st, b, each * step, (int)groups);
  return hipGetLastError();
}
template <int DC, int DR>
hipError_t launch_sums(const Decode4Args& b, hipStream_t st) {
  const int H = b.d.l.H;
  return H <= 16   ? launch_sums<DC, DR, 1, 1>(b, st)
         : H <= 32 ? launch_sums<DC, DR, 2, 1>(b, st)
         : H <= 64 ? launch_sums<DC, DR, 2, 2>(b, st)
                   : launch_sums<DC, DR, 2, 4>(b, st);
}
template <int DC, int DR>
hipError_t launch_decode4(const Decode4Args& b, hipStream_t st) {
  const DecodeArgs& a = b.d;
  hipError_t e = a.p.rows == 16   ? launch_attention<DC, DR, 1>(a, st)
                 : a.p.rows == 32 ? launch_attention<DC, DR, 2>(a, st)
                                  : launch_attention<DC, DR, 4>(a, st);
  if (e != hipSuccess) return e;
  if (!b.sums || a.max_len < 1) return launch_up<DC, kStep4>(a, st);
  e = joins_itself(a) ? launch_up<DC, kStep4>(a, st) : launch_join<kStep4>(a, st);
  return e == hipSuccess ? launch_sums<DC, DR>(b, st) : e;
}

int tiles_host(int len) { return (len + kStep4 - 1) / kStep4; }

// As moe_latent.hip's, without a shared prefix.
DecodePlan decode4_plan(int H, int Dc, int Dr, int B, int max_len, bool sums, size_t* row_ml) {
  DecodePlan p{};
  const int wgs = kCus * (Dc <= 128 ? 2 : 1);
  // 64 rows to a tile form its values once for all of them, but cost a longer start and twice the
  // partial results (512 latents, 128 heads, 8 sequences, the call: 500 tokens 38 us with 64 rows, 34 with
  // 32; 6,000 61, 57; 12,000, which is 12 tiles a workgroup, 79, 79.5; 24,000 110, 121)
  p.rows = H <= 16 ? 16 : H <= 32 || (long long)B * ((H + 63) / 64) * tiles_host(max_len) < 12 * wgs ? 32 : 64;
  p.head_blocks = (H + p.rows - 1) / p.rows;
  // (by the bound, as the lengths are on the device: under one far above them a share is long and the workgroups
  // are few: 20 sequences of up to 3,001 tokens, the call 24 us, 27 under a bound of 131,072 and 42 under 2^20)
  p.least = std::max(1, (int)(0.18 * std::sqrt((double)tiles_host(max_len)) + 0.5));
  // (so many workgroups, up to one a CU, that a short line's tiles have one each: 2 sequences of 700 tokens, the
  // call 24.8 us, with a workgroup a tile, of which the items' places leave some empty, 26.2)
  const long long tiles = (long long)B * p.head_blocks * (tiles_host(max_len) + kItemCost);
  p.wgs = (int)std::min<long long>(wgs, (std::max<long long>(tiles, 1) + 7) / 8 * 8);
  const size_t rows = (size_t)B * H, parts = (size_t)p.wgs + (size_t)B * p.head_blocks;
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
  p.part_ml = take(parts * p.rows * 32);
  p.runs = take((p.wgs + parts) * sizeof(DecodeRun));
  *row_ml = off;
  if (sums) take(rows * 8);
  p.total = off;
  return p;
}

hipError_t launch_latent4_decode(const Decode4Args& b, hipStream_t st) {
  const DecodeArgs& a = b.d;
  const LatentArgs& l = a.l;
  const dim3 ga(l.Dc / 64 + 1, l.H, (a.B + 63) / 64);
  if (l.Dn == 128)
    hipLaunchKernelGGL((latent_absorb_kernel<128, kStep4>), ga, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((latent_absorb_kernel<64, kStep4>), ga, dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (l.Dr == 64)
    return l.Dc == 512 ? launch_decode4<512, 64>(b, st) : l.Dc == 256 ? launch_decode4<256, 64>(b, st) : launch_decode4<128, 64>(b, st);
  return l.Dc == 512 ? launch_decode4<512, 32>(b, st) : l.Dc == 256 ? launch_decode4<256, 32>(b, st) : launch_decode4<128, 32>(b, st);
}

}  // namespace
}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int kMaxLen = 1 << 26, kMaxBatch = 1 << 16;

bool decode4_shape_ok(const moe_latent_spec* s, int B, int max_len) {
  if (moe_latent_spec_check(s) != MOE_OK || B < 0 || B > kMaxBatch || max_len < 0 || max_len > kMaxLen) return false;
  // places on the plan's line
  const int64_t rows = ((int64_t)B * s->heads + 15) / 16 + B;
  return rows * (((int64_t)max_len + 63) / 64 + 32) < (int64_t(1) << 30);
}

}  // namespace

extern "C" {

size_t moe_latent4_page_bytes(const moe_latent_spec* s) {
  if (moe_latent_spec_check(s) != MOE_OK) return 0;
  return moe::page4(s->d_latent, s->d_rope, s->page_tokens).bytes;
}

int moe_latent4_append(const moe_latent_spec* spec, const moe_latent_cache* cache, const float* kv, const void* gamma_f16,
                       const float* rope, int max_pos, const int32_t* seq, const int32_t* slot, const int32_t* pos, int T,
                       const void* q_f16, void* q_out_f16, uint32_t* status, void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (T < 0 || T > (1 << 22) || max_pos < 1 || (!q_f16) != (!q_out_f16)) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!kv || !gamma_f16 || !rope || !seq || !slot || !pos) return MOE_EINVAL;
  if (misaligned(kv, 16) || misaligned(gamma_f16, 16) || misaligned(rope, 16) || misaligned(seq, 4) ||
      misaligned(slot, 4) || misaligned(pos, 4) || misaligned(q_f16, 16) || misaligned(q_out_f16, 16) || misaligned(status, 4))
    return MOE_EALIGN;
  moe::Append4Args b{};
  moe::AppendArgs& a = b.a;
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
  a.q_out = static_cast<__half*>(q_out_f16);
  b.slot = slot;
  b.pages = static_cast<char*>(cache->pages);
  const int n = q_f16 ? a.l.H * (a.l.Dn + a.l.Dr) : 0;
  hipLaunchKernelGGL(moe::latent4_append_kernel, dim3(T, 1 + (n + 2047) / 2048), dim3(256), 0,
                     static_cast<hipStream_t>(stream), b);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

int moe_latent4_read(const moe_latent_spec* spec, const moe_latent_cache* cache, const int32_t* seq, const int32_t* slot,
                     int T, void* rows_f16, uint32_t* status, void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (T < 0 || T > (1 << 24)) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!seq || !slot || !rows_f16) return MOE_EINVAL;
  if (misaligned(seq, 4) || misaligned(slot, 4) || misaligned(rows_f16, 16) || misaligned(status, 4)) return MOE_EALIGN;
  moe::LatentArgs l = moe::latent_args(spec, cache);
  l.status = status;
  const int64_t n = (int64_t)T * ((l.Dc + l.Dr) / 8);
  hipLaunchKernelGGL(moe::latent4_read_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), l, seq, slot, T, static_cast<__half*>(rows_f16));
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

size_t moe_latent4_decode_workspace_bytes(const moe_latent_spec* s, int B, int max_len, int sums) {
  if (!decode4_shape_ok(s, B, max_len)) return 0;
  size_t at;
  return moe::decode4_plan(s->heads, s->d_latent, s->d_rope, B < 1 ? 1 : B, max_len, sums != 0, &at).total;
}

int moe_latent4_decode(const moe_latent_spec* spec, const moe_latent_cache* cache, const void* w_kvb_f16,
                       const void* q_f16, int B, const int32_t* kv_len, int max_len, void* out_f16, float* sums,
                       int64_t sums_stride, uint32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  if (!decode4_shape_ok(spec, B, max_len) || B > cache->n_seqs || (sums && sums_stride < max_len)) return MOE_EINVAL;
  if (B == 0) return MOE_OK;
  if (!w_kvb_f16 || !q_f16 || !kv_len || !out_f16 || !workspace) return MOE_EINVAL;
  if (misaligned(w_kvb_f16, 16) || misaligned(q_f16, 16) || misaligned(kv_len, 4) || misaligned(out_f16, 16) ||
      misaligned(sums, 4) || misaligned(status, 4) || misaligned(workspace, 16))
    return MOE_EALIGN;
  moe::Decode4Args b{};
  moe::DecodeArgs& a = b.d;
  a.l = moe::latent_args(spec, cache);
  a.l.w = static_cast<const __half*>(w_kvb_f16);
  a.l.q = static_cast<const __half*>(q_f16);
  a.l.out = static_cast<__half*>(out_f16);
  a.l.status = status;
  a.B = B;
  a.max_len = max_len;
  a.kv_len = kv_len;
  size_t row_ml;
  a.p = moe::decode4_plan(a.l.H, a.l.Dc, a.l.Dr, B, max_len, sums != nullptr, &row_ml);
  if (workspace_bytes < a.p.total) return MOE_ENOMEM;
  char* ws = static_cast<char*>(workspace);
  a.ql = reinterpret_cast<__half*>(ws + a.p.ql);
  a.lat = reinterpret_cast<__half*>(ws + a.p.lat);
  a.starts = reinterpret_cast<int32_t*>(ws + a.p.starts);
  a.part_o = reinterpret_cast<float*>(ws + a.p.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + a.p.part_ml);
  a.runs = reinterpret_cast<moe::DecodeRun*>(ws + a.p.runs);
  a.row_ml = sums ? reinterpret_cast<float*>(ws + row_ml) : nullptr;
  b.sums = sums;
  b.sums_stride = sums_stride;
  return moe::launch_latent4_decode(b, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
