// Eviction from a 4-bit latent cache by the tokens' accumulated attention weights: which of a
// sequence's tokens stay (moe_evict_select), and their rows' way into new pages
// (moe_latent4_move).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "moe_latent4.h"

namespace moe {
namespace {

// ---- the tokens that stay ---------------------------------------------------------
// One workgroup a row of sums. Of the tokens between the fixed ones (the first `sinks`, the
// last `recent`) the m largest sums stay, ties to the lower index. Their sums' order keys are
// narrowed to the m-th largest, 256 bins at a time between the smallest and the largest key
// (sums spread over few octaves: bins over all 32 bits would be hit by all at once); then
// one pass in order writes what stays.
// Rows of up to 8,192 sums are HELD in registers over these passes. Bound by the passes' barriers
// (192 rows of 6,000 sums: 15 us, read anew in each pass 19; one row of 1,100: 8.7, 8.4).
struct SelectArgs {
  const float* sums;             // [rows][width], row = layer * B + sequence
  float* sums_out;               // the same shape; may be the same array
  const int32_t* kv_len;         // [B]
  int B, width, budget, sinks, recent;
  int32_t* keep;                 // [rows][budget]
  uint32_t* status;
};

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave, kBins = 256, kEach = 4, kHeldRounds = 2;

__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v) { return ~wave_max_u32(~v); }

template <bool HELD>
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(SelectArgs a) {
  __shared__ uint32_t hist[kSelectWaves][kBins];
  __shared__ uint32_t low[kSelectWaves], high[kSelectWaves], found[2];
  const int b = blockIdx.x % a.B, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const float* sums = a.sums + (size_t)blockIdx.x * a.width;
  float* out = a.sums_out + (size_t)blockIdx.x * a.width;
  int32_t* keep = a.keep + (size_t)blockIdx.x * a.budget;
  const int n = min(max(a.kv_len[b], 0), a.width), stay = min(n, a.budget);
  if (n != a.kv_len[b] && blockIdx.x < (unsigned)a.B && tid == 0 && a.status) atomicOr(a.status, MOE_STATUS_BAD_LENGTH);
  int first = min(a.sinks, n), last = max(first, n - a.recent);  // the tokens that are ranked: first .. last - 1
  int m = stay - first - (n - last);                             // those of them that stay
  if (n <= a.budget) {
    last = first;
    m = 0;
  }
  // four tokens in a row a thread, a round behind the other
  constexpr int kRound = kSelectThreads * kEach;
  float held[HELD ? kHeldRounds : 1][kEach];
  auto load = [&](int i, float (&v)[kEach]) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = i + j < n ? sums[i + j] : 0.f;
  };
  if constexpr (HELD)
#pragma unroll
    for (int r = 0; r < kHeldRounds; ++r) load(r * kRound + kEach * tid, held[r]);
  // all of the ranked tokens' keys that are this thread's
  auto each = [&](auto f) {
    if constexpr (HELD) {
#pragma unroll
      for (int r = 0; r < kHeldRounds; ++r)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int i = r * kRound + kEach * tid + j;
          if (i >= first && i < last) f(topk_key(held[r][j]));
        }
    } else {
      for (int i = first + tid; i < last; i += kSelectThreads) f(topk_key(sums[i]));
    }
  };
  uint32_t least = 0xFFFFFFFFu;                                  // keys above it stay (none is above this), and `ties` at it
  int ties = 0;
  if (m > 0) {
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    each([&](uint32_t k) {
      lo = min(lo, k);
      hi = max(hi, k);
    });
    lo = wave_min_u32(lo);
    hi = wave_max_u32(hi);
    if (lane == 0) {
      low[wave] = lo;
      high[wave] = hi;
    }
    __syncthreads();
    lo = low[0];
    hi = high[0];
    for (int w = 1; w < kSelectWaves; ++w) {
      lo = min(lo, low[w]);
      hi = max(hi, high[w]);
    }
    int shift = max(0, 24 - __clz((int)(hi - lo)));              // (__clz(0) is 32)
    uint32_t want = m;                                           // the want-th largest key of those in [lo, lo + 256 << shift)
    uint32_t span = hi - lo;                                     // the keys in question are lo .. lo + span
    while (true) {
      for (int i = tid; i < kSelectWaves * kBins; i += kSelectThreads) (&hist[0][0])[i] = 0;
      __syncthreads();
      each([&](uint32_t key) {
        const uint32_t k = key - lo;                             // (below lo: wraps past the span)
        if (k <= span) atomicAdd(&hist[wave][k >> shift], 1u);
      });
      __syncthreads();
      if (wave == 0) {
        // lane's four bins, from the largest keys down
        uint32_t c[4], all = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int bin = kBins - 1 - (4 * lane + j);
          c[j] = 0;
          for (int w = 0; w < kSelectWaves; ++w) c[j] += hist[w][bin];
          all += c[j];
        }
        uint32_t up = all;                                       // of this lane and those before it
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const uint32_t v = __shfl_up(up, o, kWave);
          if (lane >= o) up += v;
        }
        uint32_t before = up - all;
        if (before < want && want <= up) {
          int j = 0;
          while (before + c[j] < want) before += c[j++];
          found[0] = kBins - 1 - (4 * lane + j);
          found[1] = want - before;
        }
      }
      __syncthreads();
      lo += found[0] << shift;
      want = found[1];
      if (shift == 0) break;
      span = (1u << shift) - 1;
      shift = max(0, shift - 8);
      __syncthreads();
    }
    least = lo;
    ties = want;
  }
  __syncthreads();
  // In order, four tokens a thread: a token that stays goes behind those that do before it
  // (never past its own place, so that the sums may move within one array: a step's are
  // all read before the first is written).
  int above = 0, equal = 0;                                      // tokens that stay for sure, and ties, before these
  auto round = [&](int i0, const float (&v)[kEach]) {
    const int i = i0 + kEach * tid;
    uint32_t mine = 0;                                           // of this thread: ties << 16 | sure ones
    int what[kEach];                                             // 1: stays, 2: a tie
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      what[j] = 0;
      if (i + j >= n) continue;
      const uint32_t k = topk_key(v[j]);
      what[j] = i + j < first || i + j >= last || k > least ? 1 : k == least ? 2 : 0;
      mine += what[j] == 1 ? 1u : what[j] == 2 ? 1u << 16 : 0u;
    }
    uint32_t up = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t t = __shfl_up(up, o, kWave);
      if (lane >= o) up += t;
    }
    if (lane == kWave - 1) low[wave] = up;
    __syncthreads();
    uint32_t before = up - mine, all = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) before += low[w];
      all += low[w];
    }
    int sure = above + (before & 0xFFFF), tie = equal + (int)(before >> 16);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const bool stays = what[j] == 1 || (what[j] == 2 && tie < ties);
      const int at = sure + min(tie, ties);
      if (stays && at < stay) {
        keep[at] = i + j;
        out[at] = v[j];
      }
      sure += what[j] == 1;
      tie += what[j] == 2;
    }
    above += all & 0xFFFF;
    equal += all >> 16;
    __syncthreads();
  };
  if constexpr (HELD) {
#pragma unroll
    for (int r = 0; r < kHeldRounds; ++r)
      if (r * kRound < n) round(r * kRound, held[r]);
  } else {
    for (int i0 = 0; i0 < n; i0 += kRound) {
      float v[kEach];
      load(i0 + kEach * tid, v);
      round(i0, v);
    }
  }
  for (int i = stay + tid; i < a.budget; i += kSelectThreads) keep[i] = -1;
  for (int i = stay + tid; i < a.width; i += kSelectThreads) out[i] = 0.f;
}

// ---- their rows' way into new pages -------------------------------------------------
// A wave moves 16 tokens of one sequence and layer; a kept token's codes are whole pieces,
// its steps and middles two bytes each, gathered from the pages' planes and stored by a wave in 32-byte pieces of
// them. 24 layers of 8 sequences, 280,000 tokens kept, 184 MB: 51.6 us, 3.6 TB/s, where a copy has 5.15.
struct MoveArgs {
  LatentArgs l;                  // (the layer 0 pages)
  char* pages;
  int64_t layer_bytes;
  int B, budget;
  const int32_t* keep;           // [n_layers][B][budget]
  const int32_t* to_table;       // [B][to_stride]
  int64_t to_stride;
};

__global__ void __launch_bounds__(256) latent4_move_kernel(MoveArgs a) {
  const LatentArgs& l = a.l;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int blocks = (a.budget + 63) / 64, b = blockIdx.x / blocks, i0 = (blockIdx.x % blocks) * 64 + 16 * wave;
  const int layer = blockIdx.y;
  if (i0 >= a.budget) return;
  const Page4 p4 = page4(l.Dc, l.Dr, l.page);
  char* pages = a.pages + layer * a.layer_bytes;
  const int shift = 31 - __clz(l.page), mask = l.page - 1;
  // lane i < 16: where token i comes from and goes to (-1: nowhere)
  int src = -1, from = 0, to = 0;
  if (lane < 16 && i0 + lane < a.budget) {
    const int slot = a.keep[((size_t)layer * a.B + b) * a.budget + i0 + lane];
    if (slot >= 0) {
      const bool in = slot >> shift < l.max_pages;
      from = in ? l.table[b * l.table_stride + (slot >> shift)] : 0;
      to = a.to_table[b * a.to_stride + ((i0 + lane) >> shift)];
      const bool good = in && from >= 0 && from < l.n_pages && to >= 0 && to < l.n_pages;
      if (good)
        src = slot & mask;
      else if (l.status)
        atomicOr(l.status, in ? MOE_STATUS_BAD_PAGE : MOE_STATUS_BAD_INDEX);
    }
  }
  // (the lanes of a wave fetch a token's places from the lane that has them)
  struct Way {
    const char* x;
    char* y;
  };
  auto way = [&](int k, int part, int row_bytes) {
    const int s = __shfl(src, k, kWave), f = __shfl(from, k, kWave), t = __shfl(to, k, kWave);
    return Way{s < 0 ? nullptr : pages + (size_t)f * p4.bytes + part + s * row_bytes,
               pages + (size_t)t * p4.bytes + part + ((i0 & mask) + k) * row_bytes};
  };
  const int pieces = l.Dc / 32;                          // (16 rows of them: whole waves)
  for (int e = lane; e < 16 * pieces; e += kWave) {
    const Way w = way(e / pieces, 0, l.Dc / 2);
    const int at = 16 * (e % pieces);
    if (w.x) *reinterpret_cast<U4*>(w.y + at) = ld16(w.x + at);
  }
  const int kp = l.Dr / 32;                              // (16 rows: half a wave or less)
  const Way key = way(min(lane / kp, 15), p4.keys, l.Dr / 2);
  if (lane < 16 * kp && key.x) *reinterpret_cast<U4*>(key.y + 16 * (lane % kp)) = ld16(key.x + 16 * (lane % kp));
  const Way tail = way(lane & 15, p4.steps, 2);
  if (tail.x)
    for (int n = lane >> 4; n < 2 * (l.Dc / 64 + 1); n += 4)
      *reinterpret_cast<uint16_t*>(tail.y + n * 2 * l.page) = *reinterpret_cast<const uint16_t*>(tail.x + n * 2 * l.page);
}

}  // namespace
}  // namespace moe

// ---- C ABI (contracts in include/moe_api.h) ---------------------------------------

namespace {
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
constexpr int kMaxTokens = 1 << 26, kMaxBatch = 1 << 16;
}  // namespace

extern "C" {

int moe_evict_select(const float* sums, float* sums_out, int n_layers, int B, int width, const int32_t* kv_len, int budget,
                     int sinks, int recent, int32_t* keep, uint32_t* status, void* stream) {
  if (n_layers < 1 || B < 0 || B > kMaxBatch || width < 1 || width > kMaxTokens || budget < 1 || budget > kMaxTokens ||
      sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return MOE_EINVAL;
  if ((int64_t)n_layers * B * moe::kSelectThreads > (int64_t)UINT32_MAX) return MOE_EINVAL;  // (a grid's threads)
  if (B == 0) return MOE_OK;
  if (!sums || !sums_out || !kv_len || !keep) return MOE_EINVAL;
  if (misaligned(sums, 4) || misaligned(sums_out, 4) || misaligned(kv_len, 4) || misaligned(keep, 4) || misaligned(status, 4))
    return MOE_EALIGN;
  const moe::SelectArgs a{sums, sums_out, kv_len, B, width, budget, sinks, recent, keep, status};
  const bool held = width <= moe::kHeldRounds * moe::kEach * moe::kSelectThreads;
  hipLaunchKernelGGL(held ? moe::evict_select_kernel<true> : moe::evict_select_kernel<false>, dim3((unsigned)(n_layers * B)),
                     dim3(moe::kSelectThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

int moe_latent4_move(const moe_latent_spec* spec, const moe_latent_cache* cache, int n_layers, int64_t layer_bytes,
                     const int32_t* keep, int B, int budget, const int32_t* to_table, int64_t to_stride, uint32_t* status,
                     void* stream) {
  const int rc = moe::latent_cache_check(spec, cache);
  if (rc != MOE_OK) return rc;
  const int64_t page_bytes = moe::page4(spec->d_latent, spec->d_rope, spec->page_tokens).bytes;
  if (n_layers < 1 || n_layers > 65535 || layer_bytes % 16 ||
      (n_layers > 1 && layer_bytes / cache->n_pages < page_bytes) || B < 0 || B > cache->n_seqs || budget < 1 ||
      budget > kMaxTokens || to_stride < (budget + spec->page_tokens - 1) / spec->page_tokens)
    return MOE_EINVAL;
  if ((int64_t)B * ((budget + 63) / 64) * 256 > (int64_t)UINT32_MAX) return MOE_EINVAL;  // (a grid's threads)
  if (B == 0) return MOE_OK;
  if (!keep || !to_table) return MOE_EINVAL;
  if (misaligned(keep, 4) || misaligned(to_table, 4) || misaligned(status, 4)) return MOE_EALIGN;
  moe::MoveArgs a{};
  a.l = moe::latent_args(spec, cache);
  a.l.status = status;
  a.pages = static_cast<char*>(cache->pages);
  a.layer_bytes = layer_bytes;
  a.B = B;
  a.budget = budget;
  a.keep = keep;
  a.to_table = to_table;
  a.to_stride = to_stride;
  hipLaunchKernelGGL(moe::latent4_move_kernel, dim3((unsigned)(B * ((budget + 63) / 64)), n_layers), dim3(256), 0,
                     static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
