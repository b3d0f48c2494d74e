// Latent attention (moe_latent.hip, moe_prefill.hip): the launches' arguments.
#pragma once

#include "moe_device.h"

namespace moe {

constexpr int kTile = 64;        // context tokens of a tile of the expanded form
constexpr int kStep = 32;        // and of the absorbed form

// A row's softmax weights are held as 2^(score log2(e) - reference + kRaise). The reference
// is the row's running maximum, but follows it only where that passes it by kSlack: until
// then nothing is rescaled. In fp16 a weight so has all bits down to 2^-(14 + kRaise) of the
// largest, is off by at most 2^-(25 + kRaise) of it below, and is at most 2^(kSlack +
// kRaise), which is in range. (4 and 11 would hold four more bits, but rescale more often:
// 32 sequences of 64 heads on 12,000 shared tokens 125 us against 113.) A row's sum and all
// its partial results are raised alike.
constexpr float kSlack = 8.f, kRaise = 7.f;

struct LatentArgs {
  int H, Dc, Dr, Dn, Dv, page;   // page: tokens a page, a power of two >= 16
  float scale;
  const __half* pages;           // [n_pages][page][Dc + Dr]
  int n_pages, n_seqs, max_pages;
  const int32_t* table;          // [n_seqs][table_stride]
  int64_t table_stride;
  const __half* w;               // [H][Dn + Dv][Dc]
  const __half* q;               // [rows][H][Dn + Dr]
  __half* out;                   // [rows][H][Dv]
  uint32_t* status;
};

// The checks of a description and its cache, and their fields as the launches take them.
int latent_cache_check(const moe_latent_spec* s, const moe_latent_cache* c);
LatentArgs latent_args(const moe_latent_spec* s, const moe_latent_cache* c);

struct AppendArgs {
  LatentArgs l;
  const float* kv;               // [T][Dc + Dr]
  const __half* gamma;           // [Dc]
  const float* rope;             // [max_pos][Dr / 2][2]
  int max_pos, T;
  const int32_t *seq, *pos;      // [T]
  __half* pages;
  __half* q_out;                 // [T][H][Dn + Dr]
};
hipError_t launch_latent_append(const AppendArgs& a, hipStream_t st);

// How a decode call is cut: rows of one workgroup, workgroups, and what the workspace
// holds. The tiles of all items (the shared prefix's row blocks by token chunks, then
// every sequence's head blocks) lie on one line that the workgroups share evenly; a
// workgroup writes one partial result per item that it has tiles of: O, and (m, l) from
// either half of its tokens.
struct DecodePlan {
  int rows;                      // query rows of an item: 16, 32 or 64
  int head_blocks;               // items of one sequence
  int chunks, row_blocks;        // prefix: token chunks x row blocks
  int chunk_tiles, prefix_places;
  int wgs, least;                // workgroups, and the least share of the line of one
  size_t ql, lat, starts, part_o, part_ml, total;  // byte offsets in the workspace
};
DecodePlan decode_plan(int H, int Dc, int Dr, int B, int max_len, int prefix_len);

struct DecodeArgs {
  LatentArgs l;
  int B, max_len, prefix_len;
  const int32_t* kv_len;         // [B]
  const int32_t* prefix;         // pages of the prefix, or null
  DecodePlan p;
  __half* ql;                    // [B * H][Dc + Dr]: q in latent space, and its rope part
  __half* lat;                   // [B * H][Dc]: softmax-weighted latents
  int32_t* starts;               // [B + 1]: first place of each sequence
  float* part_o;                 // [wgs + items][rows][Dc]
  float* part_ml;                // [wgs + items][2][rows][2]
};
hipError_t launch_latent_decode(const DecodeArgs& a, hipStream_t st);

constexpr int kPartGroups = 256, kPartRows = 256;  // workgroups that leave partial results, and their rows

struct PrefillArgs {
  LatentArgs l;
  int T, B, kv_total, max_q, parts;
  const int32_t *q_start, *kv_start;  // [B + 1]
  __half *k, *v, *kr;            // [H][kv_total][Dn], [H][kv_total][Dv], [kv_total][Dr]
  float *part_o, *part_ml;       // [kPartGroups][kPartRows][Dv] and [..][2], with parts > 1
  uint32_t* lost;                // per 64-token tile: its 16-token groups without a page
};
int prefill_parts(int max_q, int H, int B, int kv_total);
hipError_t launch_latent_prefill(const PrefillArgs& a, hipStream_t st);

}  // namespace moe
