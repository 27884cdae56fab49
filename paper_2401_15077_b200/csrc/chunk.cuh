// Plan records, workspace and parameters of the chunk attention (chunk.cu, chunk_rows.cu).
#pragma once
#include "common.cuh"

namespace eagle {

constexpr int kChunkTile = 128;        // keys per K/V tile
// Cost model of the planner, in keys: what starting a unit costs (pipeline fill, output), and within how many K/V tiles of a
// unit's edge a cut moves to the edge.
constexpr int kChunkItemKeys = 256;
constexpr int kChunkSnap = 2;

// Two attention kernels share the planner and the merge.  The tile kernel's workers are pairs of CTAs, with two query tiles of
// 128 rows on the tensor cores of both; the row kernel's are single CTAs, with one query tile of 16 rows.  A query tile is
// TPT tokens times the G heads of a group.  Calls with no more rows than sequences (single tokens) take the row kernel: there
// the keys and values are streamed once for a few rows, and what counts is how steadily they come.  64 single tokens over 512 to
// 8192 slots, 32 heads over 8: 203 us, the tile kernel 249 us; one token over 65536, 64 heads over 8: 59.5 us against
// 77 us.  The host sees numbers and no lengths, so the rule takes N <= B for single tokens.  The row kernel is right for more tokens of
// a sequence too, but reads its cache again for every 16 / G of them.  Rows against tiles in us (cold caches, D = 128, 8 KV heads):
//   a token each, 64 sequences of 512 to 4112 slots    32 heads 127 : 152   64 heads 127 : 152   no groups 395 : 524
//   two tokens in every other of them                  32 heads  80 :  94   64 heads  82 :  94   no groups 225 : 281
//   four in every fourth                               32 heads  51 :  59   64 heads  64 :  59   no groups 129 : 152
//   one chunk behind 8192 slots, all others empty
//     of 8 tokens                                      32 heads  29 :  31   64 heads  37 :  33   no groups  28 :  29
//     of 64 tokens                                     32 heads  88 :  35   64 heads 154 :  41   no groups  37 :  35
//     of 200 tokens                                    32 heads 231 :  55   64 heads 444 :  80   no groups  76 :  35
// So it is wrong for a chunk of many tokens among as many empty sequences; a caller that has one gets the tile kernel by leaving
// empty sequences out, or with a row behind the last sequence (N > B).  A decode batch with such a spare row takes the tile kernel, 1.2 to 1.3
// times as long.
constexpr int kTileRows = 128, kFewRows = 16;
inline bool chunk_takes_rows(const eagle_chunk_desc& d) { return d.num_tokens <= d.batch; }

// A unit is what a worker holds at once (one or two neighbouring query tiles) of one (sequence, KV head); an item is what a
// worker does of it in one go.
struct ChunkSeq {        // n = 0: empty or refused
  int32_t start, n, L, parts;    // units per KV head
};
struct ChunkUnit {
  int32_t b, g, part, tiles;     // K/V tiles
};
struct alignas(16) ChunkItem {
  int32_t b, g, part, start;     // start: the sequence's first row
  int32_t n, L, t0, t1;          // K/V tiles [t0, t1)
  int32_t slot;                  // partial slot of the first query tile (the second's is the next one), -1: write the output
  int32_t pad[3];
};
// A unit whose output is merged from the pieces (unit, c), c_lo <= c <= c_hi; unit < 0: none.
struct ChunkCut {
  int32_t unit, c_lo, c_hi, pad;
};

struct ChunkWork {
  ChunkSeq* seq;           // [B]
  int32_t* unit_base;      // [B]
  long long* cost_base;    // [B]
  long long* x;            // [units + 1]: where each unit starts on the work line
  ChunkUnit* unit;         // [units]
  ChunkItem* items;        // [units + workers]
  int4* cta;               // [workers]: whole units (first, count), pieces (first, count)
  ChunkCut* cut;           // [workers]
  int32_t* bad_page;       // [B]: cleared by the planner, set by whoever copies from a page that is not in the pool
  float2* part_ml;         // [slots, rows of a query tile]
  float* part_o;           // [slots, D / 4, rows, 4]
  size_t bytes;
};

struct ChunkParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  __nv_bfloat16* out;
  const int32_t* seq_lens;       // [B]
  const int32_t* token_start;    // [B + 1]
  const int32_t* block_table;    // paged cache, or null
  int32_t B, N, Hq, Hkv, G, D;
  int32_t few;                   // the row kernel's call
  int32_t rows, tpt, ut;         // rows and tokens of a query tile, tokens of a unit
  int32_t max_rows;              // query rows of a (sequence, KV head) at the most
  long long capacity;            // slots per sequence
  int32_t page_size, page_shift, max_pages, num_pages;
  int32_t num_workers;           // CTAs of the row kernel, pairs of CTAs of the tile kernel
  float scale_log2;
  int32_t* status;
  unsigned long long wait_limit_ns;
  int32_t stall_after_tiles;     // test hook: the kernels' STALL instantiations issue copies of that many tiles and no more (negative: off)
  ChunkWork work;
};

// Partial slots: a worker's share of the cut units begins and ends inside a unit at the most, with the query tiles of both.
// `sms` bounds the workers.
inline bool carve_chunk_work(const eagle_chunk_desc& d, void* base, int sms, ChunkWork* w, int* num_workers) {
  if (d.batch < 0 || d.num_tokens < 0 || d.num_kv_heads <= 0 || d.num_q_heads <= 0 || d.num_q_heads % d.num_kv_heads) return false;
  const int G = d.num_q_heads / d.num_kv_heads;
  if (G > kMaxGroup || (d.head_dim != 64 && d.head_dim != 128) || d.batch > 65535) return false;
  const bool few = chunk_takes_rows(d);
  const int rows = few ? kFewRows : kTileRows, tiles = few ? 1 : 2, workers = (sms < kMaxPlanCtas ? sms : kMaxPlanCtas) / tiles;
  const size_t B = static_cast<size_t>(d.batch), ut = tiles * (rows / G);
  const size_t units = static_cast<size_t>(d.num_kv_heads) * (d.num_tokens / ut + B);
  if (units > (1u << 28)) return false;
  const size_t slots = 2 * static_cast<size_t>(tiles) * workers;
  *num_workers = workers;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t n) { char* r = p ? p + off : nullptr; off += align256(n > 0 ? n : 1); return r; };
  w->seq = reinterpret_cast<ChunkSeq*>(take(sizeof(ChunkSeq) * B));
  w->unit_base = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * B));
  w->cost_base = reinterpret_cast<long long*>(take(sizeof(long long) * B));
  w->x = reinterpret_cast<long long*>(take(sizeof(long long) * (units + 1)));
  w->unit = reinterpret_cast<ChunkUnit*>(take(sizeof(ChunkUnit) * units));
  w->items = reinterpret_cast<ChunkItem*>(take(sizeof(ChunkItem) * (units + workers)));
  w->cta = reinterpret_cast<int4*>(take(sizeof(int4) * workers));
  w->cut = reinterpret_cast<ChunkCut*>(take(sizeof(ChunkCut) * workers));
  w->bad_page = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * B));
  w->part_ml = reinterpret_cast<float2*>(take(sizeof(float2) * slots * rows));
  w->part_o = reinterpret_cast<float*>(take(sizeof(float) * slots * rows * d.head_dim));
  w->bytes = off;
  return true;
}

cudaError_t chunk_prepare(int head_dim);
cudaError_t chunk_rows_prepare(int head_dim);
cudaError_t launch_chunk_rows(const ChunkParams& p, cudaStream_t stream);      // the row kernel alone, behind the planner
cudaError_t launch_chunk(const ChunkParams& p, cudaStream_t stream);

}  // namespace eagle
