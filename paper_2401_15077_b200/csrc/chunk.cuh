// Plan records, workspace and parameters of the chunk attention (chunk.cu).
#pragma once
#include "common.cuh"

namespace eagle {

constexpr int kChunkTile = 128;        // keys per K/V tile
// Cost model of the planner, in keys: what starting a unit costs (pipeline fill, output), and within how many K/V tiles of a
// unit's edge a cut moves to the edge.
constexpr int kChunkItemKeys = 256;
constexpr int kChunkSnap = 2;
constexpr int kMaxPairs = kMaxPlanCtas / 2;

// A unit is a pair of neighbouring query tiles of one (sequence, KV head); an item is what a pair of CTAs does of it in one go.
struct ChunkSeq {        // n = 0: empty or refused
  int32_t start, n, L, pairs;
};
struct ChunkUnit {
  int32_t b, g, pair, tiles;     // K/V tiles
};
struct alignas(16) ChunkItem {
  int32_t b, g, pair, start;     // start: the sequence's first row
  int32_t n, L, t0, t1;          // K/V tiles [t0, t1)
  int32_t slot;                  // partial slot of the first CTA's query tile (the second's is the next one), -1: write the output
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
  ChunkItem* items;        // [units + CTA pairs]
  int4* cta;               // [CTA pairs]: whole units (first, count), pieces (first, count)
  ChunkCut* cut;           // [CTA pairs]
  float2* part_ml;         // [slots, 128]
  float* part_o;           // [slots, D / 4, 128, 4]
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
  int32_t tpt;                   // tokens per query tile
  int32_t max_rows;              // query rows of a (sequence, KV head) at the most
  long long capacity;            // slots per sequence
  int32_t page_size, page_shift, max_pages, num_pages;
  int32_t num_pairs;             // pairs of CTAs of the attention kernel
  float scale_log2;
  int32_t* status;
  unsigned long long wait_limit_ns;
  ChunkWork work;
};

// Partial slots: a pair of CTAs' share of the cut units begins and ends inside a unit at the most: two pieces of two query tiles.
inline bool carve_chunk_work(const eagle_chunk_desc& d, void* base, int num_pairs, ChunkWork* w) {
  if (d.batch < 0 || d.num_tokens < 0 || d.num_kv_heads <= 0 || d.num_q_heads <= 0 || d.num_q_heads % d.num_kv_heads) return false;
  const int G = d.num_q_heads / d.num_kv_heads;
  if (G > kMaxGroup || (d.head_dim != 64 && d.head_dim != 128) || d.batch > 65535) return false;
  const size_t B = static_cast<size_t>(d.batch), tpt = 128 / G;
  const size_t units = static_cast<size_t>(d.num_kv_heads) * (d.num_tokens / (2 * tpt) + B);
  if (units > (1u << 28)) return false;
  const size_t slots = 4 * static_cast<size_t>(num_pairs);
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t n) { char* r = p ? p + off : nullptr; off += align256(n > 0 ? n : 1); return r; };
  w->seq = reinterpret_cast<ChunkSeq*>(take(sizeof(ChunkSeq) * B));
  w->unit_base = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * B));
  w->cost_base = reinterpret_cast<long long*>(take(sizeof(long long) * B));
  w->x = reinterpret_cast<long long*>(take(sizeof(long long) * (units + 1)));
  w->unit = reinterpret_cast<ChunkUnit*>(take(sizeof(ChunkUnit) * units));
  w->items = reinterpret_cast<ChunkItem*>(take(sizeof(ChunkItem) * (units + num_pairs)));
  w->cta = reinterpret_cast<int4*>(take(sizeof(int4) * num_pairs));
  w->cut = reinterpret_cast<ChunkCut*>(take(sizeof(ChunkCut) * num_pairs));
  w->part_ml = reinterpret_cast<float2*>(take(sizeof(float2) * slots * 128));
  w->part_o = reinterpret_cast<float*>(take(sizeof(float) * slots * 128 * d.head_dim));
  w->bytes = off;
  return true;
}

cudaError_t chunk_prepare(int head_dim);
cudaError_t launch_chunk(const ChunkParams& p, cudaStream_t stream);

}  // namespace eagle
