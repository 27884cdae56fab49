// Plan records, workspace and parameters of the chunk attention (chunk.cu, chunk_rows.cu) and of the attention with a window, over
// bf16 or block-scaled caches, of chunks or trees (window.cu, window_rows.cu, window_codes.cu), which shares planner and merge.
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
// 8192 slots, 32 heads over 8: 203 us, the tile kernel 249 us; one token over 65536, 64 heads over 8: 58 us against
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
struct alignas(16) ChunkCut {
  int32_t unit, c_lo, c_hi, pad;
  int32_t b, g, part, start;     // of the unit, and of its sequence
  int32_t n, pad2[3];
};

struct ChunkWork {
  ChunkSeq* seq;           // [B]
  int32_t* unit_base;      // [B]
  long long* cost_base;    // [B]
  long long* x;            // [units + 1]: where each unit starts on the work line
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
  // Calls with a window, a tree or block scales (the planner's and the merge's SPAN instantiations); 0 and null elsewhere
  int32_t window, sinks;         // W (0: no limit) and S, both at most the capacity
  int32_t tree;                  // T_max of the tree form: sequence b has the rows from b * tree on; 0: chunk form
  const int32_t* tree_parent;
  const int32_t* tree_sizes;
  int32_t shared_tree;
  const float* k_scale;          // one per block and KV head, or null: bf16
  const float* v_scale;
  int32_t block_shift;
  long long head_blocks;         // blocks from one KV head to the next
};

// Slots of a sequence in a windowed call: slots up to two query tiles past its end are 32-bit numbers too.  (Without a window a sequence of
// such a length would be read whole; with one it is a table of pages whose first entries nobody looks at.)
constexpr long long kMaxWindowSlots = 0x7fffff00ll;

// What a unit whose first token is `first` sees of its sequence: slots below `sinks` and from `low` on.  K/V tiles that hold neither are
// left out: the plan counts tiles without them, and tile t of the plan is tile(t) of the sequence.
struct ChunkSpan {
  int low, sinks;
  int before, skip;              // tiles in front of the gap, tiles in it
  __host__ __device__ int tile(int t) const { return t < before ? t : t + skip; }
  // a page that holds no slot that is seen is not looked up: the first one behind the gap stands for it (its rows are masked)
  __device__ int page(int pi, int shift) const { return pi < (low >> shift) && pi > ((sinks - 1) >> shift) ? low >> shift : pi; }
  __device__ bool sees(int key) const { return key >= low || key < sinks; }
  __device__ bool sees_all(int key, int n) const { return key >= low || key + n <= sinks || low <= sinks; }
  __device__ bool sees_some(int key, int n) const { return key + n > low || key < sinks; }
};
__host__ __device__ inline ChunkSpan chunk_span(const ChunkParams& p, int L, int first) {
  ChunkSpan s = {0, 0, 0, 0};
  if (p.window > 0) {
    const int low = L + (p.tree ? 0 : first) - p.window + 1;
    s.low = low > 0 ? low : 0;
    s.sinks = p.sinks < s.low ? p.sinks : s.low;
    const int w0 = s.low / kChunkTile, before = s.sinks / kChunkTile + (s.sinks % kChunkTile != 0);
    s.before = before < w0 ? before : w0;
    s.skip = w0 - s.before;
  }
  return s;
}

// Partial slots: a worker's share of the cut units begins and ends inside a unit at the most, with the query tiles of both.
// `sms` bounds the workers; few_rows: rows of the row kernel's query tiles (those of codes has 8 where a group has no more heads).
inline bool carve_chunk_work(const eagle_chunk_desc& d, void* base, int sms, ChunkWork* w, int* num_workers, int few_rows = kFewRows) {
  if (d.batch < 0 || d.num_tokens < 0 || d.num_kv_heads <= 0 || d.num_q_heads <= 0 || d.num_q_heads % d.num_kv_heads) return false;
  const int G = d.num_q_heads / d.num_kv_heads;
  if (G > kMaxGroup || (d.head_dim != 64 && d.head_dim != 128) || d.batch > 65535) return false;
  const bool few = chunk_takes_rows(d);
  const int rows = few ? few_rows : kTileRows, tiles = few ? 1 : 2, workers = (sms < kMaxPlanCtas ? sms : kMaxPlanCtas) / tiles;
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
cudaError_t launch_chunk_plan(const ChunkParams& p, cudaStream_t stream);      // SPAN instantiations
cudaError_t launch_chunk_merge(const ChunkParams& p, cudaStream_t stream);
cudaError_t window_prepare(int head_dim);
cudaError_t window_rows_prepare(int head_dim);
cudaError_t launch_window_rows(const ChunkParams& p, cudaStream_t stream);      // bf16
cudaError_t window_codes_prepare();
cudaError_t launch_window_codes(const ChunkParams& p, cudaStream_t stream);     // codes
cudaError_t launch_window(const ChunkParams& p, cudaStream_t stream);

}  // namespace eagle
