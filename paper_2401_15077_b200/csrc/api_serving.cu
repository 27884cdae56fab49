// C ABI of the calls around verification (rotary appends, attention of chunks, logit adjustment, sampling): argument checks and launches.
// As in api.cu nothing here allocates or synchronises.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "block.cuh"
#include "chunk.cuh"
#include "logits.cuh"
#include "sample.cuh"

using namespace eagle;

namespace {

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Checks of a cache descriptor that need no GPU; `capacity`: slots per sequence.
int check_store(const eagle_kv_store& kv, int head_dim, int num_kv_heads, long long* capacity) {
  if ((kv.k_scale == nullptr) != (kv.v_scale == nullptr)) return EAGLE_ERR_NULL;
  if (kv.k_scale && head_dim != 128) return EAGLE_ERR_SHAPE;
  if (misaligned(kv.k, 16) || misaligned(kv.v, 16)) return EAGLE_ERR_SHAPE;
  if (kv.block_table) {
    if (kv.num_pages < 1 || kv.page_size < 16 || (kv.page_size & (kv.page_size - 1)) || kv.max_pages_per_seq < 0) return EAGLE_ERR_SHAPE;
    if (static_cast<long long>(kv.num_pages) * num_kv_heads > 0x7fffffffll) return EAGLE_ERR_SHAPE;
    *capacity = static_cast<long long>(kv.max_pages_per_seq) * kv.page_size;
  } else {
    if (kv.kv_capacity < 0) return EAGLE_ERR_SHAPE;
    *capacity = kv.kv_capacity;
  }
  if (*capacity > 0x7fffffffll) *capacity = 0x7fffffffll;   // lengths are 32-bit
  return EAGLE_OK;
}

int page_shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

// Checks of a rotary append and its kernel's parameters; *sms stays 0 where there is nothing to do.
int rope_params(const eagle_rope_desc& d, bool tree, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                const int32_t* seq_lens, const int32_t* order, RopeParams* params, int* sms) {
  *sms = 0;
  if (d.batch < 0 || d.batch > 65535 || d.num_q_heads < 0 || d.num_kv_heads < 1 || d.num_q_heads > 65535 || d.num_kv_heads > 65535 ||
      (d.head_dim != 64 && d.head_dim != 128) || d.rotary_dim < 16 || d.rotary_dim > d.head_dim || d.rotary_dim % 16)
    return EAGLE_ERR_SHAPE;
  if (tree ? (d.max_tree < 0 || d.max_tree > kMaxTree) : d.num_tokens < 0) return EAGLE_ERR_SHAPE;
  if (!(std::fabs(d.amplitude) < 3.0e38f)) return EAGLE_ERR_SHAPE;
  const int64_t dq = static_cast<int64_t>(d.num_q_heads) * d.head_dim, dk = static_cast<int64_t>(d.num_kv_heads) * d.head_dim;
  const int64_t sq = d.q_stride ? d.q_stride : dq, sk = d.k_stride ? d.k_stride : dk, sv = d.v_stride ? d.v_stride : dk;
  if (sq < dq || sk < dk || sv < dk || sq % 8 || sk % 8 || sv % 8) return EAGLE_ERR_SHAPE;
  long long capacity = 0;
  const int rc = check_store(*kv, d.head_dim, d.num_kv_heads, &capacity);
  if (rc != EAGLE_OK) return rc;
  if (d.batch == 0 || (tree ? d.max_tree : d.num_tokens) == 0) return EAGLE_OK;
  if ((d.num_q_heads > 0 && (!q || !q_out)) || !k || !v || !kv->k || !kv->v || !seq_lens || !order || !d.freqs) return EAGLE_ERR_NULL;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(q_out, 16) || misaligned(d.freqs, 8)) return EAGLE_ERR_SHAPE;
  if (q == q_out && sq != dq && d.num_q_heads > 0) return EAGLE_ERR_SHAPE;      // in place only over the same layout
  const int dev = usable_device(sms);
  if (dev != EAGLE_OK) return dev;
  RopeParams& p = *params;
  p = {};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.q_stride = sq;
  p.k_stride = sk;
  p.v_stride = sv;
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_cache = kv->k;
  p.v_cache = kv->v;
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  p.block_table = kv->block_table;
  p.page_size = kv->page_size;
  p.page_shift = kv->block_table ? page_shift_of(kv->page_size) : 0;
  p.max_pages = kv->max_pages_per_seq;
  p.num_pages = kv->num_pages;
  p.capacity = capacity;
  p.head_rows = kv->block_table ? kv->page_size : capacity;
  p.seq_lens = seq_lens;
  p.token_start = tree ? nullptr : order;
  p.tree_parent = tree ? order : nullptr;
  p.positions = tree ? nullptr : d.positions;
  p.tree_sizes = d.tree_sizes;
  p.shared_tree = d.shared_tree != 0;
  p.freqs = d.freqs;
  p.amplitude = d.amplitude != 0.f ? d.amplitude : 1.f;
  p.B = d.batch;
  p.N = tree ? 0 : d.num_tokens;
  p.T = d.max_tree;
  p.Hq = d.num_q_heads;
  p.Hkv = d.num_kv_heads;
  p.D = d.head_dim;
  p.R = d.rotary_dim;
  p.interleaved = d.interleaved != 0;
  p.status = d.status;
  return EAGLE_OK;
}

int rope_call(const eagle_rope_desc* desc, bool tree, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
              const int32_t* seq_lens, const int32_t* order, eagle_stream_t stream) {
  if (!desc || !kv) return EAGLE_ERR_NULL;
  RopeParams p;
  int sms = 0;
  const int rc = rope_params(*desc, tree, q, k, v, q_out, kv, seq_lens, order, &p, &sms);
  if (rc != EAGLE_OK || sms == 0) return rc;
  return launch_rope(p, tree, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

// Checks of a block-scaled cache beyond those of check_store.
int check_blocks(const eagle_kv_store& kv, int block_size) {
  if (block_size != 16 && block_size != 32 && block_size != 64 && block_size != 128) return EAGLE_ERR_SHAPE;
  if ((kv.block_table ? kv.page_size : kv.kv_capacity) % block_size) return EAGLE_ERR_SHAPE;
  if (!kv.k_scale || !kv.v_scale) return EAGLE_ERR_NULL;
  if (misaligned(kv.k_scale, 4) || misaligned(kv.v_scale, 4)) return EAGLE_ERR_SHAPE;
  return EAGLE_OK;
}

int block_call(const eagle_block_desc* desc, bool tree, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
               const int32_t* seq_lens, const int32_t* order, eagle_stream_t stream) {
  if (!desc || !kv) return EAGLE_ERR_NULL;
  const eagle_block_desc& d = *desc;
  eagle_rope_desc as = {};
  as.batch = d.batch;
  as.num_tokens = d.num_tokens;
  as.max_tree = d.max_tree;
  as.num_q_heads = d.num_q_heads;
  as.num_kv_heads = d.num_kv_heads;
  as.head_dim = 128;
  as.rotary_dim = d.rotary_dim;
  as.interleaved = d.interleaved;
  as.amplitude = d.amplitude;
  as.q_stride = d.q_stride;
  as.k_stride = d.k_stride;
  as.v_stride = d.v_stride;
  as.freqs = d.freqs;
  as.positions = d.positions;
  as.tree_sizes = d.tree_sizes;
  as.shared_tree = d.shared_tree;
  as.status = d.status;
  int rc = check_blocks(*kv, d.block_size);
  if (rc != EAGLE_OK) return rc;
  BlockParams p = {};
  int sms = 0;
  rc = rope_params(as, tree, q, k, v, q_out, kv, seq_lens, order, &p.r, &sms);
  if (rc != EAGLE_OK || sms == 0) return rc;
  p.k_scale = const_cast<float*>(kv->k_scale);
  p.v_scale = const_cast<float*>(kv->v_scale);
  p.block_size = d.block_size;
  p.block_shift = page_shift_of(d.block_size);
  p.head_blocks = p.r.head_rows / d.block_size;
  return launch_block(p, tree, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

// The attention kernel's shared-memory opt-in, once per device and head size.
std::mutex g_prepared_mutex;
bool g_prepared[64][2][2];

bool prepared(int head_dim, bool window = false) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  std::lock_guard<std::mutex> lock(g_prepared_mutex);
  bool& done = g_prepared[dev][head_dim == 128][window];
  if (!done)
    done = window ? window_prepare(head_dim) == cudaSuccess && window_rows_prepare(head_dim) == cudaSuccess && window_codes_prepare() == cudaSuccess
                  : chunk_prepare(head_dim) == cudaSuccess && chunk_rows_prepare(head_dim) == cudaSuccess;
  return done;
}

// The plan of a windowed call is that of a chunk call with as many rows.
eagle_chunk_desc rows_of(const eagle_window_desc& d, bool tree) {
  eagle_chunk_desc as = {};
  as.batch = d.batch;
  as.num_tokens = d.num_tokens;
  if (tree) as.num_tokens = d.batch > 0 && d.max_tree > 0 ? d.batch * d.max_tree : 0;      // (at most 65535 * 64)
  as.num_q_heads = d.num_q_heads;
  as.num_kv_heads = d.num_kv_heads;
  as.head_dim = d.head_dim;
  return as;
}

size_t chunk_workspace(const eagle_chunk_desc& desc, int few_rows = kFewRows) {
  ChunkWork w;
  int workers = 0;
  if (!carve_chunk_work(desc, nullptr, kMaxPlanCtas, &w, &workers, few_rows)) return 0;
  size_t bytes = w.bytes;
  if (!chunk_takes_rows(desc)) {           // enough for fewer tokens too, single ones among them
    eagle_chunk_desc d = desc;
    d.num_tokens = d.batch;
    if (carve_chunk_work(d, nullptr, kMaxPlanCtas, &w, &workers, few_rows) && w.bytes > bytes) bytes = w.bytes;
  }
  return bytes;
}

// Query rows of the row kernel over codes.
int code_rows(const eagle_chunk_desc& d) { return d.num_kv_heads > 0 && d.num_q_heads / d.num_kv_heads <= 8 ? 8 : kFewRows; }

// Everything of an attention call but what tells the forms apart.
void fill_attention(ChunkParams* params, const eagle_chunk_desc& d, float sm_scale, const void* q, const eagle_kv_store& kv, const int32_t* seq_lens,
                    const int32_t* token_start, void* out, int32_t* status, int few_rows = kFewRows) {
  ChunkParams& p = *params;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(kv.k);
  p.v = static_cast<const __nv_bfloat16*>(kv.v);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.seq_lens = seq_lens;
  p.token_start = token_start;
  p.block_table = kv.block_table;
  p.B = d.batch;
  p.N = d.num_tokens;
  p.Hq = d.num_q_heads;
  p.Hkv = d.num_kv_heads;
  p.G = d.num_q_heads / d.num_kv_heads;
  p.D = d.head_dim;
  p.few = chunk_takes_rows(d);
  p.rows = p.few ? few_rows : kTileRows;
  p.tpt = p.rows / p.G;
  p.ut = p.few ? p.tpt : 2 * p.tpt;
  p.max_rows = static_cast<int>(std::fmin(1.0e9, static_cast<double>(d.num_tokens) * p.G));
  p.page_size = kv.page_size;
  p.page_shift = kv.block_table ? page_shift_of(kv.page_size) : 0;
  p.max_pages = kv.max_pages_per_seq;
  p.num_pages = kv.num_pages;
  const float scale = sm_scale != 0.f ? sm_scale : 1.0f / std::sqrt(static_cast<float>(d.head_dim));
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = status;
  p.wait_limit_ns = wait_limit_ns();
  p.stall_after_tiles = stall_after_tiles();
}

int window_call(const eagle_window_desc* desc, bool tree, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens, const int32_t* order,
                void* out, eagle_stream_t stream) {
  if (!desc || !kv) return EAGLE_ERR_NULL;
  const eagle_window_desc& d = *desc;
  if (tree && (d.max_tree < 0 || d.max_tree > kMaxTree)) return EAGLE_ERR_SHAPE;
  const eagle_chunk_desc as = rows_of(d, tree);
  ChunkParams p = {};
  ChunkWork need;
  const int few_rows = d.block_size ? code_rows(as) : kFewRows;
  if (!(d.sm_scale >= 0.f) || !(d.sm_scale < 3.0e38f) || !carve_chunk_work(as, nullptr, kMaxPlanCtas, &need, &p.num_workers, few_rows)) return EAGLE_ERR_SHAPE;
  if (d.window < 0 || d.sinks < 0 || (tree && d.window > 0 && d.window < kMaxTree)) return EAGLE_ERR_SHAPE;
  if (d.block_size == 0 && (kv->k_scale || kv->v_scale)) return EAGLE_ERR_SHAPE;
  int rc = check_store(*kv, d.head_dim, d.num_kv_heads, &p.capacity);
  if (rc == EAGLE_OK && d.block_size) rc = check_blocks(*kv, d.block_size);
  if (rc != EAGLE_OK) return rc;
  p.capacity = std::min(p.capacity, kMaxWindowSlots);
  if (as.batch == 0 || as.num_tokens == 0) return EAGLE_OK;
  if (!q || !kv->k || !kv->v || !seq_lens || !order || !out) return EAGLE_ERR_NULL;
  if (misaligned(q, 16) || misaligned(out, 32)) return EAGLE_ERR_SHAPE;
  if (!d.workspace || misaligned(d.workspace, 256) || d.workspace_bytes < need.bytes) return EAGLE_ERR_WORKSPACE;
  int sms = 0;
  const int dev = usable_device(&sms);
  if (dev != EAGLE_OK) return dev;
  if (!prepared(d.head_dim, true)) return EAGLE_ERR_DEVICE;
  carve_chunk_work(as, d.workspace, sms, &p.work, &p.num_workers, few_rows);
  fill_attention(&p, as, d.sm_scale, q, *kv, seq_lens, tree ? nullptr : order, out, d.status, few_rows);
  // (a window that reaches past the capacity is no limit)
  p.window = d.window > p.capacity ? 0 : d.window;
  p.sinks = d.sinks > p.capacity ? static_cast<int>(p.capacity) : d.sinks;
  p.tree = tree ? d.max_tree : 0;
  p.tree_parent = tree ? order : nullptr;
  p.tree_sizes = tree ? d.tree_sizes : nullptr;
  p.shared_tree = tree && d.shared_tree != 0;
  if (d.block_size) {
    p.k_scale = kv->k_scale;
    p.v_scale = kv->v_scale;
    p.block_shift = page_shift_of(d.block_size);
    p.head_blocks = (kv->block_table ? kv->page_size : p.capacity) / d.block_size;
  }
  return launch_window(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

}  // namespace

extern "C" {

int eagle_rope_frequencies(const eagle_rope_scaling* scaling, double* freqs, float* amplitude) {
  if (!scaling || !freqs || !amplitude) return EAGLE_ERR_NULL;
  const eagle_rope_scaling& s = *scaling;
  const double kTwoPi = 6.283185307179586476925;
  const bool stretched = s.kind != EAGLE_ROPE_PLAIN, banded = s.kind == EAGLE_ROPE_YARN || s.kind == EAGLE_ROPE_BANDED;
  if (s.kind < EAGLE_ROPE_PLAIN || s.kind > EAGLE_ROPE_BANDED || s.rotary_dim < 2 || s.rotary_dim % 2 || s.rotary_dim > 65536 ||
      !(s.base > 1.0) || !std::isfinite(s.base))
    return EAGLE_ERR_SHAPE;
  if (stretched && (!(s.factor >= 1.0) || !std::isfinite(s.factor))) return EAGLE_ERR_SHAPE;
  if (s.kind == EAGLE_ROPE_NTK && s.rotary_dim < 4) return EAGLE_ERR_SHAPE;
  if (banded && (!(s.context > 0.0) || !std::isfinite(s.context) || !(s.low > 0.0) || !(s.high > s.low) || !std::isfinite(s.high))) return EAGLE_ERR_SHAPE;
  const int half = s.rotary_dim / 2;
  const double R = s.rotary_dim;
  const double base = s.kind == EAGLE_ROPE_NTK ? s.base * std::pow(s.factor, R / (R - 2.0)) : s.base;
  double lo = 0.0, hi = 1.0;
  *amplitude = 1.f;
  if (s.kind == EAGLE_ROPE_YARN) {
    auto place = [&](double turns) { return R * std::log(s.context / (kTwoPi * turns)) / (2.0 * std::log(base)); };
    lo = std::fmax(std::floor(place(s.high)), 0.0);
    hi = std::fmin(std::ceil(place(s.low)), R - 1.0);
    if (hi <= lo) hi = lo + 0.001;
    *amplitude = static_cast<float>(0.1 * std::log(s.factor) + 1.0);
  }
  for (int m = 0; m < half; ++m) {
    double f = std::pow(base, -2.0 * m / R);
    if (s.kind == EAGLE_ROPE_LINEAR) {
      f /= s.factor;
    } else if (s.kind == EAGLE_ROPE_YARN) {
      const double ramp = std::fmin(std::fmax((m - lo) / (hi - lo), 0.0), 1.0);
      f = f * (1.0 - ramp) + f / s.factor * ramp;
    } else if (s.kind == EAGLE_ROPE_BANDED) {
      const double wave = kTwoPi / f;
      if (wave > s.context / s.low) f /= s.factor;
      else if (wave >= s.context / s.high) {
        const double blend = (s.context / wave - s.low) / (s.high - s.low);
        f = (1.0 - blend) * f / s.factor + blend * f;
      }
    }
    freqs[m] = f;
  }
  return EAGLE_OK;
}

int eagle_rope_append(const eagle_rope_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                      const int32_t* seq_lens, const int32_t* token_start, eagle_stream_t stream) {
  return rope_call(desc, false, q, k, v, q_out, kv, seq_lens, token_start, stream);
}

int eagle_tree_rope_append(const eagle_rope_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                           const int32_t* seq_lens, const int32_t* tree_parent, eagle_stream_t stream) {
  return rope_call(desc, true, q, k, v, q_out, kv, seq_lens, tree_parent, stream);
}

size_t eagle_chunk_attn_workspace(const eagle_chunk_desc* desc) { return desc ? chunk_workspace(*desc) : 0; }

size_t eagle_window_attn_workspace(const eagle_window_desc* desc) {
  if (!desc || desc->max_tree < 0 || desc->max_tree > kMaxTree) return 0;
  const eagle_chunk_desc as = rows_of(*desc, desc->max_tree > 0);
  size_t bytes = chunk_workspace(as);      // for a cache in either form
  if (bytes > 0 && code_rows(as) != kFewRows) bytes = std::max(bytes, chunk_workspace(as, code_rows(as)));
  return bytes;
}

int eagle_chunk_attn(const eagle_chunk_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                     const int32_t* token_start, void* out, eagle_stream_t stream) {
  if (!desc || !kv) return EAGLE_ERR_NULL;
  const eagle_chunk_desc& d = *desc;
  ChunkParams p = {};
  ChunkWork need;
  if (!(d.sm_scale >= 0.f) || !(d.sm_scale < 3.0e38f) || !carve_chunk_work(d, nullptr, kMaxPlanCtas, &need, &p.num_workers) || kv->k_scale || kv->v_scale) return EAGLE_ERR_SHAPE;
  const int rc = check_store(*kv, d.head_dim, d.num_kv_heads, &p.capacity);
  if (rc != EAGLE_OK) return rc;
  if (d.batch == 0 || d.num_tokens == 0) return EAGLE_OK;
  if (!q || !kv->k || !kv->v || !seq_lens || !token_start || !out) return EAGLE_ERR_NULL;
  if (misaligned(q, 16) || misaligned(out, 32)) return EAGLE_ERR_SHAPE;
  if (!d.workspace || misaligned(d.workspace, 256) || d.workspace_bytes < need.bytes) return EAGLE_ERR_WORKSPACE;
  int sms = 0;
  const int dev = usable_device(&sms);
  if (dev != EAGLE_OK) return dev;
  if (!prepared(d.head_dim)) return EAGLE_ERR_DEVICE;
  carve_chunk_work(d, d.workspace, sms, &p.work, &p.num_workers);
  fill_attention(&p, d, d.sm_scale, q, *kv, seq_lens, token_start, out, d.status);
  return launch_chunk(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

int eagle_tree_logits_adjust(const eagle_logits_desc* desc, const void* logits, const int32_t* draft_tokens, const int32_t* tree_parent,
                             float* out, eagle_stream_t stream) {
  if (!desc) return EAGLE_ERR_NULL;
  const eagle_logits_desc& d = *desc;
  if (d.batch < 0 || d.batch > 65535 || d.max_tree < 0 || d.max_tree > kMaxTree || d.vocab < 1 || d.vocab > (1 << 30) || d.history_cap < 0 ||
      d.max_bias < 0 || d.max_bias > kMaxBias)
    return EAGLE_ERR_SHAPE;
  if (d.batch == 0) return EAGLE_OK;
  if (!logits || !out || (d.max_tree > 0 && (!draft_tokens || !tree_parent))) return EAGLE_ERR_NULL;
  if ((d.history && !d.history_len) || (d.bias_tokens && !d.bias_values)) return EAGLE_ERR_NULL;
  if (misaligned(logits, d.bf16 ? 2 : 4) || misaligned(out, 4) || (d.bf16 && logits == static_cast<const void*>(out))) return EAGLE_ERR_SHAPE;
  int sms = 0;
  const int dev = usable_device(&sms);
  if (dev != EAGLE_OK) return dev;
  LogitsParams p = {};
  p.logits = logits;
  p.out = out;
  p.draft_tokens = draft_tokens;
  p.tree_parent = tree_parent;
  p.tree_sizes = d.max_tree > 0 ? d.tree_sizes : nullptr;
  p.history = d.history_cap > 0 ? d.history : nullptr;
  p.history_len = d.history_len;
  p.prompt_len = d.prompt_len;
  p.repetition = d.repetition;
  p.presence = d.presence;
  p.frequency = d.frequency;
  p.bias_tokens = d.max_bias > 0 ? d.bias_tokens : nullptr;
  p.bias_values = d.bias_values;
  p.bias_len = d.bias_len;
  p.allowed = d.allowed;
  p.B = d.batch;
  p.T = d.max_tree;
  p.V = d.vocab;
  p.H = d.history_cap;
  p.max_bias = d.max_bias;
  p.bf16 = d.bf16 != 0;
  p.shared_tree = d.shared_tree != 0;
  p.status = d.status;
  return launch_logits(p, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

int eagle_window_attn(const eagle_window_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                      const int32_t* token_start, void* out, eagle_stream_t stream) {
  return window_call(desc, false, q, kv, seq_lens, token_start, out, stream);
}

int eagle_tree_window_attn(const eagle_window_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                           const int32_t* tree_parent, void* out, eagle_stream_t stream) {
  return window_call(desc, true, q, kv, seq_lens, tree_parent, out, stream);
}

int eagle_block_append(const eagle_block_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                       const int32_t* seq_lens, const int32_t* token_start, eagle_stream_t stream) {
  return block_call(desc, false, q, k, v, q_out, kv, seq_lens, token_start, stream);
}

int eagle_tree_block_append(const eagle_block_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                            const int32_t* seq_lens, const int32_t* tree_parent, eagle_stream_t stream) {
  return block_call(desc, true, q, k, v, q_out, kv, seq_lens, tree_parent, stream);
}

int eagle_sample(const eagle_sample_desc* desc, const void* logits, const float* uniforms, int32_t* tokens, float* probs, eagle_stream_t stream) {
  if (!desc) return EAGLE_ERR_NULL;
  const eagle_sample_desc& d = *desc;
  if (d.batch < 0 || d.batch > 65535 || d.rows < 0 || d.vocab < 1 || d.vocab > EAGLE_MAX_SAMPLE_VOCAB ||
      static_cast<long long>(d.batch) * d.rows > (1ll << 27))
    return EAGLE_ERR_SHAPE;
  if (d.batch == 0 || d.rows == 0) return EAGLE_OK;
  if (!logits || (!tokens && !probs) || (tokens && !uniforms)) return EAGLE_ERR_NULL;
  if (misaligned(logits, d.bf16 ? 2 : 4) || misaligned(probs, 4) || logits == static_cast<const void*>(probs)) return EAGLE_ERR_SHAPE;
  int sms = 0;
  const int dev = usable_device(&sms);
  if (dev != EAGLE_OK) return dev;
  SampleParams p = {};
  p.logits = logits;
  p.uniforms = uniforms;
  p.tokens = tokens;
  p.probs = probs;
  p.num_rows = d.num_rows;
  p.temperature = d.temperature;
  p.top_k = d.top_k;
  p.top_p = d.top_p;
  p.min_p = d.min_p;
  p.B = d.batch;
  p.R = d.rows;
  p.V = d.vocab;
  p.bf16 = d.bf16 != 0;
  p.status = d.status;
  return launch_sample(p, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? EAGLE_OK : EAGLE_ERR_LAUNCH;
}

}  // extern "C"
