// Penalties for repeated tokens, biases and grammar masks on the target's rows of a draft tree.
//
// Row 0 of a sequence is the distribution after the committed context, row i + 1 the one after tree node i, so what counts as
// "already there" differs from row to row: the history, and the draft tokens on the path from the root to node i.  For token v
//     c = times v was generated (history past the prompt, and the path),  seen = v in the prompt or c > 0
//     z <- seen ? (z > 0 ? z / rho : z * rho) : z;   z <- z - phi c - pi [c > 0];   z <- z + bias(v);   masked: -inf.
//
// A CTA takes 2048 tokens of the vocabulary and some rows of one sequence.  It counts the history's tokens that fall into its
// range in shared memory (the list is short next to the rows: 16 KB against 8 KB * rows at 4096 tokens), turns them into a
// factor choice and an addend for each of its eight tokens per thread, kept in registers, and then streams the rows: one read
// and one write of each logit, nothing else of that size, no workspace.  Draft tokens on a row's path are rare in a CTA's
// range: a bit set says which nodes matter, and the thread that owns such a token computes it again.  A warp has 256
// consecutive tokens, 32 at a time: every access is coalesced whatever the vocabulary's alignment, and lane l holds word l & 7
// of the grammar's mask for all of them.  Logits and mask of the rows to come are on their way while one is worked on.
// Counts are integers and a token's biases are added up by one thread in list order, so a call gives the same bits every time.
//
// Bound by HBM for a batch of trees, and there by what a CTA does before its first row: all its loads set out together as soon as
// the sequence's lengths are known.  Replayed from a graph, 64 trees of 16 to 64 nodes x 32000 tokens, 4096 tokens of history, biases and
// masks (699 MB): 135 us, 5.2 of the 6.6 TB/s that a plain copy reaches (147 us with the loads where they are used).  16 bf16 rows of 129537
// tokens: 8.3 to 9.3 us, of which 1.9 us would be the bytes: two rounds of CTAs, a launch and three trips to memory.
#include "logits.cuh"

namespace eagle {

namespace {

constexpr int kLogThreads = 256;
constexpr int kPerThread = 8;
constexpr int kRange = kLogThreads * kPerThread;
constexpr int kRowsPerCta = 16;
constexpr uint32_t kInPrompt = 0x80000000u;

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* base, size_t i) {
  if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(base)[i]) << 16);
  else return __ldcs(static_cast<const float*>(base) + i);
}

template <bool BF16>
__global__ void __launch_bounds__(kLogThreads, 4) logits_kernel(LogitsParams p) {
  __shared__ __align__(16) uint32_t s_count[kRange];
  __shared__ __align__(16) float s_bias[kRange];
  __shared__ int s_btok[kMaxBias];
  __shared__ unsigned long long s_path[kMaxTree];   // nodes on the path of node i whose token lies in this CTA's range
  __shared__ int s_parent[kMaxTree], s_off[kMaxTree];   // parent; place of the node's token in the range, -1: outside
  const int tid = threadIdx.x, b = blockIdx.y, v0 = blockIdx.x * kRange, r_lo = blockIdx.z * p.rows_per_block;
  const bool first = blockIdx.x == 0 && blockIdx.z == 0 && tid == 0;      // reports for the sequence

  // ---- what the sequence has: everything below sets out as soon as its lengths are there
  const int n = p.tree_sizes ? p.tree_sizes[p.shared_tree ? 0 : b] : p.T;
  int len = p.history ? min(max(p.history_len[b], 0), p.H) : 0;
  const int prompt = p.history && p.prompt_len ? p.prompt_len[b] : 0;
  const int nb = p.bias_tokens ? min(max(p.bias_len ? p.bias_len[b] : p.max_bias, 0), p.max_bias) : 0;
  const float rho = p.repetition ? p.repetition[b] : 1.f, pi = p.presence ? p.presence[b] : 0.f, phi = p.frequency ? p.frequency[b] : 0.f;
#pragma unroll
  for (int i = 4 * tid; i < kRange; i += 4 * kLogThreads) {
    *reinterpret_cast<uint4*>(s_count + i) = make_uint4(0u, 0u, 0u, 0u);
    *reinterpret_cast<float4*>(s_bias + i) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  bool bad = n < 0 || n > p.T;
  const int rows = bad ? p.T + 1 : n + 1, r_hi = min(rows, r_lo + p.rows_per_block);
  const size_t row0 = static_cast<size_t>(b) * (p.T + 1) * p.V;
  if (r_lo >= r_hi) len = 0;                         // (no row of this CTA exists: it only looks whether the tree is valid)
  const int lane = tid & 31, v_warp = (tid >> 5) * (32 * kPerThread), words = (p.V + 31) / 32;
  const int n_here = min(max(p.V - v0 - v_warp - lane, 0) + 31, 32 * kPerThread) >> 5;     // this lane's tokens that exist
  const int w_at = (v0 + v_warp) / 32 + (lane & (kPerThread - 1));                         // this lane's word of the mask
  const bool has_word = p.allowed && w_at < words;
  auto fetch = [&](int r, float (&z)[kPerThread], uint32_t& mask) __attribute__((always_inline)) {
    if (r >= r_hi) return;
    const size_t at = row0 + static_cast<size_t>(r) * p.V + v0 + v_warp + lane;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
      if (k < n_here) z[k] = load_logit<BF16>(p.logits, at + k * 32);
    if (has_word) mask = __ldg(p.allowed + (static_cast<size_t>(b) * (p.T + 1) + r) * words + w_at);
  };
  const int32_t* h = p.history + static_cast<size_t>(b) * p.H;
  int t[8];                                          // this thread's next tokens of the history
  auto fetch_history = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = i0 + j * kLogThreads < len ? __ldg(h + i0 + j * kLogThreads) : 0;
  };
  fetch_history(tid);
  int parent = -1, token = 0;
  if (!bad && tid < n) {
    parent = p.tree_parent[(p.shared_tree ? 0 : static_cast<size_t>(b) * p.T) + tid];
    token = p.draft_tokens[static_cast<size_t>(b) * p.T + tid];
  }
  float z0[kPerThread], z1[kPerThread];
  uint32_t m0 = 0u, m1 = 0u;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) z0[k] = z1[k] = 0.f;
  fetch(r_lo, z0, m0);
  fetch(r_lo + 1, z1, m1);

  for (int i = tid; i < nb; i += kLogThreads) s_btok[i] = p.bias_tokens[static_cast<size_t>(b) * p.max_bias + i];
  // ---- the tree
  {
    int wrong = 0, off = -1;
    if (!bad && tid < n) {
      wrong = parent < -1 || parent >= tid;
      if (token < 0 || token >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); }
      else if (token >= v0 && token < v0 + kRange) off = token - v0;
      s_parent[tid] = parent;
      s_off[tid] = off;
    }
    bad = __syncthreads_or(bad || wrong);
  }
  if (bad) {
    if (first) report_status(p.status, EAGLE_ERR_TREE);
    for (int r = r_lo; r < min(p.T + 1, r_lo + p.rows_per_block); ++r)
      for (int k = 0; k < kPerThread; ++k) {
        const int v = v0 + tid + k * kLogThreads;
        if (v < p.V) p.out[row0 + static_cast<size_t>(r) * p.V + v] = 0.f;
      }
    return;
  }
  if (r_lo >= r_hi) return;

  // ---- history: counts of the tokens in the range
  if (tid < n) {
    unsigned long long path = 0ull;
    for (int m = tid; m >= 0; m = s_parent[m])
      if (s_off[m] >= 0) path |= 1ull << m;
    s_path[tid] = path;
  }
  for (int i0 = tid; i0 < len; i0 += 8 * kLogThreads) {
    if (i0 != tid) fetch_history(i0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = i0 + j * kLogThreads;
      if (i >= len) break;
      if (t[j] < 0 || t[j] >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); }
      else if (t[j] >= v0 && t[j] < v0 + kRange) {
        if (i < prompt) atomicOr(&s_count[t[j] - v0], kInPrompt);
        else atomicAdd(&s_count[t[j] - v0], 1u);
      }
    }
  }
  for (int i = tid; i < nb; i += kLogThreads) {
    const int tok = s_btok[i];
    if (tok < 0 || tok >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); continue; }
    if (tok < v0 || tok >= v0 + kRange) continue;
    bool mine = true;                                // the first entry of a token adds up all of them
    for (int j = 0; j < i; ++j) mine = mine && s_btok[j] != tok;
    if (!mine) continue;
    float sum = 0.f;
    for (int j = i; j < nb; ++j)
      if (s_btok[j] == tok) sum += p.bias_values[static_cast<size_t>(b) * p.max_bias + j];
    s_bias[tok - v0] = sum;
  }
  __syncthreads();

  // z' = (z > 0 ? z / rho : z * rho) + add for a token that is there already, z + add for any other (the product with 1 / rho is one
  // rounding more than a quotient, and one instruction where a division for every logit would be ten)
  const float inv_rho = 1.f / rho;
  float add[kPerThread];
  uint32_t seen = 0;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int off = v_warp + k * 32 + lane;
    const uint32_t c = s_count[off];
    seen |= (c != 0u ? 1u : 0u) << k;
    add[k] = s_bias[off];
    if (c & ~kInPrompt) add[k] -= phi * static_cast<float>(c & ~kInPrompt) + pi;
  }

  // ---- rows
  auto work = [&](int r, const float (&z0)[kPerThread], uint32_t m0) __attribute__((always_inline)) {
    if (r >= r_hi) return;
    float x[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const float f = z0[k] > 0.f ? inv_rho : rho;
      x[k] = (seen >> k) & 1u ? fmaf(z0[k], f, add[k]) : z0[k] + add[k];
    }
    const unsigned long long path = r > 0 ? s_path[r - 1] : 0ull;
    for (unsigned long long left = path; left; left &= left - 1) {
      const int off = s_off[__ffsll(static_cast<long long>(left)) - 1], mine = off - v_warp - lane;
      if (mine < 0 || mine >= 32 * kPerThread || (mine & 31)) continue;      // another lane's token
      int c = static_cast<int>(s_count[off] & ~kInPrompt);
      for (unsigned long long q = path; q; q &= q - 1) c += s_off[__ffsll(static_cast<long long>(q)) - 1] == off;
      const uint32_t hit = 1u << (mine >> 5);        // (a bit per token: a comparison with k would put the rows into local memory)
      const float plus = s_bias[off] - (phi * static_cast<float>(c) + pi);
#pragma unroll
      for (int k = 0; k < kPerThread; ++k)
        if ((hit >> k) & 1u) x[k] = fmaf(z0[k], z0[k] > 0.f ? inv_rho : rho, plus);
    }
    if (p.allowed) {
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) {
        const uint32_t word = __shfl_sync(0xffffffffu, m0, k);
        if (!((word >> lane) & 1u)) x[k] = -INFINITY;
      }
    }
    float* to = p.out + row0 + static_cast<size_t>(r) * p.V + v0 + v_warp + lane;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
      if (k < n_here) __stcs(to + k * 32, x[k]);
  };
  // (two buffers in turn, not moved along: a move would wait for the loads that have just set out)
  for (int r = r_lo; r < r_hi; r += 2) {
    work(r, z0, m0);
    fetch(r + 2, z0, m0);
    work(r + 1, z1, m1);
    fetch(r + 3, z1, m1);
  }
}

}  // namespace

cudaError_t launch_logits(const LogitsParams& p_in, int sm_count, cudaStream_t stream) {
  LogitsParams p = p_in;
  const int ranges = (p.V + kRange - 1) / kRange, rows = p.T + 1;
  // Rows are shared out over several CTAs (each counts the history again): at most 16 to one, so that trees of 16 and of 64
  // nodes end together (135 us for 64 trees x 32000 tokens; 139 us with 33 rows, 143 us with 8), fewer while the CTAs do not fill
  // the machine.
  int splits = (rows + kRowsPerCta - 1) / kRowsPerCta;
  while (static_cast<long long>(ranges) * p.B * splits < 4ll * sm_count && splits < rows) ++splits;
  p.rows_per_block = (rows + splits - 1) / splits;
  const dim3 grid(static_cast<unsigned>(ranges), static_cast<unsigned>(p.B), static_cast<unsigned>((rows + p.rows_per_block - 1) / p.rows_per_block));
  if (p.bf16) logits_kernel<true><<<grid, kLogThreads, 0, stream>>>(p);
  else logits_kernel<false><<<grid, kLogThreads, 0, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace eagle
