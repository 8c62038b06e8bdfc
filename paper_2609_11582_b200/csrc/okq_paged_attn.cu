// Attention over the 8-bit paged cache (okq_paged_attention, with a window, for a tree of drafted tokens): checks, workspace, and which of the
// two kernels takes a call.
//
// Rows (query x head of the GQA group) of a KV head are cut into row tiles: eight rows in the decode kernel, whose products have eight
// columns for them and read the codes as they are, 256 in the prompt kernel, which turns codes into fp16.  Both read a head's tokens once
// per row tile.
#include "okq_paged_attn.cuh"

namespace okq {

namespace {

struct Plan {
  bool decode;
  int grid, ranges;         // blocks of the line of tiles, its parts
  int cluster;              // decode: blocks to a (layer, sequence, KV head), 0 where the line is cut evenly
  size_t heads, bytes;      // of the workspace: heads; what any plan for as many layers and queries or fewer takes
};

// Which kernel, for sequences as long as their rows of the table (lengths are the device's).  Measured in turn, us:
//   rows up to 16: the decode kernel (12 rows, 16 sequences x 4 heads of up to 12345 tokens 43 against 62; 32768 each 174 against 228)
//   up to 24 where two thirds of the three readings come from the second-level cache (1 sequence x 4 heads of 131072 tokens 58 against
//   75; 16 x 4 of 32768 253 against 232; 32 rows: 76 against 76 and 333 against 234)
//   any number of rows with items so few that each can have a cluster of blocks: one launch, no search for the first tile, no merge
//   kernel, parts put together in shared memory.  An item has no more than its cluster's pipelines then, so both sides are reckoned in
//   tiles (2 us), fixed costs included (64 rows of 1 head of 2048 tokens 8.0 against 17.2, 192 rows of 4 heads of 1000 tokens 14.1 against
//   22.8; 8 rows, 4 heads of 131072 tokens: 34 in the line, 90 as clusters; 96 rows of 8 heads of 4000 tokens 22 by the prompt kernel).
// A window (0: none) bounds what an item reads: its own tokens and the sinks', tiles that are begun included.  Fewer tiles to an item need no
// more scratch, so that without a window serves every call.
// False: more units than their numbers hold.
bool make_plan(const okq_paged* c, int layer_count, int n_new, int window, int sinks, Plan& p) {
  const int group = c->n_q_heads / c->n_kv_heads;
  const long long rows = (long long)n_new * group;
  if (rows > 1 << 29) return false;
  const long long room = ((long long)c->max_pages * c->page_tokens + PT - 1) / PT, n = sm_count();
  auto tiles_of = [&](long long per) {   // of an item of `per` rows
    if (!window) return room;
    const long long queries = ((rows < per ? rows : per) - 1) / group + 2;
    const long long t = ((long long)sinks + PT - 1) / PT + (window + queries + PT - 2) / PT + 1;
    return t < room ? t : room;
  };
  const long long per_few = tiles_of(DECODE_ROWS), per_many = tiles_of(PROMPT_ROWS);
  const double heads = (double)layer_count * c->batch * c->n_kv_heads;
  auto items_of = [&](int per) { return heads * (double)((rows + per - 1) / per); };
  const double few = items_of(DECODE_ROWS), many = items_of(PROMPT_ROWS);
  auto in_line = [&](double items, long long per, int extra, int pipes) { return (long long)(items * (double)(per + extra) / (double)(pipes * n)) + 1; };
  p.decode = rows <= 2 * DECODE_ROWS || (rows <= 3 * DECODE_ROWS && heads * (double)per_few <= 8192.0);   // (tiles of 32 KB)
  p.cluster = 0;
  if (few <= n) {
    const long long other = p.decode ? in_line(few, per_few, DECODE_EXTRA, DECODE_PIPES) + 2 : in_line(many, per_many, PROMPT_EXTRA, 1) + 4;
    for (int size = 8; size >= 1 && p.cluster == 0; size--)   // (the largest that all run at once: 15 of eight blocks, 22 of six, 33 of four, 74 of two)
      if (few <= decode_clusters(size) && (per_few + DECODE_PIPES * size - 1) / (DECODE_PIPES * size) <= other) p.cluster = size;
    if (p.cluster) p.decode = true;
  }
  // blocks, ranges and bytes of the line (the workspace is the line's, cluster or not)
  auto line = [&](bool decode) {
    const double tiles = decode ? few * (double)per_few : many * (double)per_many;
    p.grid = (int)(tiles < (double)n ? tiles : (double)n);
    p.ranges = p.grid * (decode ? DECODE_PIPES : 1);
    p.heads = (size_t)p.ranges * sizeof(Head);
    return p.heads + (size_t)2 * p.ranges * (decode ? DECODE_ROWS : PROMPT_ROWS) * (D + 2) * sizeof(float);
  };
  const size_t other = rows > 2 * DECODE_ROWS ? line(!p.decode) : 0, own = line(p.decode);
  p.bytes = own > other ? own : other;
  if ((p.decode ? few * (double)(per_few + DECODE_EXTRA) : many * (double)(per_many + PROMPT_EXTRA)) > 2147483647.0) return false;
  return true;
}

}  // namespace

}  // namespace okq

extern "C" {

size_t okq_paged_workspace_bytes(const okq_paged* cache, int32_t layer_count, int32_t n_new) {
  using namespace okq;
  Plan p{};
  if (check_paged(cache, false) != OKQ_OK || layer_count <= 0 || layer_count > cache->n_layers || n_new < 0) return 0;
  if (n_new > 0 && !make_plan(cache, layer_count, n_new, 0, 0, p)) return 0;
  const size_t pages = pages_workspace(cache);
  return ((p.bytes > pages ? p.bytes : pages) + 255) & ~(size_t)255;
}

// what a query sees: all with neither window nor seen
struct AttnSight {
  int32_t window, sinks;
  const uint64_t* seen;
};

static okq_status attention(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                            const int32_t* q_len, const okq_rope* rope, float sm_scale, void* workspace, size_t workspace_bytes, void* out,
                            const int64_t os[4], const AttnSight& sight, long long limit, int withhold, void* stream) {
  using namespace okq;
  okq_status st = check_paged_layers(cache, layer, layer_count);
  if (st != OKQ_OK) return st;
  if (n_new < 0 || (n_new > 0 && (!q || !out)) || !qs || !os) return OKQ_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !strides_ok(qs, 4, 8) || !strides_ok(os, 4, 8) ||
      (reinterpret_cast<uintptr_t>(q_len) & 3))
    return OKQ_ERR_ALIGNMENT;
  RopeView r;
  if ((st = make_rope(rope, r)) != OKQ_OK) return st;
  if (n_new == 0) return OKQ_OK;
  Plan p;
  // (with a window there may be a plan for rows that no scratch is known for)
  const size_t need = okq_paged_workspace_bytes(cache, layer_count, n_new);
  if (need == 0 || !make_plan(cache, layer_count, n_new, sight.window, sight.sinks, p)) return OKQ_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < need) return OKQ_ERR_WORKSPACE;
  AttnArgs a{paged_view(cache), {q, {qs[0], qs[1], qs[2], qs[3]}}, {out, {os[0], os[1], os[2], os[3]}}, q_len, r, layer, layer_count, n_new,
             sm_scale * 1.44269504088896340736f, limit, withhold, static_cast<Head*>(workspace),
             reinterpret_cast<float*>(static_cast<char*>(workspace) + p.heads), sight.window, sight.sinks,
             reinterpret_cast<const unsigned long long*>(sight.seen), (n_new + 63) / 64};
  const Sight how = sight.window ? WINDOW : sight.seen ? TREE : CAUSAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p.decode ? launch_paged_decode(a, cache->dtype, how, p.grid, p.cluster, s) : launch_paged_prompt(a, cache->dtype, how, p.grid, s);
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    (void)cudaGetLastError();
    return OKQ_ERR_CUDA;
  }
  return launch_status();
}

okq_status okq_paged_attention(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                               const int32_t* q_len, const okq_rope* rope, float sm_scale, void* workspace, size_t workspace_bytes, void* out,
                               const int64_t os[4], void* stream) {
  return attention(cache, layer, layer_count, q, qs, n_new, q_len, rope, sm_scale, workspace, workspace_bytes, out, os, {}, okq::WAIT_LIMIT_CLOCKS, 0, stream);
}

// a window that leaves no token of a full row out is none
static AttnSight window_of(const okq_paged* cache, int32_t window, int32_t sinks) {
  const long long room = (long long)cache->max_pages * cache->page_tokens;
  return window >= room || sinks >= room ? AttnSight{} : AttnSight{window, sinks, nullptr};
}

okq_status okq_paged_attention_window(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                                      const int32_t* q_len, const okq_rope* rope, float sm_scale, int32_t window, int32_t sinks, void* workspace,
                                      size_t workspace_bytes, void* out, const int64_t os[4], void* stream) {
  if (!cache || window <= 0 || sinks < 0) return OKQ_ERR_INVALID_ARG;
  return attention(cache, layer, layer_count, q, qs, n_new, q_len, rope, sm_scale, workspace, workspace_bytes, out, os, window_of(cache, window, sinks),
                   okq::WAIT_LIMIT_CLOCKS, 0, stream);
}

okq_status okq_paged_attention_tree(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                                    const int32_t* q_len, const okq_rope* rope, float sm_scale, const uint64_t* seen, void* workspace,
                                    size_t workspace_bytes, void* out, const int64_t os[4], void* stream) {
  if (n_new > 0 && !seen) return OKQ_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(seen) & 7) return OKQ_ERR_ALIGNMENT;
  return attention(cache, layer, layer_count, q, qs, n_new, q_len, rope, sm_scale, workspace, workspace_bytes, out, os, {0, 0, seen},
                   okq::WAIT_LIMIT_CLOCKS, 0, stream);
}

okq_status okq_debug_paged_timeout(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                                   void* workspace, size_t workspace_bytes, void* out, const int64_t os[4], int64_t limit_clocks, void* stream) {
  if (limit_clocks <= 0) return OKQ_ERR_INVALID_ARG;
  return attention(cache, layer, layer_count, q, qs, n_new, nullptr, nullptr, 0.08838834764831845f, workspace, workspace_bytes, out, os, {}, limit_clocks, 1, stream);
}

okq_status okq_debug_paged_timeout_sight(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                                         int32_t window, int32_t sinks, const uint64_t* seen, void* workspace, size_t workspace_bytes, void* out,
                                         const int64_t os[4], int64_t limit_clocks, void* stream) {
  if (!cache || limit_clocks <= 0 || window < 0 || sinks < 0 || (window > 0) == (seen != nullptr)) return OKQ_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(seen) & 7) return OKQ_ERR_ALIGNMENT;
  return attention(cache, layer, layer_count, q, qs, n_new, nullptr, nullptr, 0.08838834764831845f, workspace, workspace_bytes, out, os,
                   seen ? AttnSight{0, 0, seen} : window_of(cache, window, sinks), limit_clocks, 1, stream);
}

static int32_t plan_of(const okq_paged* cache, int32_t layer_count, int32_t n_new, const AttnSight& sight) {
  okq::Plan p;
  if (layer_count <= 0 || layer_count > cache->n_layers || n_new <= 0 || okq_paged_workspace_bytes(cache, layer_count, n_new) == 0 ||
      !okq::make_plan(cache, layer_count, n_new, sight.window, sight.sinks, p)) return 0;
  return p.decode ? (p.cluster ? p.cluster : OKQ_PLAN_LINE) : OKQ_PLAN_PROMPT;
}

int32_t okq_debug_paged_plan(const okq_paged* cache, int32_t layer_count, int32_t n_new) {
  return okq::check_paged(cache, false) != OKQ_OK ? 0 : plan_of(cache, layer_count, n_new, {});
}

int32_t okq_debug_paged_plan_window(const okq_paged* cache, int32_t layer_count, int32_t n_new, int32_t window, int32_t sinks) {
  if (okq::check_paged(cache, false) != OKQ_OK || window <= 0 || sinks < 0) return 0;
  return plan_of(cache, layer_count, n_new, window_of(cache, window, sinks));
}

}  // extern "C"
