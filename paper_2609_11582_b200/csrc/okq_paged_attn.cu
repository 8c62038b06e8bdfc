// Attention over the 8-bit paged cache (okq_paged_attention).
//
// One warp per (layer, sequence, query head, query): it walks the tokens that its query sees with the running maximum and sum of the
// softmax, four channels per lane.
#include "okq_paged_attn.cuh"

namespace okq {

namespace {

constexpr int NT = 128;

template <class T>
__global__ void __launch_bounds__(NT) k_paged_attention(const PagedView c, int layer, const QRows q, const ORows o, int n_new, const int32_t* q_len,
                                                        const RopeView rope, float scale2, long long rows) {
  depend_wait();
  const int lane = threadIdx.x & 31;
  long long u = (long long)blockIdx.x * (NT / 32) + (threadIdx.x >> 5);
  if (u >= rows) return;
  const int i = (int)(u % n_new);
  u /= n_new;
  const int hq = (int)(u % (c.n_kv * c.group));
  u /= c.n_kv * c.group;
  const int b = (int)(u % c.batch), li = (int)(u / c.batch), l = layer + li, h = hq / c.group;
  const int m = count_of(q_len, b, n_new);
  if (i >= m) return;
  const int seen = max(0, c.held(l, b) - m + i + 1);
  const T* qp = static_cast<const T*>(q.p) + li * q.s[0] + b * q.s[1] + hq * q.s[2] + i * q.s[3];
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int ch = 4 * lane + e;
    x[e] = to_f(qp[ch]);
    if (rope.freq && ch < 2 * rope.half) {
      const int pair = ch < rope.half ? ch : ch - rope.half;
      float cs, sn, a = to_f(qp[pair]), d = to_f(qp[pair + rope.half]);
      const size_t step = (size_t)c.batch * n_new;
      turn((double)rope.positions[rope.axis(pair) * step + (size_t)b * n_new + i] * rope.freq[pair], cs, sn);
      rotate_pair(a, d, cs, sn);
      x[e] = to_f(from_f<T>(ch < rope.half ? a : d));
    }
  }
  float mx = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  bool lost = false;
  for (int t = 0; t < seen; t++) {
    const int page = c.page_of(b, t);
    if (page < 0) { lost = true; break; }
    const size_t kr = c.code_row(l, page, h, 0) + (t & (c.page - 1)), vr = kr + c.page;
    const char4 kc = *reinterpret_cast<const char4*>(c.codes + kr * D + 4 * lane), vc = *reinterpret_cast<const char4*>(c.codes + vr * D + 4 * lane);
    float s = x[0] * kc.x + x[1] * kc.y + x[2] * kc.z + x[3] * kc.w;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= c.scales[kr / PB] * scale2;
    const float mn = fmaxf(mx, s), f = exp2f(mx - mn), p = exp2f(s - mn), pv = p * c.scales[vr / PB];
    mx = mn;
    sum = sum * f + p;
    acc[0] = acc[0] * f + pv * vc.x;
    acc[1] = acc[1] * f + pv * vc.y;
    acc[2] = acc[2] * f + pv * vc.z;
    acc[3] = acc[3] * f + pv * vc.w;
  }
  if (lost && lane == 0) set_status(c.status, OKQ_ERR_INVALID_ARG);
  T* op = static_cast<T*>(o.p) + li * o.s[0] + b * o.s[1] + hq * o.s[2] + i * o.s[3];
#pragma unroll
  for (int e = 0; e < 4; e++) op[4 * lane + e] = from_f<T>(lost ? NAN : seen == 0 ? 0.f : acc[e] / sum);
}

// tiles that a call could have, were all sequences as long as their rows of the table
long long most_tiles(const okq_paged* c, int layer_count, int n_new) {
  const long long units = (long long)layer_count * c->batch * c->n_kv_heads, rows = (long long)n_new * (c->n_q_heads / c->n_kv_heads);
  return units * ((rows + DECODE_ROWS - 1) / DECODE_ROWS) * (((long long)c->max_pages * c->page_tokens + PT - 1) / PT);
}

// blocks of the attention kernel: one per SM, no more than there could be tiles
int grid_of(const okq_paged* c, int layer_count, int n_new) {
  const long long tiles = most_tiles(c, layer_count, n_new), n = sm_count();
  return (int)(tiles < n ? tiles : n);
}

okq_status failed(cudaError_t e) {
  set_last_cuda_error((int)e);
  (void)cudaGetLastError();
  return OKQ_ERR_CUDA;
}

}  // namespace

}  // namespace okq

extern "C" {

size_t okq_paged_workspace_bytes(const okq_paged* cache, int32_t layer_count, int32_t n_new) {
  if (okq::check_paged(cache, false) != OKQ_OK || layer_count <= 0 || layer_count > cache->n_layers || n_new < 0) return 0;
  const size_t slots = okq::attn_workspace(okq::DECODE_PIPES * okq::grid_of(cache, layer_count, n_new), okq::DECODE_ROWS);
  const size_t pages = okq::pages_workspace(cache);
  return ((slots > pages ? slots : pages) + 255) & ~(size_t)255;
}

okq_status okq_paged_attention(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t qs[4], int32_t n_new,
                               const int32_t* q_len, const okq_rope* rope, float sm_scale, void* workspace, size_t workspace_bytes, void* out,
                               const int64_t os[4], void* stream) {
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
  if (!workspace || workspace_bytes < okq_paged_workspace_bytes(cache, layer_count, n_new)) return OKQ_ERR_WORKSPACE;
  const PagedView c = paged_view(cache);
  if (c.group * n_new <= DECODE_ROWS) {
    if (most_tiles(cache, layer_count, n_new) > INT32_MAX) return OKQ_ERR_UNSUPPORTED;
    AttnArgs a{c, {q, {qs[0], qs[1], qs[2], qs[3]}}, {out, {os[0], os[1], os[2], os[3]}}, q_len, r, layer, layer_count, n_new,
               sm_scale * 1.44269504088896340736f, static_cast<Head*>(workspace), nullptr};
    const int grid = grid_of(cache, layer_count, n_new);
    a.slots = reinterpret_cast<float*>(a.heads + DECODE_PIPES * grid);
    const cudaError_t e = launch_paged_decode(a, cache->dtype, grid, static_cast<cudaStream_t>(stream));
    return e != cudaSuccess ? failed(e) : launch_status();
  }
  const long long rows = (long long)layer_count * c.batch * c.n_kv * c.group * n_new, grid = (rows + NT / 32 - 1) / (NT / 32);
  if (grid > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  const QRows qr{q, {qs[0], qs[1], qs[2], qs[3]}};
  const ORows orow{out, {os[0], os[1], os[2], os[3]}};
  const float scale2 = sm_scale * 1.44269504088896340736f;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->dtype == OKQ_FP16
      ? launch_dependent(k_paged_attention<__half>, dim3((unsigned)grid), NT, 0, s, 1, c, layer, qr, orow, n_new, q_len, r, scale2, rows)
      : launch_dependent(k_paged_attention<__nv_bfloat16>, dim3((unsigned)grid), NT, 0, s, 1, c, layer, qr, orow, n_new, q_len, r, scale2, rows);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // extern "C"
