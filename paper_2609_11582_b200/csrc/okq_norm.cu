// Root-mean-square norm of every head of queries and keys with the rotary positions in the same pass (okq_norm_rope_apply), and its
// gradients (okq_norm_rope_grad).  For a row x of 128 channels with weight w, R the rotation of its token:
//     r = (mean(x^2) + eps)^(-1/2),  y = R (w x r)
//     u = R^T g,  dw = sum over rows of u x r,  dx = r (w u - x r mean(x r w u))
// all in 32 bits, rounded once at the end.
//
// Both are bound by memory: every element is read once (x, and g) and written once.  Eight lanes have a token's row of a head, sixteen
// channels each in two pieces of 16 bytes (32 in fp32), which hold both channels of each pair they turn; the row's sums take three
// exchanges.  A thread keeps its token's cosines and sines, and the weights, over a range of heads.  The backward pass keeps its sums
// for the weights in registers too: a block works through tokens of one side, queries or keys, leaves one row of 128 sums at the end,
// and a second kernel adds these rows in a fixed order.
#include "okq_paged.cuh"

namespace okq {

namespace {

constexpr int NT = 128, TOKENS = NT / 8;
// blocks of the backward pass: as many as the GPU holds at once, or more (148 SMs, up to eight each)
constexpr int GRAD_BLOCKS = 1184;

struct NormSide {
  const void *in, *up;
  void* out;
  int64_t is[3], us[3], os[3];
  const void* weight;
  float* weight_grad;
  int weight_dtype, heads, groups;   // groups: parts that the heads are cut into, `per` heads each
};

// the thread's sixteen channels: eight from c0, eight from c1
struct Place {
  int c0, c1;
  bool turns;
  __device__ __forceinline__ Place(const RopeView& rope, int j) {
    const int half = rope.half ? rope.half : 64, nc = half >> 3;   // (without a rotation laid out, and added up, as with one of all channels)
    turns = rope.half && j < nc;
    c0 = j < nc ? 8 * j : 2 * half + 16 * (j - nc);
    c1 = j < nc ? c0 + half : c0 + 8;
  }
};

template <class T> __device__ __forceinline__ void weights8(const T* w, int c, float (&to)[16], int at) {
  const Vec8<T> x = *reinterpret_cast<const Vec8<T>*>(w + c);
#pragma unroll
  for (int e = 0; e < 8; e++) to[at + e] = to_f(x.v[e]);
}
__device__ __forceinline__ void load_weights(const NormSide& x, const Place& p, float (&w)[16]) {
#pragma unroll
  for (int z = 0; z < 2; z++) {
    const int c = z ? p.c1 : p.c0;
    if (!x.weight) {
#pragma unroll
      for (int e = 0; e < 8; e++) w[8 * z + e] = 1.f;
    } else if (x.weight_dtype == OKQ_FP16) weights8(static_cast<const __half*>(x.weight), c, w, 8 * z);
    else if (x.weight_dtype == OKQ_BF16) weights8(static_cast<const __nv_bfloat16*>(x.weight), c, w, 8 * z);
    else weights8(static_cast<const float*>(x.weight), c, w, 8 * z);
  }
}

__device__ __forceinline__ float row_sum(float x) {   // over the eight lanes of a row; the same number in each
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

template <class T> struct Row {
  Vec8<T> a, b;
  __device__ __forceinline__ void load(const void* p, int64_t at, const Place& pl) {
    const T* x = static_cast<const T*>(p) + at;
    a = *reinterpret_cast<const Vec8<T>*>(x + pl.c0);
    b = *reinterpret_cast<const Vec8<T>*>(x + pl.c1);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < 8; e++) a.v[e] = b.v[e] = from_f<T>(0.f);
  }
  __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
    for (int e = 0; e < 8; e++) { x[e] = to_f(a.v[e]); x[8 + e] = to_f(b.v[e]); }
  }
  __device__ __forceinline__ void put(const float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 8; e++) { a.v[e] = from_f<T>(x[e]); b.v[e] = from_f<T>(x[8 + e]); }
  }
  __device__ __forceinline__ void store(void* p, int64_t at, const Place& pl) const {
    T* x = static_cast<T*>(p) + at;
    *reinterpret_cast<Vec8<T>*>(x + pl.c0) = a;
    *reinterpret_cast<Vec8<T>*>(x + pl.c1) = b;
  }
};

// x becomes x r; returns r, times 2^96 where the row was multiplied by 2^-96 because its squares have no sum in fp32 (fp16 rows never are)
__device__ __forceinline__ float normalise(float (&x)[16], float eps, bool& scaled) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 16; e++) s = fmaf(x[e], x[e], s);
  s = row_sum(s);
  scaled = s > 1e37f;
  if (__any_sync(0xffffffffu, scaled)) {
    const float f = scaled ? 1.2621774483536189e-29f : 1.f;   // 2^-96: eps is nothing beside such rows
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) {
      x[e] *= f;
      z = fmaf(x[e], x[e], z);
    }
    z = row_sum(z);
    if (scaled) s = z;
  }
  const float r = __frsqrt_rn(fmaf(s, 1.f / D, scaled ? 0.f : eps));
#pragma unroll
  for (int e = 0; e < 16; e++) x[e] *= r;
  return r;
}

// grid (16 tokens, range of heads): first the queries' ranges, then the keys'
template <class T>
__global__ void __launch_bounds__(NT) k_norm_rope(const RopeView rope, const NormSide q, const NormSide k, float eps, int batch, int n, int per) {
  constexpr int G = sizeof(T) == 4 ? 2 : 4;   // heads at a time, all their loads first (in place, stores alias them)
  depend_wait();
  const bool is_q = (int)blockIdx.y < q.groups;
  const NormSide& x = is_q ? q : k;
  const int h_first = ((int)blockIdx.y - (is_q ? 0 : q.groups)) * per, h_end = min(x.heads, h_first + per);
  const long long tok = (long long)blockIdx.x * TOKENS + (threadIdx.x >> 3);
  const int b = (int)(tok / n), i = (int)(tok % n);
  const bool there = b < batch;
  const Place pl(rope, threadIdx.x & 7);
  const int64_t in0 = (int64_t)b * x.is[0] + (int64_t)i * x.is[2], out0 = (int64_t)b * x.os[0] + (int64_t)i * x.os[2];
  float w[16], cs[8] = {}, sn[8] = {};
  for (int h0 = h_first; h0 < h_end; h0 += G) {
    Row<T> row[G];
#pragma unroll
    for (int g = 0; g < G; g++) {
      if (there && h0 + g < h_end) row[g].load(x.in, in0 + (h0 + g) * x.is[1], pl);
      else row[g].zero();
    }
    if (h0 == h_first) {   // (while the first rows are on their way)
      load_weights(x, pl, w);
      if (pl.turns && there) turns8(rope, rope.positions + (size_t)b * n + i, (size_t)batch * n, pl.c0, cs, sn);
    }
#pragma unroll
    for (int g = 0; g < G; g++) {
      if (h0 + g >= h_end) break;
      float y[16];
      bool scaled;
      row[g].get(y);
      normalise(y, eps, scaled);
#pragma unroll
      for (int e = 0; e < 16; e++) y[e] *= w[e];
      if (pl.turns) {
#pragma unroll
        for (int e = 0; e < 8; e++) rotate_pair(y[e], y[8 + e], cs[e], sn[e]);
      }
      row[g].put(y);
      if (there) row[g].store(x.out, out0 + (h0 + g) * x.os[1], pl);
    }
  }
}

// Blocks 0 .. q_blocks - 1 work on queries, the others on keys, each on every so many-th unit of its side: 16 tokens and a range of heads.
// partial[block][128]: what the block's rows add to the weight's gradient.
template <class T>
__global__ void __launch_bounds__(NT) k_norm_rope_grad(const RopeView rope, const NormSide q, const NormSide k, float eps, int batch, int n, int per,
                                                        int q_blocks, long long tiles, float* partial) {
  __shared__ float sums[NT / 32][8][17];
  depend_wait();
  const bool is_q = (int)blockIdx.x < q_blocks;
  const NormSide& x = is_q ? q : k;
  const int who = is_q ? blockIdx.x : blockIdx.x - q_blocks, n_who = is_q ? q_blocks : gridDim.x - q_blocks;
  const Place pl(rope, threadIdx.x & 7);
  float w[16], dw[16];
  load_weights(x, pl, w);
#pragma unroll
  for (int e = 0; e < 16; e++) dw[e] = 0.f;
  for (long long unit = who; unit < tiles * x.groups; unit += n_who) {
    const long long tile = unit / x.groups, tok = tile * TOKENS + (threadIdx.x >> 3);
    const int h_first = (int)(unit - tile * x.groups) * per, h_end = min(x.heads, h_first + per);
    const int b = (int)(tok / n), i = (int)(tok % n);
    const bool there = b < batch;
    const int64_t in0 = (int64_t)b * x.is[0] + (int64_t)i * x.is[2], up0 = (int64_t)b * x.us[0] + (int64_t)i * x.us[2], out0 = (int64_t)b * x.os[0] + (int64_t)i * x.os[2];
    float cs[8] = {}, sn[8] = {};   // (rows behind the last token add nothing to the weights' sums)
    constexpr int G = 2;
    for (int h0 = h_first; h0 < h_end; h0 += G) {
      Row<T> row[G], up[G];
#pragma unroll
      for (int g = 0; g < G; g++) {
        if (there && h0 + g < h_end) {
          row[g].load(x.in, in0 + (h0 + g) * x.is[1], pl);
          up[g].load(x.up, up0 + (h0 + g) * x.us[1], pl);
        } else {
          row[g].zero();
          up[g].zero();
        }
      }
      if (h0 == h_first && pl.turns && there) turns8(rope, rope.positions + (size_t)b * n + i, (size_t)batch * n, pl.c0, cs, sn);
#pragma unroll
      for (int g = 0; g < G; g++) {
        if (h0 + g >= h_end) break;
        float y[16], u[16];
        bool scaled;
        row[g].get(y);
        up[g].get(u);
        const float r = normalise(y, eps, scaled);
        if (pl.turns) {
#pragma unroll
          for (int e = 0; e < 8; e++) rotate_pair(u[e], u[8 + e], cs[e], -sn[e]);
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          dw[e] = fmaf(u[e], y[e], dw[e]);
          u[e] *= w[e];
          dot = fmaf(u[e], y[e], dot);
        }
        dot = row_sum(dot) * (1.f / D);
#pragma unroll
        for (int e = 0; e < 16; e++) {
          u[e] = fmaf(-y[e], dot, u[e]) * r;
          if (scaled) u[e] *= 1.2621774483536189e-29f;
        }
        up[g].put(u);
        if (there) up[g].store(x.out, out0 + (h0 + g) * x.os[1], pl);
      }
    }
  }
  if (!x.weight_grad) return;
#pragma unroll
  for (int e = 0; e < 16; e++) {
    dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], 8);
    dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], 16);
  }
  const int lane = threadIdx.x & 31;
  if (lane < 8) {
#pragma unroll
    for (int e = 0; e < 16; e++) sums[threadIdx.x >> 5][lane][e] = dw[e];
  }
  __syncthreads();
  const int j = threadIdx.x >> 4, e = threadIdx.x & 15;
  const Place mine(rope, j);
  partial[(size_t)blockIdx.x * D + (e < 8 ? mine.c0 + e : mine.c1 + e - 8)] = (sums[0][j][e] + sums[1][j][e]) + (sums[2][j][e] + sums[3][j][e]);
}

// Block (x, side): sums of eight channels over the side's rows, 32 threads to each, row by row and then in a tree: always the same order.
__global__ void __launch_bounds__(256) k_norm_weight_grad(const float* partial, int q_blocks, int blocks, float* q_grad, float* k_grad) {
  __shared__ float sums[32][9];
  depend_wait();
  const int side = blockIdx.y, c = threadIdx.x & 7, r = threadIdx.x >> 3;
  float* to = side ? k_grad : q_grad;
  if (!to) return;
  const int first = side ? q_blocks : 0, last = side ? blocks : q_blocks;
  float s = 0.f;
#pragma unroll 8
  for (int row = first + r; row < last; row += 32) s += __ldcg(&partial[(size_t)row * D + 8 * blockIdx.x + c]);
  sums[r][c] = s;
  __syncthreads();
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) {
    if (r < d) sums[r][c] += sums[r + d][c];
    __syncthreads();
  }
  if (r == 0) to[8 * blockIdx.x + c] = sums[0][c];
}

okq_status failed(cudaError_t e) {
  set_last_cuda_error((int)e);
  (void)cudaGetLastError();
  return OKQ_ERR_CUDA;
}

// (a tensor without rows may have no address)
okq_status check_sides(int32_t dtype, bool rows, const okq_norm_tensor* q, const okq_norm_tensor* k, bool grad, NormSide (&side)[2]) {
  if (dtype != OKQ_FP16 && dtype != OKQ_BF16 && dtype != OKQ_FP32) return OKQ_ERR_UNSUPPORTED;
  for (int t = 0; t < 2; t++) {
    const okq_norm_tensor* x = t ? k : q;
    NormSide& s = side[t];
    s = NormSide{};
    if (!x) continue;
    if (x->heads < 0 || (rows && x->heads > 0 && (!x->in || !x->out || (grad && !x->grad_out)))) return OKQ_ERR_INVALID_ARG;
    if (x->weight && x->weight_dtype != OKQ_FP16 && x->weight_dtype != OKQ_BF16 && x->weight_dtype != OKQ_FP32) return OKQ_ERR_UNSUPPORTED;
    const int m = dtype == OKQ_FP32 ? 4 : 8;
    if (!aligned16(x->in) || !aligned16(x->out) || !aligned16(x->weight) || !strides_ok(x->in_strides, 3, m) || !strides_ok(x->out_strides, 3, m))
      return OKQ_ERR_ALIGNMENT;
    if (grad && (!aligned16(x->grad_out) || !aligned16(x->weight_grad) || !strides_ok(x->grad_strides, 3, m))) return OKQ_ERR_ALIGNMENT;
    s.in = x->in; s.up = x->grad_out; s.out = x->out;
    s.weight = x->weight; s.weight_dtype = x->weight_dtype; s.weight_grad = grad ? x->weight_grad : nullptr;
    s.heads = x->heads;
    for (int i = 0; i < 3; i++) { s.is[i] = x->in_strides[i]; s.us[i] = x->grad_strides[i]; s.os[i] = x->out_strides[i]; }
  }
  return (long long)side[0].heads + side[1].heads > 65535 ? OKQ_ERR_UNSUPPORTED : OKQ_OK;
}

// parts that `heads` heads are cut into, `per` each
int parts(int heads, int per) { return (heads + per - 1) / per; }

template <class T> cudaError_t launch_apply(const RopeView& r, NormSide (&x)[2], float eps, int batch, int n, cudaStream_t s) {
  const long long blocks = ((long long)batch * n + TOKENS - 1) / TOKENS;
  const int heads = x[0].heads > x[1].heads ? x[0].heads : x[1].heads;
  // heads per thread: as many as leave the GPU's threads busy
  const long long want = 16ll * sm_count();
  const int groups = (int)((want + blocks - 1) / blocks < heads ? (want + blocks - 1) / blocks : heads), per = (heads + groups - 1) / groups;
  for (NormSide& y : x) y.groups = parts(y.heads, per);
  return launch_dependent(k_norm_rope<T>, dim3((unsigned)blocks, (unsigned)(x[0].groups + x[1].groups)), NT, 0, s, 1, r, x[0], x[1], eps, batch, n, per);
}

// Backward: how the heads are cut, and the blocks of both sides, in proportion to their units.
struct GradPlan {
  int per, blocks[2];
  long long tiles;
  GradPlan(long long rows, int q_heads, int k_heads) {
    tiles = (rows + TOKENS - 1) / TOKENS;
    const int heads[2] = {q_heads, k_heads};
    const long long all = (long long)q_heads + k_heads;
    per = 8;
    while (per > 1 && tiles * (parts(q_heads, per) + parts(k_heads, per)) < GRAD_BLOCKS) per >>= 1;
    for (int t = 0; t < 2; t++) {
      const long long units = tiles * parts(heads[t], per), share = all ? (GRAD_BLOCKS * (long long)heads[t] + all - 1) / all : 0;
      blocks[t] = (int)(units < share ? units : share);
    }
  }
};

template <class T> cudaError_t launch_grad(const RopeView& r, NormSide (&x)[2], float eps, int batch, int n, const GradPlan& p, float* partial, cudaStream_t s) {
  for (NormSide& y : x) y.groups = parts(y.heads, p.per);
  const int blocks = p.blocks[0] + p.blocks[1];
  const cudaError_t e = launch_dependent(k_norm_rope_grad<T>, dim3((unsigned)blocks), NT, 0, s, 1, r, x[0], x[1], eps, batch, n, p.per, p.blocks[0], p.tiles, partial);
  if (e != cudaSuccess || (!x[0].weight_grad && !x[1].weight_grad)) return e;
  return launch_dependent(k_norm_weight_grad, dim3(D / 8, 2), 256, 0, s, 1, partial, p.blocks[0], blocks, x[0].weight_grad, x[1].weight_grad);
}

}  // namespace

}  // namespace okq

extern "C" {

okq_status okq_norm_rope_apply(const okq_rope* rope, float eps, int32_t dtype, int32_t batch, int32_t n, const okq_norm_tensor* q,
                               const okq_norm_tensor* k, void* stream) {
  using namespace okq;
  if (!q || batch < 0 || n < 0 || !(eps >= 1e-30f && eps <= 3e38f)) return OKQ_ERR_INVALID_ARG;
  NormSide x[2];
  okq_status st = check_sides(dtype, batch > 0 && n > 0, q, k, false, x);
  if (st != OKQ_OK) return st;
  RopeView r;
  if ((st = make_rope(rope, r)) != OKQ_OK) return st;
  if (batch == 0 || n == 0 || x[0].heads + x[1].heads == 0) return OKQ_OK;
  if (((long long)batch * n + TOKENS - 1) / TOKENS > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OKQ_FP16   ? launch_apply<__half>(r, x, eps, batch, n, s)
                        : dtype == OKQ_BF16 ? launch_apply<__nv_bfloat16>(r, x, eps, batch, n, s)
                                            : launch_apply<float>(r, x, eps, batch, n, s);
  return e != cudaSuccess ? failed(e) : launch_status();
}

size_t okq_norm_rope_workspace_bytes(int32_t batch, int32_t n, int32_t q_heads, int32_t k_heads) {
  if (batch < 0 || n < 0 || q_heads < 0 || k_heads < 0 || (long long)q_heads + k_heads > 65535) return 0;
  // a row for each block (both sides' shares are rounded up), whatever the sizes: scratch for one call serves every other
  return (size_t)(okq::GRAD_BLOCKS + 2) * okq::D * sizeof(float);
}

okq_status okq_norm_rope_grad(const okq_rope* rope, float eps, int32_t dtype, int32_t batch, int32_t n, const okq_norm_tensor* q,
                              const okq_norm_tensor* k, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace okq;
  if (!q || batch < 0 || n < 0 || !(eps >= 1e-30f && eps <= 3e38f)) return OKQ_ERR_INVALID_ARG;
  NormSide x[2];
  okq_status st = check_sides(dtype, batch > 0 && n > 0, q, k, true, x);
  if (st != OKQ_OK) return st;
  if (!aligned16(workspace)) return OKQ_ERR_ALIGNMENT;
  RopeView r;
  if ((st = make_rope(rope, r)) != OKQ_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool sums = x[0].weight_grad || x[1].weight_grad;
  if (batch == 0 || n == 0 || x[0].heads + x[1].heads == 0) {   // no rows: sums of nothing
    const cudaError_t e = sums ? launch_dependent(k_norm_weight_grad, dim3(D / 8, 2), 256, 0, s, 1, nullptr, 0, 0, x[0].weight_grad, x[1].weight_grad) : cudaSuccess;
    return e != cudaSuccess ? failed(e) : OKQ_OK;
  }
  if (sums && (!workspace || workspace_bytes < okq_norm_rope_workspace_bytes(batch, n, x[0].heads, x[1].heads))) return OKQ_ERR_WORKSPACE;
  const GradPlan p((long long)batch * n, x[0].heads, x[1].heads);
  float* partial = static_cast<float*>(workspace);
  const cudaError_t e = dtype == OKQ_FP16   ? launch_grad<__half>(r, x, eps, batch, n, p, partial, s)
                        : dtype == OKQ_BF16 ? launch_grad<__nv_bfloat16>(r, x, eps, batch, n, p, partial, s)
                                            : launch_grad<float>(r, x, eps, batch, n, p, partial, s);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // extern "C"
