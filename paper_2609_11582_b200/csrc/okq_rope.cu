// Rotary positions with three axes (okq_rope_apply): channels c and c + pairs of every head are one point of the plane, turned by
// positions[axis(c)] * freq[c].  Backwards is the same with the opposite sign, the rotation's transpose.
//
// Bound by memory: every element is read and written once.  A thread has eight channel pairs of one token and walks a range of
// heads with the sines and cosines in registers, so that they are worked out once per token and not once per head; the eight threads of a
// token read 128 consecutive bytes at a time.  8191 tokens x 36 heads in fp32, there and back: 114 us, 5.3 TB/s; one token of 8 sequences 4.3
// us, a launch and the turn.
#include "okq_paged.cuh"

namespace okq {

namespace {

constexpr int NT = 128;

struct RopeSide {
  const void* in;
  void* out;
  int64_t is[3], os[3];
  int heads;
};

template <class T>
__global__ void __launch_bounds__(NT) k_rope(const RopeView rope, const RopeSide q, const RopeSide k, int batch, int n, int per, int inverse) {
  depend_wait();
  const long long id = (long long)blockIdx.x * NT + threadIdx.x, tok = id >> 3;
  const int j = (int)id & 7, b = (int)(tok / n), i = (int)(tok % n);
  if (b >= batch) return;
  // pairs of chunks of eight channels: those that turn, then those that stay
  const int nc = rope.half >> 3;
  const bool turns = j < nc;
  const int c0 = turns ? 8 * j : 2 * rope.half + 16 * (j - nc), c1 = turns ? c0 + rope.half : c0 + 8;
  float cs[8], sn[8];
  if (turns) {
    turns8(rope, rope.positions + (size_t)b * n + i, (size_t)batch * n, c0, cs, sn);
    if (inverse) {
#pragma unroll
      for (int e = 0; e < 8; e++) sn[e] = -sn[e];
    }
  }
  const int h_end = min(q.heads + k.heads, ((int)blockIdx.y + 1) * per);
  // four heads at a time, all loads first: the stores may alias them for the compiler, and in place they do
  for (int h0 = (int)blockIdx.y * per; h0 < h_end; h0 += 4) {
    Vec8<T> u[4], v[4];
    T* to[4];
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int h = h0 + g;
      if (h >= h_end) continue;
      const bool is_q = h < q.heads;
      const RopeSide& x = is_q ? q : k;
      const int hh = is_q ? h : h - q.heads;
      const T* in = static_cast<const T*>(x.in) + b * x.is[0] + hh * x.is[1] + i * x.is[2];
      to[g] = static_cast<T*>(x.out) + b * x.os[0] + hh * x.os[1] + i * x.os[2];
      u[g] = *reinterpret_cast<const Vec8<T>*>(in + c0);
      v[g] = *reinterpret_cast<const Vec8<T>*>(in + c1);
    }
#pragma unroll
    for (int g = 0; g < 4; g++) {
      if (h0 + g >= h_end) continue;
      if (turns) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
          float a = to_f(u[g].v[e]), d = to_f(v[g].v[e]);
          rotate_pair(a, d, cs[e], sn[e]);
          u[g].v[e] = from_f<T>(a);
          v[g].v[e] = from_f<T>(d);
        }
      }
      *reinterpret_cast<Vec8<T>*>(to[g] + c0) = u[g];
      *reinterpret_cast<Vec8<T>*>(to[g] + c1) = v[g];
    }
  }
}

template <class T> okq_status launch_rope(const RopeView& r, const RopeSide& q, const RopeSide& k, int batch, int n, int inverse, cudaStream_t s) {
  const long long blocks = ((long long)batch * n * 8 + NT - 1) / NT;
  if (blocks > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  const int heads = q.heads + k.heads;
  // heads per thread: as many as leave the GPU's threads busy
  const long long want = 16ll * sm_count();
  int groups = (int)((want + blocks - 1) / blocks);
  groups = groups < heads ? groups : heads;
  const int per = (heads + groups - 1) / groups;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + per - 1) / per));
  const cudaError_t e = launch_dependent(k_rope<T>, grid, NT, 0, s, 1, r, q, k, batch, n, per, inverse);
  if (e != cudaSuccess) { set_last_cuda_error((int)e); (void)cudaGetLastError(); return OKQ_ERR_CUDA; }
  return launch_status();
}

}  // namespace

okq_status make_rope(const okq_rope* rope, RopeView& out) {
  out = RopeView{};
  if (!rope) return OKQ_OK;
  if (!rope->freq || !rope->positions) return OKQ_ERR_INVALID_ARG;
  long long half = 0;
  for (int i = 0; i < 3; i++) {
    if (rope->sections[i] < 0) return OKQ_ERR_INVALID_ARG;
    half += rope->sections[i];
  }
  if (half == 0 || (rope->interleaved != 0 && rope->interleaved != 1)) return OKQ_ERR_INVALID_ARG;
  if (half > 64 || half % 8 != 0) return OKQ_ERR_UNSUPPORTED;
  const int s0 = rope->sections[0], s1 = rope->sections[1], s2 = rope->sections[2];
  if (rope->interleaved && ((s1 > 0 && 3 * s1 - 2 >= half) || (s2 > 0 && 3 * s2 - 1 >= half))) return OKQ_ERR_INVALID_ARG;
  if (!aligned16(rope->freq) || !aligned16(rope->positions)) return OKQ_ERR_ALIGNMENT;
  out.freq = rope->freq;
  out.positions = rope->positions;
  out.half = (int)half;
  out.interleaved = rope->interleaved;
  out.s1 = rope->interleaved ? s1 : s0;
  out.s01 = s0 + s1;
  out.s2 = s2;
  return OKQ_OK;
}

}  // namespace okq

extern "C" okq_status okq_rope_apply(const okq_rope* rope, int32_t dtype, int32_t batch, int32_t n, const okq_rope_tensor* q,
                                     const okq_rope_tensor* k, int32_t inverse, void* stream) {
  using namespace okq;
  if (!rope || !q || batch < 0 || n < 0) return OKQ_ERR_INVALID_ARG;
  if (dtype != OKQ_FP16 && dtype != OKQ_BF16 && dtype != OKQ_FP32) return OKQ_ERR_UNSUPPORTED;
  if (inverse != 0 && inverse != 1) return OKQ_ERR_INVALID_ARG;
  RopeSide side[2] = {};
  for (int t = 0; t < 2; t++) {
    const okq_rope_tensor* x = t ? k : q;
    if (!x) continue;
    if (x->heads < 0 || (x->heads > 0 && (!x->in || !x->out))) return OKQ_ERR_INVALID_ARG;
    const int m = dtype == OKQ_FP32 ? 4 : 8;
    if (!aligned16(x->in) || !aligned16(x->out) || !strides_ok(x->in_strides, 3, m) || !strides_ok(x->out_strides, 3, m)) return OKQ_ERR_ALIGNMENT;
    side[t].in = x->in;
    side[t].out = x->out;
    side[t].heads = x->heads;
    for (int i = 0; i < 3; i++) { side[t].is[i] = x->in_strides[i]; side[t].os[i] = x->out_strides[i]; }
  }
  if ((long long)side[0].heads + side[1].heads > 65535) return OKQ_ERR_UNSUPPORTED;
  RopeView r;
  const okq_status st = make_rope(rope, r);
  if (st != OKQ_OK) return st;
  if (batch == 0 || n == 0 || side[0].heads + side[1].heads == 0) return OKQ_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == OKQ_FP16) return launch_rope<__half>(r, side[0], side[1], batch, n, inverse, s);
  if (dtype == OKQ_BF16) return launch_rope<__nv_bfloat16>(r, side[0], side[1], batch, n, inverse, s);
  return launch_rope<float>(r, side[0], side[1], batch, n, inverse, s);
}
