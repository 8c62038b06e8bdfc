// Root-mean-square norm of every head of queries and keys with the rotary positions in the same pass (okq_norm_rope_apply), and its
// gradients (okq_norm_rope_grad).  For a row x of 128 channels with weight w, R the rotation of its token:
//     r = (mean(x^2) + eps)^(-1/2),  y = R (w x r)
//     u = R^T g,  dw = sum over rows of u x r,  dx = r (w u - x r mean(x r w u))
// all in 32 bits, rounded once at the end.
//
// Both should be bound by memory: every element is read once (x, and g) and written once.  What has to be kept small is everything else: a
// number is worth 11 instructions forwards and 15 backwards (turns included), packed pairs of fp32 wherever two go alike.  Eight lanes
// have a row, sixteen channels each, which hold both channels of each pair they turn; its sums take three exchanges.  A token's cosines and sines
// are worked out once for all of its heads, and all blocks have equal parts of the line of tokens and heads; rows come by copies into
// shared memory two steps ahead, each thread its own.
// Times, ten calls in a graph (copy rate of 6.55 TB/s: floor): 32767 tokens x 36 heads in bf16 116 us (92); 8191 in fp32 56 (46); gradients
// of 12285 tokens x 36 heads in bf16 65 (52), of 8191 in fp32 85 (69), 5 of each the sums of the weights; 8 tokens 4.3.  Few heads: 65536 tokens x 8
// heads 50 to 54 (41), the gradients 78 to 82 (62): the copies begin anew with each side of a tile, its likely cause.  Measured and left, each beside the kernel of
// its time: rows by loads into registers, one step ahead 131 (the gradients of
// 12285 tokens), queries' and keys' rows on blocks of their own, each with its own cosines 96; copies five steps ahead 92, three 70;
// five blocks to an SM forwards (spills) 119; a thread's heads as grid rows, cosines three times per token 154.
#include "okq_device.cuh"
#include "okq_paged.cuh"
#include "okq_tc.cuh"

namespace okq {

namespace {

constexpr int NT = 128, TOKENS = NT / 8;
// Blocks that run at once on an SM, by registers (124 and 128) and shared memory.
constexpr int APPLY_PER_SM = 4;
template <class T> constexpr int GRAD_PER_SM = sizeof(T) == 4 ? 3 : 4;
constexpr int GRAD_BLOCKS = 1024;   // of the backward pass at most, and what the scratch is for

struct NormSide {
  const void *in, *up;
  void* out;
  int64_t is[3], us[3], os[3];
  const void* weight;
  float* weight_grad;
  int weight_dtype, heads;
};

// A thread's sixteen channels: in 16 bits eight from c0 and eight from c1, in 32 twice four and four, so that the eight lanes of a row read
// 128 consecutive bytes at a time.  Chunks that turn have both channels of each of their pairs.
template <class T> struct Place {
  static constexpr int PER = 16 / (int)sizeof(T), CHUNKS = 8 / PER;   // channels of 16 bytes
  int c0[CHUNKS], c1[CHUNKS];
  bool turns[CHUNKS];
  int axes;   // of the eight pairs, two bits each
  __device__ __forceinline__ Place(const RopeView& rope, int j) {
    const int half = rope.half ? rope.half : 64, nc = half / PER;   // (without a rotation laid out, and added up, as with one of all channels)
    axes = 0;
#pragma unroll
    for (int z = 0; z < CHUNKS; z++) {
      const int m = j + 8 * z;
      turns[z] = rope.half && m < nc;
      c0[z] = m < nc ? PER * m : 2 * half + 2 * PER * (m - nc);
      c1[z] = m < nc ? c0[z] + half : c0[z] + PER;
#pragma unroll
      for (int e = 0; e < PER; e++) axes |= rope.axis(c0[z] + e) << 2 * (PER * z + e);
    }
  }
  __device__ __forceinline__ bool turns_any() const {
    bool any = false;
#pragma unroll
    for (int z = 0; z < CHUNKS; z++) any |= turns[z];
    return any;
  }
};

// Sixteen numbers as pairs: those of the chunks' first channels in [0 .. 3], of the others in [4 .. 7].  Packed operations round like single ones.
__device__ __forceinline__ F2 pair_of(uint32_t w, __nv_bfloat16) { return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ F2 pair_of(uint32_t w, __half) {
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return f2(x.x, x.y);
}
__device__ __forceinline__ uint32_t word_of(F2 x, __nv_bfloat16) {
  const __nv_bfloat162 y = __float22bfloat162_rn(un2(x));
  return *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ uint32_t word_of(F2 x, __half) {
  const __half2 y = __float22half2_rn(un2(x));
  return *reinterpret_cast<const uint32_t*>(&y);
}

// a side's weights as fp32 in shared memory, by the first 128 threads that call it
__device__ __forceinline__ void stage_weights(const NormSide& x, float* w) {
  const int c = threadIdx.x;
  if (c >= D) return;
  w[c] = !x.weight                       ? 1.f
         : x.weight_dtype == OKQ_FP16 ? to_f(static_cast<const __half*>(x.weight)[c])
         : x.weight_dtype == OKQ_BF16 ? to_f(static_cast<const __nv_bfloat16*>(x.weight)[c])
                                      : static_cast<const float*>(x.weight)[c];
}
template <class T> __device__ __forceinline__ void load_weights(const float* from, const Place<T>& p, F2 (&w)[8]) {
#pragma unroll
  for (int z = 0; z < 4; z++) {
    const int c = Place<T>::CHUNKS == 1 ? (z < 2 ? p.c0[0] + 4 * z : p.c1[0] + 4 * (z - 2)) : z < 2 ? p.c0[z % Place<T>::CHUNKS] : p.c1[z % Place<T>::CHUNKS];
    const float4 x = *reinterpret_cast<const float4*>(from + c);
    w[2 * z] = f2(x.x, x.y);
    w[2 * z + 1] = f2(x.z, x.w);
  }
}

// cosines, sines and negative sines of the thread's eight pairs of channels
struct Turn {
  F2 c[4], s[4], n[4];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 4; e++) c[e] = s[e] = n[e] = f2(0.f, 0.f);
  }
  template <class T> __device__ __forceinline__ void of(const RopeView& rope, int b, int i, int batch, int n_tok, const Place<T>& p) {
    const int32_t* pos = rope.positions + (size_t)b * n_tok + i;
    const size_t axis = (size_t)batch * n_tok;
    const double p0 = (double)pos[0], p1 = (double)pos[axis], p2 = (double)pos[2 * axis];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      float cs[2], sn[2];
#pragma unroll
      for (int z = 0; z < 2; z++) {
        const int k = 2 * e + z, ax = p.axes >> 2 * k & 3;
        const int c0 = p.c0[k / Place<T>::PER] + k % Place<T>::PER;
        turn((ax == 0 ? p0 : ax == 1 ? p1 : p2) * (p.turns[k / Place<T>::PER] ? rope.freq[c0] : 0.0), cs[z], sn[z]);
      }
      c[e] = f2(cs[0], cs[1]);
      s[e] = f2(sn[0], sn[1]);
      n[e] = f2(-sn[0], -sn[1]);
    }
  }
};
// as rotate_pair, and with s and n exchanged its transpose
template <class T> __device__ __forceinline__ void rotate(F2 (&x)[8], const Place<T>& p, const F2 (&c)[4], const F2 (&s)[4], const F2 (&n)[4]) {
  constexpr int PAIRS = 4 / Place<T>::CHUNKS;
#pragma unroll
  for (int z = 0; z < Place<T>::CHUNKS; z++) {
    if (!p.turns[z]) continue;
#pragma unroll
    for (int e = PAIRS * z; e < PAIRS * (z + 1); e++) {
      const F2 a = x[e], b = x[4 + e];
      x[e] = fma2(a, c[e], mul2(b, n[e]));
      x[4 + e] = fma2(b, c[e], mul2(a, s[e]));
    }
  }
}

__device__ __forceinline__ float row_sum(float x) {   // over the eight lanes of a row; the same number in each
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}
__device__ __forceinline__ float dot(const F2 (&x)[8], const F2 (&y)[8]) {
  F2 s = mul2(x[0], y[0]);
#pragma unroll
  for (int e = 1; e < 8; e++) s = fma2(x[e], y[e], s);
  const float2 z = un2(s);
  return row_sum(z.x + z.y);
}

// A thread's rows on their way: DEPTH steps of `ROWS` rows' sixteen channels each, copied to shared memory ahead of their use.  Each thread
// copies what it reads itself, so that no barrier is needed; rows that are not there are zeros.
template <class T, int ROWS> struct Ring {
  static constexpr int PIECES = sizeof(T) == 4 ? 4 : 2, DEPTH = 3;   // (pieces of 16 bytes)
  static constexpr int BYTES = DEPTH * ROWS * PIECES * NT * 16;
  uint32_t at;   // the thread's first piece
  __device__ __forceinline__ explicit Ring(const void* smem) : at(smem_u32(smem) + 16 * threadIdx.x) {}
  __device__ __forceinline__ uint32_t place(int stage, int row, int piece) const { return at + (uint32_t)(((stage * ROWS + row) * PIECES + piece) * NT * 16); }
  // of the row at p
  __device__ __forceinline__ void fetch(int stage, int row, const T* p, const Place<T>& pl, bool there) const {
    const int bytes = there ? 16 : 0;
#pragma unroll
    for (int z = 0; z < PIECES; z++)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n"
                   ::"r"(place(stage, row, z)), "l"(p + (z < PIECES / 2 ? pl.c0[z % (PIECES / 2)] : pl.c1[z % (PIECES / 2)])), "r"(bytes) : "memory");
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
  static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(DEPTH - 2) : "memory"); }   // the oldest of DEPTH - 1
  __device__ __forceinline__ uint4 piece(int stage, int row, int z) const {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(place(stage, row, z)) : "memory");
    return v;
  }
  __device__ __forceinline__ void get(int stage, int row, F2 (&x)[8]) const {
    if constexpr (PIECES == 2) {
#pragma unroll
      for (int z = 0; z < 2; z++) {
        const uint4 v = piece(stage, row, z);
        x[4 * z] = pair_of(v.x, T()); x[4 * z + 1] = pair_of(v.y, T()); x[4 * z + 2] = pair_of(v.z, T()); x[4 * z + 3] = pair_of(v.w, T());
      }
    } else {
#pragma unroll
      for (int z = 0; z < 4; z++) {
        const uint4 v = piece(stage, row, z);
        x[2 * z] = f2(__uint_as_float(v.x), __uint_as_float(v.y));
        x[2 * z + 1] = f2(__uint_as_float(v.z), __uint_as_float(v.w));
      }
    }
  }
};
template <class T> __device__ __forceinline__ void store_row(const F2 (&x)[8], T* p, const Place<T>& pl) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(p + pl.c0[0]) = make_uint4(word_of(x[0], T()), word_of(x[1], T()), word_of(x[2], T()), word_of(x[3], T()));
    *reinterpret_cast<uint4*>(p + pl.c1[0]) = make_uint4(word_of(x[4], T()), word_of(x[5], T()), word_of(x[6], T()), word_of(x[7], T()));
  } else {
#pragma unroll
    for (int z = 0; z < 4; z++) {
      const float2 y = un2(x[2 * z]), w = un2(x[2 * z + 1]);
      *reinterpret_cast<float4*>(p + (z < 2 ? pl.c0[z % 2] : pl.c1[z % 2])) = make_float4(y.x, y.y, w.x, w.y);
    }
  }
}

constexpr float SMALL = 1.2621774483536189e-29f;   // 2^-96

// x becomes x r; returns r, times 2^96 where the row was multiplied by 2^-96 because its squares have no sum in fp32 (fp16 rows never are)
__device__ __forceinline__ float normalise(F2 (&x)[8], float eps, bool& scaled) {
  float s = dot(x, x);
  scaled = s > 1e37f;
  if (__any_sync(0xffffffffu, scaled)) {
    const float f = scaled ? SMALL : 1.f;
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = mul2(x[e], f2(f, f));
    const float z = dot(x, x);
    if (scaled) s = z;
  }
  float r;   // (of a normal number: eps is one, and where it is made smaller the rest is not below 2^-77; two units in the last place)
  asm("rsqrt.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(fmaf(s, 1.f / D, scaled ? eps * SMALL * SMALL : eps)));
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = mul2(x[e], f2(r, r));
  return r;
}

// token of the thread's rows
struct Token {
  int b, i;
  bool there;
  __device__ __forceinline__ Token(long long tile, int batch, int n) {
    const long long tok = tile * TOKENS + (threadIdx.x >> 3);
    b = (int)(tok / n);
    i = (int)(tok - (long long)b * n);
    there = b < batch;
  }
};

// heads [h, end) of one side for the thread's token, two at a time
template <class T, class R>
__device__ __forceinline__ void norm_heads(const R& ring, const NormSide& x, const float* weights, const Place<T>& pl, const Token& tok, const RopeView& rope, Turn& turn,
                                           bool& turned, int batch, int n, float eps, int h, int end) {
  const int64_t is1 = x.is[1], os1 = x.os[1];
  const T* in = static_cast<const T*>(x.in);
  T* out = static_cast<T*>(x.out);
  if (tok.there) {
    in += (int64_t)tok.b * x.is[0] + (int64_t)tok.i * x.is[2] + h * is1;
    out += (int64_t)tok.b * x.os[0] + (int64_t)tok.i * x.os[2] + h * os1;
  }
  int ahead = h, put = 0, got = 0;   // first head that has not been asked for; stages
  auto fetch = [&] {
    if (ahead < end) {
      ring.fetch(put, 0, in, pl, tok.there);
      ring.fetch(put, 1, ahead + 1 < end ? in + is1 : in, pl, tok.there && ahead + 1 < end);
      in += 2 * is1;
      ahead += 2;
    }
    put = put + 1 == R::DEPTH ? 0 : put + 1;
    R::commit();
  };
#pragma unroll
  for (int i = 0; i < R::DEPTH - 1; i++) fetch();
  if (!turned) turn.of(rope, tok.b, tok.i, batch, n, pl);   // (while the first rows are on their way)
  turned = true;
#pragma unroll 1
  for (; h < end; h += 2) {
    R::wait();
    F2 y[2][8], w[8];
    ring.get(got, 0, y[0]);
    ring.get(got, 1, y[1]);
    got = got + 1 == R::DEPTH ? 0 : got + 1;
    fetch();
#pragma unroll
    for (int g = 0; g < 2; g++) {
      bool scaled;
      normalise(y[g], eps, scaled);
    }
    load_weights(weights, pl, w);
#pragma unroll
    for (int g = 0; g < 2; g++) {
#pragma unroll
      for (int e = 0; e < 8; e++) y[g][e] = mul2(y[g][e], w[e]);
      rotate(y[g], pl, turn.c, turn.s, turn.n);
    }
    if (tok.there) {
      store_row<T>(y[0], out, pl);
      if (h + 1 < end) store_row<T>(y[1], out + os1, pl);
    }
    out += 2 * os1;
  }
}

// All blocks have equal parts of one line of steps: tile after tile of 16 tokens, and in a tile the heads two by two, queries' before keys'.
// So a tile's cosines and sines are worked out about once.
template <class T>
__global__ void __launch_bounds__(NT, APPLY_PER_SM) k_norm_rope(const RopeView rope, const NormSide q, const NormSide k, float eps, int batch, int n, long long tiles) {
  extern __shared__ uint4 rows[];
  __shared__ __align__(16) float weights[2][D];
  const Ring<T, 2> ring(rows);
  depend_wait();
  stage_weights(q, weights[0]);
  stage_weights(k, weights[1]);
  __syncthreads();
  const Place<T> pl(rope, threadIdx.x & 7);
  const int q_steps = (q.heads + 1) >> 1, steps = q_steps + ((k.heads + 1) >> 1);
  const long long first = tiles * steps * blockIdx.x / gridDim.x, last = tiles * steps * (blockIdx.x + 1) / gridDim.x;
  long long tile = first / steps;
  int j = (int)(first - tile * steps);
#pragma unroll 1
  for (long long left = last - first; left > 0; tile++, j = 0) {
    const int end = (int)min((long long)steps, j + left);
    left -= end - j;
    const Token tok(tile, batch, n);
    Turn turn;
    turn.clear();
    bool turned = !(pl.turns_any() && tok.there);
    if (j < q_steps) norm_heads<T>(ring, q, weights[0], pl, tok, rope, turn, turned, batch, n, eps, 2 * j, min(q.heads, 2 * end));
    if (end > q_steps) norm_heads<T>(ring, k, weights[1], pl, tok, rope, turn, turned, batch, n, eps, 2 * max(0, j - q_steps), min(k.heads, 2 * (end - q_steps)));
  }
}

// The same line, a head to a step.  partial[side][block][128]: what the block's rows add to the side's weight's gradient; a thread's sums
// are kept in registers over the heads of a side and a token, and in shared memory from there on.
template <class T>
__global__ void __launch_bounds__(NT, GRAD_PER_SM<T>) k_norm_rope_grad(const RopeView rope, const NormSide q, const NormSide k, float eps, int batch, int n, long long tiles,
                                                                    float* partial) {
  using Rows = Ring<T, 2>;   // x and the gradient
  extern __shared__ uint4 rows[];
  __shared__ __align__(16) float weights[2][D];
  __shared__ float2 sums[2][8][NT];
  const Rows ring(rows);
  depend_wait();
  stage_weights(q, weights[0]);
  stage_weights(k, weights[1]);
#pragma unroll
  for (int e = 0; e < 16; e++) sums[e >> 3][e & 7][threadIdx.x] = make_float2(0.f, 0.f);
  __syncthreads();
  const Place<T> pl(rope, threadIdx.x & 7);
  const int steps = q.heads + k.heads;
  const long long first = tiles * steps * blockIdx.x / gridDim.x, last = tiles * steps * (blockIdx.x + 1) / gridDim.x;
  long long tile = first / steps;
  int j = (int)(first - tile * steps);
#pragma unroll 1
  for (long long left = last - first; left > 0; tile++, j = 0) {
    const int j_end = (int)min((long long)steps, j + left);
    left -= j_end - j;
    const Token tok(tile, batch, n);
    Turn turn;
    turn.clear();   // (rows behind the last token add nothing to the weights' sums)
    bool turned = !(pl.turns_any() && tok.there);
#pragma unroll 1
    for (int side = 0; side < 2; side++) {
      const NormSide& x = side ? k : q;
      int h = max(0, j - (side ? q.heads : 0));
      const int end = min(x.heads, j_end - (side ? q.heads : 0));
      if (h >= end) continue;
      const int64_t is1 = x.is[1], us1 = x.us[1], os1 = x.os[1];
      const T *in = static_cast<const T*>(x.in), *from = static_cast<const T*>(x.up);
      T* out = static_cast<T*>(x.out);
      if (tok.there) {
        in += (int64_t)tok.b * x.is[0] + (int64_t)tok.i * x.is[2] + h * is1;
        from += (int64_t)tok.b * x.us[0] + (int64_t)tok.i * x.us[2] + h * us1;
        out += (int64_t)tok.b * x.os[0] + (int64_t)tok.i * x.os[2] + h * os1;
      }
      int ahead = h, put = 0, got = 0;
      auto fetch = [&] {
        if (ahead < end) {
          ring.fetch(put, 0, in, pl, tok.there);
          ring.fetch(put, 1, from, pl, tok.there);
          in += is1;
          from += us1;
          ahead++;
        }
        put = put + 1 == Rows::DEPTH ? 0 : put + 1;
        Rows::commit();
      };
#pragma unroll
      for (int i = 0; i < Rows::DEPTH - 1; i++) fetch();
      if (!turned) turn.of(rope, tok.b, tok.i, batch, n, pl);
      turned = true;
      F2 dw[8];
#pragma unroll
      for (int e = 0; e < 8; e++) dw[e] = f2(0.f, 0.f);
#pragma unroll 1
      for (; h < end; h++) {
        F2 y[8], u[8], w[8];
        bool scaled;
        Rows::wait();
        ring.get(got, 0, y);
        ring.get(got, 1, u);
        got = got + 1 == Rows::DEPTH ? 0 : got + 1;
        fetch();
        const float r = normalise(y, eps, scaled);
        rotate(u, pl, turn.c, turn.n, turn.s);
        load_weights(weights[side], pl, w);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          dw[e] = fma2(u[e], y[e], dw[e]);
          u[e] = mul2(u[e], w[e]);
        }
        const float mean = dot(u, y) * (-1.f / D);
#pragma unroll
        for (int e = 0; e < 8; e++) u[e] = mul2(fma2(y[e], f2(mean, mean), u[e]), f2(r, r));
        if (scaled) {
#pragma unroll
          for (int e = 0; e < 8; e++) u[e] = mul2(u[e], f2(SMALL, SMALL));
        }
        if (tok.there) store_row<T>(u, out, pl);
        out += os1;
      }
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float2 a = sums[side][e][threadIdx.x], z = un2(dw[e]);
        sums[side][e][threadIdx.x] = make_float2(a.x + z.x, a.y + z.y);
      }
    }
  }
  if (!partial) return;
  __syncthreads();
  // channel c = threadIdx.x: the lane of a row that has it, its place among the lane's sixteen, then the block's sixteen rows
  for (int side = 0; side < 2; side++) {
    const int lane = threadIdx.x >> 4, e = threadIdx.x & 15;
    const Place<T> mine(rope, lane);
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < TOKENS; r++) {
      const float2 z = sums[side][e >> 1][8 * r + lane];
      s += e & 1 ? z.y : z.x;
    }
    int c = 0;
#pragma unroll
    for (int z = 0; z < Place<T>::CHUNKS; z++)
      if ((e & 7) / Place<T>::PER == z) c = (e < 8 ? mine.c0[z] : mine.c1[z]) + (e & 7) % Place<T>::PER;
    partial[((size_t)side * gridDim.x + blockIdx.x) * D + c] = s;
  }
}

// Block (x, side): sums of eight channels over the side's rows, 32 threads to each, row by row and then in a tree: always the same order.
__global__ void __launch_bounds__(256) k_norm_weight_grad(const float* partial, int blocks, float* q_grad, float* k_grad) {
  __shared__ float sums[32][9];
  depend_wait();
  const int side = blockIdx.y, c = threadIdx.x & 7, r = threadIdx.x >> 3;
  float* to = side ? k_grad : q_grad;
  if (!to) return;
  const int first = side * blocks, last = first + blocks;
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

// dynamic shared memory beyond the default, once per thread and device
template <class K> cudaError_t allow_smem(K kernel, int bytes, unsigned long long& mask) {
  int dev = 0;
  if (!attr_needed(mask, dev)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) attr_done(mask, dev);
  return e;
}

template <class T> cudaError_t launch_apply(const RopeView& r, const NormSide (&x)[2], float eps, int batch, int n, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  const cudaError_t e = allow_smem(k_norm_rope<T>, Ring<T, 2>::BYTES, attr_mask);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)batch * n + TOKENS - 1) / TOKENS, steps = tiles * ((x[0].heads + 1) / 2 + (x[1].heads + 1) / 2);
  const long long most = (long long)APPLY_PER_SM * sm_count();
  return launch_dependent(k_norm_rope<T>, dim3((unsigned)(steps < most ? steps : most)), NT, Ring<T, 2>::BYTES, s, 1, r, x[0], x[1], eps, batch, n, tiles);
}

template <class T> cudaError_t launch_grad(const RopeView& r, const NormSide (&x)[2], float eps, int batch, int n, float* partial, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  cudaError_t e = allow_smem(k_norm_rope_grad<T>, Ring<T, 2>::BYTES, attr_mask);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)batch * n + TOKENS - 1) / TOKENS, steps = tiles * (x[0].heads + x[1].heads);
  const int most = GRAD_PER_SM<T> * sm_count() < GRAD_BLOCKS ? GRAD_PER_SM<T> * sm_count() : GRAD_BLOCKS, blocks = (int)(steps < most ? steps : most);
  const bool sums = x[0].weight_grad || x[1].weight_grad;
  e = launch_dependent(k_norm_rope_grad<T>, dim3((unsigned)blocks), NT, Ring<T, 2>::BYTES, s, 1, r, x[0], x[1], eps, batch, n, tiles, sums ? partial : nullptr);
  if (e != cudaSuccess || !sums) return e;
  return launch_dependent(k_norm_weight_grad, dim3(D / 8, 2), 256, 0, s, 1, partial, blocks, x[0].weight_grad, x[1].weight_grad);
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
  // a row for each block and side, whatever the sizes: scratch for one call serves every other
  return (size_t)2 * okq::GRAD_BLOCKS * okq::D * sizeof(float);
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
  if (((long long)batch * n + TOKENS - 1) / TOKENS > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  if (batch == 0 || n == 0 || x[0].heads + x[1].heads == 0) {   // no rows: sums of nothing
    const cudaError_t e = sums ? launch_dependent(k_norm_weight_grad, dim3(D / 8, 2), 256, 0, s, 1, nullptr, 0, x[0].weight_grad, x[1].weight_grad) : cudaSuccess;
    return e != cudaSuccess ? failed(e) : OKQ_OK;
  }
  if (sums && (!workspace || workspace_bytes < okq_norm_rope_workspace_bytes(batch, n, x[0].heads, x[1].heads))) return OKQ_ERR_WORKSPACE;
  float* partial = static_cast<float*>(workspace);
  const cudaError_t e = dtype == OKQ_FP16   ? launch_grad<__half>(r, x, eps, batch, n, partial, s)
                        : dtype == OKQ_BF16 ? launch_grad<__nv_bfloat16>(r, x, eps, batch, n, partial, s)
                                            : launch_grad<float>(r, x, eps, batch, n, partial, s);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // extern "C"
