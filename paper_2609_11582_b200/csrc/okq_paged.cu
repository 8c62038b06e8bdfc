// The 8-bit paged cache: argument checks, append (quantising whole blocks of 32 tokens and one head), read-back.
//
// Append.  A block of keys or values is 32 x 128 numbers with one scale, so its codes are known when all of its tokens are: 128 threads
// read the tokens that are there (those of an unfinished block from the raw copies, the new ones from the caller's tensor), take the
// maximum and write codes, scale and, for the block that stays unfinished, the raw copies.  A thread block has one side, keys or values,
// of up to four consecutive blocks of a head; with up to 32 new tokens, the sides of a sequence's heads are dealt over a cluster.
// Requantising the unfinished block with every append costs at most 16 KB of reads per head and makes the cache
// independent of how its tokens were dealt over calls; keeping the codes and only lowering their scale would round twice.
#include "okq_device.cuh"
#include "okq_paged.cuh"

namespace okq {

namespace {

constexpr int NT = 256;    // threads of a block, but for the append kernels
constexpr int AT = 128;

// rows of one call's keys or values
struct Rows {
  const void* p;
  int64_t s[4];
  template <class T> __device__ const T* at(int l, int b, int h, int i) const {
    return static_cast<const T*>(p) + l * s[0] + b * s[1] + h * s[2] + i * s[3];
  }
};

// whether the sequence can take `m` tokens behind `len`: room in its row and a page for each (all threads of the block call it)
__device__ __forceinline__ int pages_missing(const PagedView& c, int b, int len, int m, int tid, int nt) {
  if (m == 0) return 0;
  if (m > c.room() - len) return 1;
  int bad = 0;
  const int j0 = len >> c.page_shift, j1 = (len + m - 1) >> c.page_shift;
  for (int j = j0 + tid; j <= j1; j += nt) bad |= c.page_of(b, j << c.page_shift) < 0;
  return bad;
}

// rint(x / scale) of numbers no larger than 127.5 scale, the quotient rounded to fp32.  With the reciprocal r of the scale correctly
// rounded, one residual step from x r gives the correctly rounded quotient (Markstein's theorem; the residual is exact), three
// multiply-adds for a division; scales so small that the residual would be cut off are divided by.  1.5 * 2^23 + q rounds q to an
// integer, whose low byte is the code.
struct Quotient {
  float scale, r;
  int how;   // 0: codes 0 (a scale of zero or NaN), 1: residual step, 2: division
  template <class T> __device__ __forceinline__ void codes(const Vec8<T>& x, uint32_t (&q)[8]) const {
    if (how == 1) {
      const F2 r2 = f2(r, r), s2 = f2(-scale, -scale), one = f2(12582912.f, 12582912.f);
#pragma unroll
      for (int e = 0; e < 4; e++) {   // (packed pairs round like single operations)
        const F2 v = f2(to_f(x.v[2 * e]), to_f(x.v[2 * e + 1])), a = mul2(v, r2);
        const float2 y = un2(add2(fma2(fma2(a, s2, v), r2, a), one));
        q[2 * e] = __float_as_uint(y.x);
        q[2 * e + 1] = __float_as_uint(y.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++)   // (a subnormal scale may be too small by half of itself)
        q[e] = how == 0 ? 0u : __float_as_uint(__fadd_rn(fminf(fmaxf(__fdiv_rn(to_f(x.v[e]), scale), -127.f), 127.f), 12582912.f));
    }
  }
};

__device__ __forceinline__ Quotient quotient_by(float scale) {
  return Quotient{scale, __fdiv_rn(1.f, scale), !(scale > 0.f) ? 0 : scale >= 7.9e-31f ? 1 : 2};
}

// One block's keys, or values, by AT threads: thread tid has row tid / 4 and four chunks of eight channels, two of them apart by the
// pairs of a rotation, as okq_rope_apply deals them.
struct Chunks {
  int t, j, c[4];
  bool turns[2];
  __device__ __forceinline__ Chunks(int tid, const RopeView& rope, bool keys) : t(tid >> 2), j(tid & 3) {
    const int nc = rope.half >> 3;
    const bool deal = rope.freq && keys;
#pragma unroll
    for (int z = 0; z < 2; z++) {
      const int k = j + 4 * z;
      turns[z] = deal && k < nc;
      c[2 * z] = !deal || k < nc ? 8 * k : 2 * rope.half + 16 * (k - nc);
      c[2 * z + 1] = !deal ? 8 * k + 64 : k < nc ? 8 * k + rope.half : c[2 * z] + 8;
    }
  }
};
template <class T> struct BlockRows { Vec8<T> x[4]; };
// largest magnitude of two numbers each, NaN where there is one
__device__ __forceinline__ __half2 top2(__half2 a, __half2 b) { return __hmax2_nan(a, __habs2(b)); }
__device__ __forceinline__ __nv_bfloat162 top2(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2_nan(a, __habs2(b)); }
template <class T> struct Pair;
template <> struct Pair<__half> { using type = __half2; };
template <> struct Pair<__nv_bfloat16> { using type = __nv_bfloat162; };
using Turns = float2[PB][72];   // cosines and sines of a block's new rows: pair 8 j + e in place 8 e + j, rows apart in the banks
struct BlockSmem {
  unsigned top[2][AT / 32];     // (two blocks in turn)
  Turns turns;
};
// What a thread block knows of the sequence that it appends `m` tokens to, and its side of the head.
struct Append {
  int l, li, b, h, side, len, m, n_new;
  __device__ __forceinline__ int first(int blk) const { return len - len % PB + blk * PB; }
  __device__ __forceinline__ int rows(int blk) const { return min(PB, len + m - first(blk)); }
};
// block blk of the new tokens: rows, raw ones first
template <class T>
__device__ __forceinline__ void load_rows(const PagedView& c, const Append& w, int blk, const Rows& src, const Chunks& at, BlockRows<T>& y) {
  const int i = w.first(blk) + at.t - w.len;   // among the new tokens, negative for raw ones
  if (at.t < w.rows(blk)) {
    const T* p = i < 0 ? c.raw_of<T>(w.l, w.b, w.h, w.side) + (size_t)at.t * D : src.at<T>(w.li, w.b, w.h, i);
#pragma unroll
    for (int z = 0; z < 4; z++) y.x[z] = *reinterpret_cast<const Vec8<T>*>(p + at.c[z]);
  } else {
#pragma unroll
    for (int e = 0; e < 32; e++) y.x[e >> 3].v[e & 7] = from_f<T>(0.f);
  }
}
// the turns of its new rows (one at a time, a pair to a thread: code that runs once is paid for by its length)
__device__ __forceinline__ void make_turns(const PagedView& c, const Append& w, int blk, const RopeView& rope, BlockSmem& sm) {
  const int first = w.first(blk), first_new = max(0, w.len - first), n = w.rows(blk) - first_new, pair = threadIdx.x & 63;
  const double f = pair < rope.half ? rope.freq[pair] : 0.0;
  const int32_t* pos = rope.positions + rope.axis(pair) * ((size_t)c.batch * w.n_new) + (size_t)w.b * w.n_new + (first + first_new - w.len);
#pragma unroll 1
  for (int e = threadIdx.x >> 6; e < n; e += AT / 64) {
    float2& z = sm.turns[first_new + e][8 * (pair & 7) + (pair >> 3)];
    turn((double)pos[e] * f, z.x, z.y);
  }
}
// rotates them; the warp's largest magnitude goes to top[which] (as an integer: the order is the numbers' own, infinities and NaN at the top)
template <class T>
__device__ __forceinline__ void turn_rows(const Append& w, int blk, const Chunks& at, BlockRows<T>& y, BlockSmem& sm, int which) {
  if (at.t < w.rows(blk) && w.first(blk) + at.t >= w.len) {
#pragma unroll
    for (int z = 0; z < 2; z++) {
      if (!at.turns[z]) continue;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float2 cs = sm.turns[at.t][8 * e + at.j + 4 * z];
        float u = to_f(y.x[2 * z].v[e]), v = to_f(y.x[2 * z + 1].v[e]);
        rotate_pair(u, v, cs.x, cs.y);
        y.x[2 * z].v[e] = from_f<T>(u);
        y.x[2 * z + 1].v[e] = from_f<T>(v);
      }
    }
  }
  using P = typename Pair<T>::type;
  const P* v = reinterpret_cast<const P*>(&y);
  P mx = __habs2(v[0]);
#pragma unroll
  for (int e = 1; e < 16; e++) mx = top2(mx, v[e]);
  const unsigned both = max(__float_as_uint(to_f(mx.x)) & 0x7fffffffu, __float_as_uint(to_f(mx.y)) & 0x7fffffffu);
  const unsigned all = __reduce_max_sync(0xffffffffu, both);
  if ((threadIdx.x & 31) == 0) sm.top[which][threadIdx.x >> 5] = all;
}
template <class T>
__device__ __forceinline__ void store_codes(const PagedView& c, const Append& w, int blk, int page, const Chunks& at, const BlockRows<T>& y, const BlockSmem& sm, int which) {
  const int first = w.first(blk), rows = w.rows(blk);
  unsigned mx = 0;
#pragma unroll
  for (int e = 0; e < AT / 32; e++) mx = max(mx, sm.top[which][e]);
  float scale = __fdiv_rn(__uint_as_float(mx), 127.f);
  if (mx >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);   // infinities, NaN
  const Quotient by = quotient_by(scale);
  const size_t row = c.code_row(w.l, page, w.h, w.side) + (first & (c.page - 1));
  if (at.t < rows) {
    int8_t* dst = c.codes + (row + at.t) * D;
#pragma unroll
    for (int z = 0; z < 4; z++) {
      uint32_t q[8];
      by.codes(y.x[z], q);
      uint2 u;
      u.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
      u.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(dst + at.c[z]) = u;
    }
    if (rows < PB && first + at.t >= w.len) {   // a block that stays unfinished
      T* keep = c.raw_of<T>(w.l, w.b, w.h, w.side) + (size_t)at.t * D;
#pragma unroll
      for (int z = 0; z < 4; z++) *reinterpret_cast<Vec8<T>*>(keep + at.c[z]) = y.x[z];
    }
  }
  if (threadIdx.x == 0) c.scales[row / PB] = scale;
}

// A thread block has one side of `per` consecutive 32-token blocks and loads each while it quantises the one before.  Bound by memory
// and the quotients' issue: 28 layers x 4097 tokens x 4 heads 78 us, 4.5 TB/s (keys and values in one block of 256 threads, two blocks
// on an SM, 199; apart and one by one 121; rows of 128 threads with the next block's loads ahead 78).
template <class T>
__global__ void __launch_bounds__(AT, 8) k_paged_append(const PagedView c, int layer, const Rows k, const Rows v, int n_new, const int32_t* new_len,
                                                     const RopeView rope, int n_ranges, int per) {
  __shared__ BlockSmem sm;
  depend_wait();
  const int tid = threadIdx.x;
  unsigned u = blockIdx.x;
  Append w;
  const int blk0 = (int)(u % (unsigned)n_ranges) * per;
  u /= (unsigned)n_ranges;
  w.side = (int)(u & 1);
  u >>= 1;
  w.h = (int)(u % (unsigned)c.n_kv);
  u /= (unsigned)c.n_kv;
  w.li = (int)(u / (unsigned)c.batch);
  w.b = (int)(u - (unsigned)w.li * c.batch);
  w.l = layer + w.li;
  w.n_new = n_new;
  w.m = count_of(new_len, w.b, n_new);
  w.len = c.held(w.l, w.b);
  const int r = w.len % PB, blocks = (r + w.m + PB - 1) / PB;
  if (w.m == 0 || blk0 >= blocks) return;
  // The raw tokens are read by the first block and replaced by the last, so one thread block does both, in that order.
  const int last = blocks - 1;
  const bool follows = r > 0 && last >= per && (r + w.m) % PB != 0;
  int n = min(per, blocks - blk0);
  if (follows && blk0 == 0) n = per + 1;
  if (follows && blk0 > 0 && blk0 + n > last && --n == 0) return;
  auto block = [&](int e) { return follows && blk0 == 0 && e == per ? last : blk0 + e; };
  const Rows& src = w.side ? v : k;
  const Chunks at(tid, rope, w.side == 0);
  const bool turns = rope.freq && w.side == 0;
  BlockRows<T> y, z;
  load_rows<T>(c, w, blk0, src, at, y);
  if (turns) make_turns(c, w, blk0, rope, sm);
  if (__syncthreads_or(pages_missing(c, w.b, w.len, w.m, tid, AT))) return;   // (while the rows are on their way)
  for (int e = 0; e < n; e++) {
    const int blk = block(e), page = c.page_of(w.b, w.first(blk));
    turn_rows<T>(w, blk, at, y, sm, e & 1);
    __syncthreads();
    if (e + 1 < n) {
      load_rows<T>(c, w, block(e + 1), src, at, z);
      if (turns) make_turns(c, w, block(e + 1), rope, sm);
    }
    store_codes<T>(c, w, blk, page, at, y, sm, e & 1);
    if (turns) __syncthreads();
    y = z;
  }
}

// The same for up to FEW new tokens (two blocks of a sequence at most) in one launch: a cluster has a (layer, sequence), each of its
// blocks every size-th side of a head, and the length is advanced when all of them have read it.
constexpr int FEW = PB, MOST = 8;
template <class T>
__global__ void __launch_bounds__(AT) k_paged_append_few(const PagedView c, int layer, const Rows k, const Rows v, int n_new, const int32_t* new_len,
                                                         const RopeView rope, int size) {
  __shared__ BlockSmem sm;
  depend_wait();
  const int tid = threadIdx.x, rank = blockIdx.x % size, u = blockIdx.x / size;
  Append w;
  w.li = u / c.batch;
  w.b = u - w.li * c.batch;
  w.l = layer + w.li;
  w.n_new = n_new;
  w.m = count_of(new_len, w.b, n_new);
  w.len = c.held(w.l, w.b);
  const int r = w.len % PB;
  if (w.m == 0) return;                       // (the whole cluster)
  const int last = (r + w.m - 1) / PB;        // 0 or 1
  int which = 0, bad = 0;
  for (int e = rank; e < 2 * c.n_kv && !bad; e += size) {
    w.h = e >> 1;
    w.side = e & 1;
    const Chunks at(tid, rope, w.side == 0);
    for (int blk = 0; blk <= last; blk++, which ^= 1) {
      BlockRows<T> y;
      load_rows<T>(c, w, blk, w.side ? v : k, at, y);
      if (rope.freq && w.side == 0) {
        make_turns(c, w, blk, rope, sm);
        __syncthreads();
      }
      // (the first rows are on their way while the table is looked at)
      if (e == rank && blk == 0 && (bad = __syncthreads_or(pages_missing(c, w.b, w.len, w.m, tid, AT)))) break;
      const int page = c.page_of(w.b, w.first(blk));
      turn_rows<T>(w, blk, at, y, sm, which);
      __syncthreads();                        // (behind the loads: raw tokens are read before they are replaced)
      store_codes<T>(c, w, blk, page, at, y, sm, which);
    }
  }
  if (size > 1) {
    asm volatile("barrier.cluster.arrive.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;\n" ::: "memory");
  } else {
    __syncthreads();
  }
  if (tid != 0 || rank != 0) return;
  if (bad) set_status(c.status, OKQ_ERR_CAPACITY);
  else c.seq_len[(size_t)w.l * c.batch + w.b] = w.len + w.m;
}

// lengths after an append, and the status of sequences that could not take theirs; one warp per (layer, sequence)
__global__ void __launch_bounds__(NT) k_paged_advance(const PagedView c, int layer, int layer_count, int n_new, const int32_t* new_len) {
  depend_wait();
  const int u = blockIdx.x * (NT / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (u >= layer_count * c.batch) return;
  const int b = u % c.batch, l = layer + u / c.batch;
  const int m = count_of(new_len, b, n_new), len = c.held(l, b);
  const int bad = __any_sync(0xffffffffu, pages_missing(c, b, len, m, lane, 32));
  if (lane) return;
  if (bad) set_status(c.status, OKQ_ERR_CAPACITY);
  else if (m) c.seq_len[(size_t)l * c.batch + b] = len + m;
}

// Block: NT / 8 tokens of a (layer, sequence, head), eight threads to a token; 8-byte loads of codes so that a warp's stores are whole
// lines.  Bound by memory: 28 layers x 4097 tokens x 4 heads 55 us, 6.4 TB/s.
template <class T>
__global__ void __launch_bounds__(NT) k_paged_read(const PagedView c, int layer, int begin, int n, T* k_out, T* v_out, int chunks) {
  depend_wait();
  const unsigned unit = blockIdx.x / (unsigned)chunks;
  const unsigned pair = unit / (unsigned)c.n_kv, h = unit - pair * c.n_kv, li = pair / (unsigned)c.batch, b = pair - li * c.batch;
  const int i = (int)(blockIdx.x - unit * chunks) * (NT / 8) + (threadIdx.x >> 3), j = threadIdx.x & 7, l = layer + (int)li, t = begin + i;
  if (i >= n || t >= c.held(l, b)) return;
  const int page = c.page_of(b, t);
  if (page < 0) { set_status(c.status, OKQ_ERR_INVALID_ARG); return; }
  uint2 w[2][2];
  float scale[2];
#pragma unroll
  for (int side = 0; side < 2; side++) {
    const size_t row = c.code_row(l, page, h, side) + (t & (c.page - 1));
    scale[side] = c.scales[row / PB];
#pragma unroll
    for (int z = 0; z < 2; z++) w[side][z] = *reinterpret_cast<const uint2*>(c.codes + row * D + 64 * z + 8 * j);
  }
#pragma unroll
  for (int side = 0; side < 2; side++) {
    T* out = (side ? v_out : k_out) + ((size_t)unit * n + i) * D + 8 * j;
#pragma unroll
    for (int z = 0; z < 2; z++) {
      // 0x4b000000 | (code + 128) is 2^23 + 128 + code (the conversions' unit is busy two thirds of the time with them, 56 us and not 55)
      const uint32_t u[2] = {w[side][z].x ^ 0x80808080u, w[side][z].y ^ 0x80808080u};
      Vec8<T> y;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const F2 q = add2(f2(__uint_as_float(__byte_perm(u[e >> 2], 0x4b000000u, 0x7440 + (e & 3))), __uint_as_float(__byte_perm(u[e >> 2], 0x4b000000u, 0x7440 + (e & 3) + 1))),
                          f2(-8388736.f, -8388736.f));
        const float2 x = un2(mul2(q, f2(scale[side], scale[side])));
        y.v[e] = from_f<T>(x.x);
        y.v[e + 1] = from_f<T>(x.y);
      }
      *reinterpret_cast<Vec8<T>*>(out + 64 * z) = y;
    }
  }
}

okq_status failed(cudaError_t e) {
  set_last_cuda_error((int)e);
  (void)cudaGetLastError();
  return OKQ_ERR_CUDA;
}

template <class T>
okq_status launch_append(const PagedView& c, int layer, int layer_count, const Rows& k, const Rows& v, int n_new, const int32_t* new_len,
                         const RopeView& rope, cudaStream_t s) {
  if (n_new <= FEW) {
    const int size = 2 * c.n_kv < MOST ? 2 * c.n_kv : MOST;
    const cudaError_t e = launch_dependent(k_paged_append_few<T>, dim3((unsigned)(layer_count * c.batch * size)), AT, 0, s, size, c, layer, k, v, n_new, new_len, rope, size);
    return e != cudaSuccess ? failed(e) : launch_status();
  }
  // blocks in a row: as many as leave each SM sixteen thread blocks or more, four at most
  const int n_blocks = (PB - 1 + n_new + PB - 1) / PB;
  const long long units = 2ll * layer_count * c.batch * c.n_kv, want = units * n_blocks / (16ll * sm_count());
  const int per = want < 1 ? 1 : want > 4 ? 4 : (int)want, n_ranges = (n_blocks + per - 1) / per;
  if (units * n_ranges > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  cudaError_t e = launch_dependent(k_paged_append<T>, dim3((unsigned)(units * n_ranges)), AT, 0, s, 1, c, layer, k, v, n_new, new_len, rope, n_ranges, per);
  if (e != cudaSuccess) return failed(e);
  const int warps = NT / 32;
  e = launch_dependent(k_paged_advance, dim3((layer_count * c.batch + warps - 1) / warps), NT, 0, s, 1, c, layer, layer_count, n_new, new_len);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // namespace

okq_status check_paged(const okq_paged* c, bool need_ptrs) {
  if (!c) return OKQ_ERR_INVALID_ARG;
  if (c->n_layers <= 0 || c->batch <= 0 || c->n_kv_heads <= 0 || c->n_q_heads <= 0 || c->n_pages <= 0 || c->max_pages <= 0) return OKQ_ERR_INVALID_ARG;
  if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256) return OKQ_ERR_UNSUPPORTED;
  if (c->dtype != OKQ_FP16 && c->dtype != OKQ_BF16) return OKQ_ERR_UNSUPPORTED;
  if (c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads / c->n_kv_heads > OKQ_MAX_GROUP) return OKQ_ERR_UNSUPPORTED;
  // token numbers, (layer, sequence, head) units and rows of the pool are 32-bit numbers in the kernels
  if ((long long)c->max_pages * c->page_tokens > (1ll << 30)) return OKQ_ERR_UNSUPPORTED;
  if ((double)c->n_layers * c->batch * c->n_kv_heads > 1 << 24) return OKQ_ERR_UNSUPPORTED;
  if ((double)c->n_layers * c->n_pages * c->n_kv_heads * 2.0 * c->page_tokens > 2147483647.0) return OKQ_ERR_UNSUPPORTED;
  if ((double)c->batch * c->max_pages > 2147483647.0) return OKQ_ERR_UNSUPPORTED;
  if (need_ptrs) {
    const void* p[7] = {c->codes, c->scales, c->raw, c->table, c->refs, c->seq_len, c->status};
    for (const void* x : p)
      if (!x) return OKQ_ERR_INVALID_ARG;
    for (const void* x : p)
      if (!aligned16(x)) return OKQ_ERR_ALIGNMENT;
  }
  return OKQ_OK;
}

okq_status check_paged_layers(const okq_paged* c, int32_t layer, int32_t layer_count) {
  const okq_status st = check_paged(c, true);
  if (st != OKQ_OK) return st;
  return layer < 0 || layer_count <= 0 || layer > c->n_layers - layer_count ? OKQ_ERR_INVALID_ARG : OKQ_OK;
}

PagedView paged_view(const okq_paged* c) {
  PagedView v;
  v.n_layers = c->n_layers; v.batch = c->batch; v.n_kv = c->n_kv_heads; v.group = c->n_q_heads / c->n_kv_heads;
  v.page = c->page_tokens;
  v.page_shift = 5;
  while ((1 << v.page_shift) < v.page) v.page_shift++;
  v.n_pages = c->n_pages; v.max_pages = c->max_pages;
  v.codes = c->codes; v.scales = c->scales; v.raw = c->raw;
  v.inv_group = (unsigned)(((1ull << 32) + v.group - 1) / v.group);
  v.table = c->table; v.refs = c->refs; v.seq_len = c->seq_len; v.status = c->status;
  return v;
}

}  // namespace okq

extern "C" {

okq_status okq_paged_sizes(const okq_paged* c, size_t out[7]) {
  const okq_status st = okq::check_paged(c, false);
  if (st != OKQ_OK) return st;
  if (!out) return OKQ_ERR_INVALID_ARG;
  const size_t rows = (size_t)c->n_layers * c->n_pages * c->n_kv_heads * 2 * c->page_tokens;
  out[0] = rows * OKQ_HEAD_DIM;
  out[1] = rows / okq::PB * sizeof(float);
  out[2] = (size_t)c->n_layers * c->batch * c->n_kv_heads * 2 * okq::PB * OKQ_HEAD_DIM * 2;
  out[3] = (size_t)c->batch * c->max_pages * sizeof(int32_t);
  out[4] = (size_t)c->n_pages * sizeof(int32_t);
  out[5] = (size_t)c->n_layers * c->batch * sizeof(int32_t);
  out[6] = 16;
  return OKQ_OK;
}

okq_status okq_paged_append(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* k, const int64_t ks[4], const void* v,
                            const int64_t vs[4], int32_t n_new, const int32_t* new_len, const okq_rope* rope, void* stream) {
  using namespace okq;
  okq_status st = check_paged_layers(cache, layer, layer_count);
  if (st != OKQ_OK) return st;
  if (n_new < 0 || (n_new > 0 && (!k || !v)) || !ks || !vs) return OKQ_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !strides_ok(ks, 4, 8) || !strides_ok(vs, 4, 8) || (reinterpret_cast<uintptr_t>(new_len) & 3))
    return OKQ_ERR_ALIGNMENT;
  if (n_new > (1 << 30)) return OKQ_ERR_UNSUPPORTED;
  RopeView r;
  if ((st = make_rope(rope, r)) != OKQ_OK) return st;
  if (n_new == 0) return OKQ_OK;
  const PagedView c = paged_view(cache);
  Rows kr{k, {ks[0], ks[1], ks[2], ks[3]}}, vr{v, {vs[0], vs[1], vs[2], vs[3]}};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return cache->dtype == OKQ_FP16 ? launch_append<__half>(c, layer, layer_count, kr, vr, n_new, new_len, r, s)
                                  : launch_append<__nv_bfloat16>(c, layer, layer_count, kr, vr, n_new, new_len, r, s);
}

okq_status okq_paged_read(const okq_paged* cache, int32_t layer, int32_t layer_count, int32_t begin, int32_t n, void* k_out, void* v_out,
                          void* stream) {
  using namespace okq;
  const okq_status st = check_paged_layers(cache, layer, layer_count);
  if (st != OKQ_OK) return st;
  if (begin < 0 || n < 0 || (n > 0 && (!k_out || !v_out)) || begin > INT32_MAX - n) return OKQ_ERR_INVALID_ARG;
  if (!aligned16(k_out) || !aligned16(v_out)) return OKQ_ERR_ALIGNMENT;
  if (n == 0) return OKQ_OK;
  const PagedView c = paged_view(cache);
  const int chunks = n / (NT / 8) + (n % (NT / 8) != 0);
  const long long grid = (long long)layer_count * c.batch * c.n_kv * chunks;
  if (grid > 0x7fffffffll) return OKQ_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (cache->dtype == OKQ_FP16)
    e = launch_dependent(k_paged_read<__half>, dim3((unsigned)grid), NT, 0, s, 1, c, layer, begin, n, static_cast<__half*>(k_out), static_cast<__half*>(v_out), chunks);
  else
    e = launch_dependent(k_paged_read<__nv_bfloat16>, dim3((unsigned)grid), NT, 0, s, 1, c, layer, begin, n, static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out), chunks);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // extern "C"
