// Addresses, checks and rotary positions shared by the kernels of the 8-bit paged cache (okq_paged.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/okq_paged.h"
#include "okq_common.cuh"

namespace okq {

constexpr int PB = 32;   // tokens of a block: one scale per block, head and side

struct PagedView {
  int n_layers, batch, n_kv, group, page, page_shift, n_pages, max_pages;
  int8_t* codes;
  float* scales;
  void* raw;
  int32_t *table, *refs, *seq_len, *status;
  unsigned inv_group;   // ceil(2^32 / group): row / group without a division, exact for rows below 2^29

  __device__ __forceinline__ int query_of(int row) const { return group == 1 ? row : (int)__umulhi((unsigned)row, inv_group); }
  // first code of a page's head, keys (side 0) or values (side 1)
  __host__ __device__ size_t code_row(int l, int p, int h, int side) const {
    return ((((size_t)l * n_pages + p) * n_kv + h) * 2 + side) * page;   // in rows of 128
  }
  __device__ float* scale_of(int l, int p, int h, int side) const { return scales + code_row(l, p, h, side) / PB; }
  // (tables and lengths are read past the first cache: a kernel placed early may find what stood there before its predecessor's end)
  // page with token t of sequence b, -1 where there is none or the entry names none of the pool
  __device__ int page_of(int b, int t) const {
    const int j = t >> page_shift;
    const int p = j < max_pages ? __ldcg(&table[(size_t)b * max_pages + j]) : -1;
    return (unsigned)p < (unsigned)n_pages ? p : -1;
  }
  __device__ int room() const { return max_pages << page_shift; }   // tokens that a row has entries for
  __device__ int held(int l, int b) const {                         // tokens of a sequence
    const int n = __ldcg(&seq_len[(size_t)l * batch + b]);
    return n < 0 ? 0 : n > room() ? room() : n;
  }
  template <class T> __device__ T* raw_of(int l, int b, int h, int side) const {
    return static_cast<T*>(raw) + ((((size_t)l * batch + b) * n_kv + h) * 2 + side) * (PB * D);
  }
};

__device__ __forceinline__ void set_status(int32_t* status, int code) { atomicCAS(status, 0, code); }

// what a call asks for of n: all of it, or the sequence's own number
__device__ __forceinline__ int count_of(const int32_t* lens, int b, int n) {
  if (!lens) return n;
  const int m = __ldcg(&lens[b]);
  return m < 0 ? 0 : m > n ? n : m;
}

// ---- element types
template <class T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(float x) { return x; }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ float from_f(float x) { return x; }

template <class T> struct alignas(16) Vec8 { T v[8]; };   // eight channels (tensors and strides are multiples of 16 bytes, of fp32 too)

// ---- rotary positions
struct RopeView {
  const double* freq;        // null: no rotation
  const int32_t* positions;  // [3][batch][n]
  int half, s1, s2, s01, interleaved;   // pairs; sections 1 and 2 (interleaved); ends of the first two sections

  __device__ int axis(int c) const {
    if (!interleaved) return c < s1 ? 0 : c < s01 ? 1 : 2;
    const int m = c % 3;
    return m == 1 && c < 3 * s1 ? 1 : m == 2 && c < 3 * s2 ? 2 : 0;
  }
};

// cos and sin of an angle given in 64 bits: it is brought to a quarter of a turn around 0 there (fp32 would lose the fraction of a turn
// from a few thousand positions on) and rounded to fp32 once, an error of 2^-25 of a quarter; sincospif adds its two units in the last
// place.  The roundings in 64 bits are relative to the angle, 2^-51 of it at most: seen from 2^27 on, and in sines next to zero.
// Six operations of the fp64 pipe (with the series in 64 bits too one token of 8 sequences x 32 heads took 6.3 us, and not 4.3).
__device__ __forceinline__ void turn(double angle, float& c, float& s) {
  const double quarter = angle * 0.63661977236758134308;    // 2 / pi
  const double t = quarter + 6755399441055744.0;            // 1.5 * 2^52: rounds to an integer, whose low bits are t's
  const int q = __double2loint(t) & 3;
  float sn, cs;
  sincospif(0.5f * (float)(quarter - (t - 6755399441055744.0)), &sn, &cs);
  const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;
  c = (q == 1 || q == 2) ? -a : a;
  s = (q & 2) ? -b : b;
}
// of pairs c0 .. c0 + 7 of a token whose positions lie at pos[0], pos[axis_stride], pos[2 * axis_stride]
__device__ __forceinline__ void turns8(const RopeView& r, const int32_t* pos, size_t axis_stride, int c0, float (&c)[8], float (&s)[8]) {
  const double p0 = (double)pos[0], p1 = (double)pos[axis_stride], p2 = (double)pos[2 * axis_stride];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int ax = r.axis(c0 + i);
    turn((ax == 0 ? p0 : ax == 1 ? p1 : p2) * r.freq[c0 + i], c[i], s[i]);
  }
}
__device__ __forceinline__ void rotate_pair(float& a, float& b, float c, float s) {
  const float x = fmaf(a, c, -(b * s)), y = fmaf(b, c, a * s);
  a = x;
  b = y;
}

// ---- host side (okq_rope.cu, okq_paged.cu)
okq_status check_paged(const okq_paged* c, bool need_ptrs);
okq_status check_paged_layers(const okq_paged* c, int32_t layer, int32_t layer_count);
okq_status make_rope(const okq_rope* rope, RopeView& out);   // null gives a view without rotation
PagedView paged_view(const okq_paged* c);
// scratch of okq_pages_compact (the moves, at most one for every two pages, and a place per page), and of okq_pages_fork for `batch` pairs
inline size_t pages_workspace(const okq_paged* c) {
  const size_t compact = 16 + 8 * ((size_t)c->n_pages / 2 + 1) + 4 * (size_t)c->n_pages, fork = 16 * (size_t)c->batch;
  return compact > fork ? compact : fork;
}
inline bool strides_ok(const int64_t* s, int n, int multiple) {
  for (int i = 0; i < n; i++)
    if (s[i] % multiple != 0) return false;
  return true;
}

}  // namespace okq
