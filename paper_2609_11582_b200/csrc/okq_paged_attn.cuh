// What the two attention kernels over the 8-bit paged cache share: how the work is cut and numbered, partial results, the merge.
//
// An item is a (layer, sequence, KV head) with up to ROWS of its query rows (row = query * group + head of the group), a tile 128 of its
// tokens.  Items follow one another in one long line of tiles, which is cut into as many even ranges as there are pipelines on the GPU
// (fewer where there are fewer tiles), whatever the lengths are, which only the device knows.  A piece is what a range holds of an
// item: all of it (its pipeline writes the output), or a part, whose unnormalised sums, maximum and normaliser go to one of the
// range's two slots (2 v for an item that began in an earlier range, 2 v + 1 for one that goes on in a later one).  k_paged_merge
// puts parts together, in order.
#pragma once
#include "okq_device.cuh"
#include "okq_paged.cuh"

namespace okq {

constexpr int PT = 128;   // tokens of a tile

struct QRows {
  const void* p;
  int64_t s[4];
};
struct ORows {
  void* p;
  int64_t s[4];
};

struct AttnArgs {
  PagedView c;
  QRows q;
  ORows o;
  const int32_t* q_len;
  RopeView rope;
  int layer, layer_count, n_new;
  float scale2;     // softmax scale times log2(e)
  struct Head* heads;   // [ranges]
  float* slots;         // [2 * ranges][ROWS * (128 + 2)]: sums, maxima, normalisers
};

// tiles that an item reads: those up to the last token that its last row sees
template <int ROWS> struct Work {
  int pairs, n_kv, group;
  const AttnArgs& a;
  __device__ __forceinline__ explicit Work(const AttnArgs& args) : pairs(args.layer_count * args.c.batch), n_kv(args.c.n_kv), group(args.c.group), a(args) {}
  __device__ __forceinline__ void lens(int pair, int& len, int& m) const {   // tokens held, queries
    len = a.c.held(a.layer + pair / a.c.batch, pair % a.c.batch);
    m = count_of(a.q_len, pair % a.c.batch, a.n_new);
  }
  __device__ __forceinline__ int row_tiles(int m) const { return (m * group + ROWS - 1) / ROWS; }
  __device__ __forceinline__ int tiles(int len, int m, int rt) const {
    const int last = (min(m * group, (rt + 1) * ROWS) - 1) / group;   // query of the last row
    const int seen = len - m + last + 1;
    return seen <= 0 ? 0 : (seen + PT - 1) / PT;
  }
  __device__ __forceinline__ int head_tiles(int len, int m) const {   // of all row tiles of one head
    int s = 0;
    for (int rt = 0; rt < row_tiles(m); rt++) s += tiles(len, m, rt);
    return s;
  }
};

// A place in the line of tiles.
template <int ROWS> struct Cursor {
  int pair, h, rt, tile;     // item and tile inside it
  int len, m, nt;            // of the item: tokens, queries, tiles
  __device__ __forceinline__ void load(const Work<ROWS>& w) { w.lens(pair, len, m); nt = m ? w.tiles(len, m, rt) : 0; }
  __device__ __forceinline__ void next_item(const Work<ROWS>& w) {
    tile = 0;
    for (;;) {
      if (++rt < w.row_tiles(m)) nt = w.tiles(len, m, rt);
      else if (rt = 0, ++h < w.n_kv) nt = m ? w.tiles(len, m, 0) : 0;
      else {
        h = 0;
        if (++pair >= w.pairs) return;
        load(w);
      }
      if (nt > 0) return;
    }
  }
  __device__ __forceinline__ void next(const Work<ROWS>& w) {
    if (++tile == nt) next_item(w);
  }
};

// The line of `total` tiles in `ranges` parts: range v has tiles [start(v), start(v + 1)).
struct Cuts {
  long long total;
  int ranges;        // of those, min(ranges, total) hold tiles
  __device__ __forceinline__ int used() const { return total < ranges ? (int)total : ranges; }
  __device__ __forceinline__ long long start(int v) const { return v >= used() ? total : (long long)v * total / used(); }
  __device__ __forceinline__ int range_of(long long tile) const { return (int)(((tile + 1) * used() - 1) / total); }
};

// All threads of a block find the line's length and where the first tiles of the block's ranges v0, v0 + step, .. lie.  Threads hold
// consecutive pairs.
template <int G> struct FindSmem {
  long long warp[32];
  long long total;
  long long item0[G];   // first tile of the item that the range starts in
  int place[G][4];
};
template <int ROWS, int NT, int G>
__device__ __forceinline__ Cuts find_places(FindSmem<G>& sm, const Work<ROWS>& w, int ranges, int v0, int step) {
  const int tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  const int chunk = (w.pairs + NT - 1) / NT, p0 = min(w.pairs, tid * chunk), p1 = min(w.pairs, p0 + chunk);
  long long mine = 0;
  for (int p = p0; p < p1; p++) {
    int len, m;
    w.lens(p, len, m);
    mine += (long long)w.head_tiles(len, m) * w.n_kv;
  }
  long long v = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += y;
  }
  if (lane == 31) sm.warp[wp] = v;
  __syncthreads();
  long long before = v - mine, total = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; i++) {
    if (i < wp) before += sm.warp[i];
    total += sm.warp[i];
  }
  const Cuts cuts{total, ranges};
  if (tid == 0) sm.total = total;
  for (int g = 0; g < G && mine > 0; g++) {
    const long long target = cuts.start(v0 + g * step);
    if (target < before || target >= before + mine) continue;
    long long at = before;
    for (int p = p0; p < p1; p++) {
      int len, m;
      w.lens(p, len, m);
      const int per_head = w.head_tiles(len, m);
      if (target >= at + (long long)per_head * w.n_kv) { at += (long long)per_head * w.n_kv; continue; }
      const int h = (int)((target - at) / per_head);
      at += (long long)h * per_head;
      int rt = 0;
      while (target >= at + w.tiles(len, m, rt)) at += w.tiles(len, m, rt++);
      sm.place[g][0] = p; sm.place[g][1] = h; sm.place[g][2] = rt; sm.place[g][3] = (int)(target - at);
      sm.item0[g] = at;
      break;
    }
  }
  __syncthreads();
  return cuts;
}
// the place found for range v0 + g * step; not to be called for a range without tiles
template <int ROWS, int G> __device__ __forceinline__ Cursor<ROWS> place(const FindSmem<G>& sm, const Work<ROWS>& w, int g) {
  Cursor<ROWS> c;
  c.pair = sm.place[g][0]; c.h = sm.place[g][1]; c.rt = sm.place[g][2]; c.tile = sm.place[g][3];
  c.load(w);
  return c;
}

template <class T> __device__ __forceinline__ T* out_row(const AttnArgs& a, int pair, int h, int row) {
  const int li = pair / a.c.batch, b = pair % a.c.batch, g = a.c.group;
  return static_cast<T*>(a.o.p) + li * a.o.s[0] + b * a.o.s[1] + (h * g + row % g) * a.o.s[2] + (row / g) * a.o.s[3];
}

// zeros for the rows of items without tiles: a query that sees nothing.  `who` of `n_who` groups of 32 lanes.
template <class T, int ROWS> __device__ __forceinline__ void write_empty(const AttnArgs& a, const Work<ROWS>& w, int who, int n_who, int lane) {
  for (int pair = who; pair < w.pairs; pair += n_who) {
    int len, m;
    w.lens(pair, len, m);
    if (m <= len) continue;                  // every query sees at least its own token
    for (int rt = 0; rt < w.row_tiles(m) && w.tiles(len, m, rt) == 0; rt++)
      for (int row = rt * ROWS; row < min(m * w.group, (rt + 1) * ROWS); row++)
        for (int h = 0; h < w.n_kv; h++) *reinterpret_cast<uint2*>(out_row<T>(a, pair, h, row) + 4 * lane) = make_uint2(0u, 0u);
  }
}

// What a range leaves for the merge: its last item goes on in the next `more` ranges (0: it does not).
struct Head {
  int more, pair, h, rt;
};

constexpr int MERGE_NT = 512, MERGE_ROWS = 8;

// Block (v, y): rows [8 y, 8 y + 8) of the item that begins in range v and goes on behind it, if there is one.  A thread has four
// channels of a row, and the parts of its half; factors of 32 parts at a time.  Bound by latency: the parts are a megabyte at most in
// all; loads of eight parts are in flight per thread.
template <class T, int ROWS>
__global__ void __launch_bounds__(MERGE_NT) k_paged_merge(const AttnArgs a) {
  constexpr int CH = 64;                       // parts whose factors are in shared memory
  __shared__ float fac[MERGE_ROWS][CH], norm[MERGE_ROWS];
  __shared__ float4 half_sum[MERGE_ROWS * D / 4];
  depend_wait();
  const int v = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Head hd = a.heads[v];
  if (hd.more == 0) return;
  constexpr size_t SLOT = (size_t)ROWS * (D + 2);
  const int n = hd.more + 1, row0 = MERGE_ROWS * blockIdx.y;
  auto slot = [&](int k) { return a.slots + (size_t)(k == 0 ? 2 * v + 1 : 2 * (v + k)) * SLOT; };
  const int r = (tid & 255) >> 5, part = tid >> 8;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY;
  if (warp < MERGE_ROWS) {
    for (int k = lane; k < n; k += 32) top = fmaxf(top, slot(k)[ROWS * D + row0 + warp]);
#pragma unroll
    for (int w = 16; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    if (top == -INFINITY) top = 0.f;
  }
  float l = 0.f;
  for (int k0 = 0; k0 < n; k0 += CH) {
    const int kn = min(CH, n - k0);
    __syncthreads();
    if (warp < MERGE_ROWS)
      for (int k = lane; k < kn; k += 32) {
        const float* s = slot(k0 + k) + ROWS * D + row0 + warp;
        const float f = ex2(s[0] - top);
        fac[warp][k] = f;
        l += s[ROWS] * f;
      }
    __syncthreads();
#pragma unroll 8
    for (int k = part; k < kn; k += 2) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(slot(k0 + k) + (size_t)(row0 + r) * D) + lane);
      const float f = fac[r][k];
      acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y); acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
    }
  }
  if (warp < MERGE_ROWS) {
#pragma unroll
    for (int w = 16; w >= 1; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    if (lane == 0) norm[warp] = l;
  }
  if (part == 1) half_sum[tid & 255] = acc;
  __syncthreads();
  const Work<ROWS> w(a);
  int len, m;
  w.lens(hd.pair, len, m);
  const int row = hd.rt * ROWS + row0 + r;
  if (part == 0 && row < m * w.group) {
    const float4 y = half_sum[tid & 255];
    const float d = norm[r];
    T o[4] = {from_f<T>(d == 0.f ? 0.f : (acc.x + y.x) / d), from_f<T>(d == 0.f ? 0.f : (acc.y + y.y) / d),
              from_f<T>(d == 0.f ? 0.f : (acc.z + y.z) / d), from_f<T>(d == 0.f ? 0.f : (acc.w + y.w) / d)};
    *reinterpret_cast<uint2*>(out_row<T>(a, hd.pair, hd.h, row) + 4 * lane) = *reinterpret_cast<const uint2*>(o);
  }
}

// okq_paged_decode.cu: up to DECODE_ROWS rows, DECODE_PIPES pipelines per block
constexpr int DECODE_ROWS = 8, DECODE_PIPES = 3;
cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, int grid, cudaStream_t s);
inline size_t attn_workspace(int ranges, int rows) { return (size_t)ranges * (sizeof(int) * 4 + 2 * (size_t)rows * (D + 2) * sizeof(float)); }

}  // namespace okq
