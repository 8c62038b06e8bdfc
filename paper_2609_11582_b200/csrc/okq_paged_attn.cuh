// What the two attention kernels over the 8-bit paged cache share: how the work is cut and numbered, partial results, the merge.
//
// An item is a (layer, sequence, KV head) with up to ROWS of its query rows (row = query * group + head of the group), a tile 128 of its
// tokens.  Items follow one another in one long line of tiles; block c of the grid takes tiles [c * per, (c + 1) * per) of it,
// whatever the lengths are, which only the device knows.  A piece is what a block holds of an item: all of it (the block writes the
// output), or a part, whose unnormalised sums, maximum and normaliser go to one of the block's two slots (2 c for an item that began
// in an earlier block, 2 c + 1 for one that goes on in a later one).  k_paged_merge puts parts together, in order.
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
  float* slots;     // [2 * grid][ROWS * (128 + 2)]: sums, maxima, normalisers
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

// All threads of a block find the whole line's length and the place of tile `want(total)`: cur, and the number of the first
// tile of its item.  Threads hold consecutive ranges of pairs.
struct FindSmem {
  long long warp[32];
  long long total, item0;
  int place[4];
};
template <int ROWS, int NT, class F>
__device__ __forceinline__ void find_place(FindSmem& sm, const Work<ROWS>& w, F&& want, Cursor<ROWS>& cur, long long& target) {
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
  if (tid == 0) { sm.place[0] = w.pairs; sm.place[1] = sm.place[2] = sm.place[3] = 0; sm.item0 = 0; }
  __syncthreads();
  long long before = v - mine, total = 0;
  for (int i = 0; i < NT / 32; i++) {
    if (i < wp) before += sm.warp[i];
    total += sm.warp[i];
  }
  if (tid == 0) sm.total = total;
  target = want(total);
  if (target >= before && target < before + mine) {
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
      sm.place[0] = p; sm.place[1] = h; sm.place[2] = rt; sm.place[3] = (int)(target - at);
      sm.item0 = at;
      break;
    }
  }
  __syncthreads();
  cur.pair = sm.place[0]; cur.h = sm.place[1]; cur.rt = sm.place[2]; cur.tile = sm.place[3];
  cur.len = cur.m = cur.nt = 0;
  if (cur.pair < w.pairs) cur.load(w);
}

__device__ __forceinline__ long long tiles_per_block(long long total, int grid) { return total <= 0 ? 1 : (total + grid - 1) / grid; }

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

// Block i merges the item that the cut between blocks i and i + 1 of the attention kernel lies in, if it is that item's first cut.
template <class T, int ROWS, int NT>
__global__ void __launch_bounds__(NT) k_paged_merge(const AttnArgs a, int grid) {
  __shared__ FindSmem fs;
  depend_wait();
  const Work<ROWS> w(a);
  Cursor<ROWS> cur;
  long long g, per = 1;
  find_place<ROWS, NT>(fs, w, [&](long long total) { per = tiles_per_block(total, grid); return ((long long)blockIdx.x + 1) * per; }, cur, g);
  if (cur.pair >= w.pairs || cur.tile == 0) return;                 // behind the last tile, or between two items
  const long long item0 = fs.item0;
  const int first = (int)(item0 / per), last = (int)((item0 + cur.nt - 1) / per);
  if (first != (int)blockIdx.x) return;
  constexpr size_t SLOT = (size_t)ROWS * (D + 2);
  const int rows = min(ROWS, cur.m * w.group - cur.rt * ROWS);
  for (int e = threadIdx.x; e < rows * D; e += NT) {
    const int r = e / D, ch = e % D;
    const float* s0 = a.slots + (size_t)(2 * first + 1) * SLOT;
    float mx = s0[ROWS * D + r], l = s0[ROWS * D + ROWS + r], o = s0[e];
    for (int c = first + 1; c <= last; c++) {
      const float* s = a.slots + (size_t)(2 * c) * SLOT;
      const float m2 = s[ROWS * D + r], l2 = s[ROWS * D + ROWS + r], o2 = s[e];
      const float mn = fmaxf(mx, m2), at = mn == -INFINITY ? 0.f : mn, f1 = ex2(mx - at), f2 = ex2(m2 - at);
      l = l * f1 + l2 * f2;
      o = o * f1 + o2 * f2;
      mx = mn;
    }
    out_row<T>(a, cur.pair, cur.h, cur.rt * ROWS + r)[ch] = from_f<T>(l == 0.f ? 0.f : o / l);
  }
}

// launches (okq_paged_attn.cu, okq_paged_decode.cu)
cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, int grid, cudaStream_t s);
constexpr int DECODE_ROWS = 8;

}  // namespace okq
