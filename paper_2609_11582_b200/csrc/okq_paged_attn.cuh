// What the two attention kernels over the 8-bit paged cache share: how the work is cut and numbered, partial results, the merge.
//
// An item is a (layer, sequence, KV head) with up to ROWS of its query rows (row = query * group + head of the group), a tile 128 of its
// tokens.  Items follow one another in one long line of units, a unit for each tile and EXTRA behind an item's last for what an item
// costs besides (its queries, its output), and the line is cut into as many even ranges as there are pipelines on the GPU (fewer where
// there are fewer units), whatever the lengths are, which only the device knows.  A piece is what a range holds of an
// item: all of it (its pipeline writes the output), or a part, whose unnormalised sums, maximum and normaliser go to one of the
// range's two slots (2 v for an item that began in an earlier range, 2 v + 1 for one that goes on in a later one).  k_paged_merge
// puts parts together, in order.
#pragma once
#include "okq_device.cuh"
#include "okq_paged.cuh"
#include "okq_tc.cuh"

namespace okq {

constexpr int PT = 128;   // tokens of a tile

// Wait of a whole warp for one phase of an mbarrier: one look first, since most phases are complete when they are asked for and the
// bounded wait's clock and abort flag cost a hundred cycles.
template <class SM> __device__ __forceinline__ bool bar_wait(SM& sm, unsigned long long* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
               : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  if (__all_sync(0xffffffffu, ok != 0)) return true;
  return mbar_wait(sm, bar, parity);
}

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
  long long limit;  // SM clocks that a wait may take
  int withhold;     // testing aid: the first tile of every range is never delivered, so that the waits for it run out
  struct Head* heads;   // [Heads::count]
  float* slots;         // [2 * ranges][ROWS * (128 + 2)]: sums, maxima, normalisers
};

// tiles that an item reads: those up to the last token that its last row sees
template <int ROWS, int EXTRA> struct Work {
  int pairs, n_kv, group;
  const AttnArgs& a;
  __device__ __forceinline__ explicit Work(const AttnArgs& args) : pairs(args.layer_count * args.c.batch), n_kv(args.c.n_kv), group(args.c.group), a(args) {}
  __device__ __forceinline__ void lens(int li, int b, int& len, int& m) const {   // tokens held, queries
    const int n = __ldcg(&a.c.seq_len[(size_t)(a.layer + li) * a.c.batch + b]), q = a.q_len ? __ldcg(&a.q_len[b]) : a.n_new;   // (both loads before either is used)
    len = max(0, min(n, a.c.room()));
    m = max(0, min(q, a.n_new));
  }
  __device__ __forceinline__ int layer_of(int pair) const { return a.layer_count == 1 ? 0 : pair / a.c.batch; }
  __device__ __forceinline__ void lens(int pair, int& len, int& m) const {
    const int li = layer_of(pair);
    lens(li, pair - li * a.c.batch, len, m);
  }
  __device__ __forceinline__ int row_tiles(int m) const { return (m * group + ROWS - 1) / ROWS; }
  __device__ __forceinline__ int tiles(int len, int m, int rt) const {
    const int last = a.c.query_of(min(m * group, (rt + 1) * ROWS) - 1);   // query of the last row
    const int seen = len - m + last + 1;
    return seen <= 0 ? 0 : (seen + PT - 1) / PT;
  }
  __device__ __forceinline__ int units(int nt) const { return nt > 0 ? nt + EXTRA : 0; }
  __device__ __forceinline__ int head_units(int len, int m) const {   // of all row tiles of one head
    int s = 0;
    for (int rt = 0; rt < row_tiles(m); rt++) s += units(tiles(len, m, rt));
    return s;
  }
};

// A walk over the tiles of a range.
template <int ROWS, int EXTRA> struct Cursor {
  int pair, h, rt, tile;     // item and tile inside it
  int li, b;                 // layer (of the call's) and sequence of the pair
  int len, m, nt;            // of the item: tokens, queries, tiles
  int left;                  // units of the range from this tile on
  bool ok, ended;            // there is a tile here; the tile before was its item's last
  __device__ __forceinline__ void next_item(const Work<ROWS, EXTRA>& w) {
    tile = 0;
    for (;;) {
      if (++rt < w.row_tiles(m)) nt = w.tiles(len, m, rt);
      else if (rt = 0, ++h < w.n_kv) nt = m ? w.tiles(len, m, 0) : 0;
      else {
        h = 0;
        if (++pair >= w.pairs) { ok = false; return; }
        if (++b == w.a.c.batch) { b = 0; li++; }
        w.lens(li, b, len, m);
        nt = m ? w.tiles(len, m, 0) : 0;
      }
      if (nt > 0) return;
    }
  }
  __device__ __forceinline__ int piece() const { return min(nt - tile, left); }   // tiles of the item in the range, from this one on
  __device__ __forceinline__ void skip(const Work<ROWS, EXTRA>& w, int n) {       // no more than piece()
    tile += n;
    left -= n;
    ended = tile == nt;
    if (ended) left -= EXTRA;
    ok = left > 0;
    if (ended && ok) next_item(w);
  }
  __device__ __forceinline__ void next(const Work<ROWS, EXTRA>& w) { skip(w, 1); }
};

// The line of `total` units in `ranges` parts, as even as they go: the first `extra` of them have one unit more.  With fewer units than
// ranges the last ranges have none.  (Numbers of units have 32 bits: the caller sees to it.)
struct Cuts {
  int total, each, extra;
  __device__ __forceinline__ Cuts(int t, int ranges) : total(t), each(t / ranges), extra(t - each * ranges) {}
  __device__ __forceinline__ int start(int v) const { return v * each + min(v, extra); }
  __device__ __forceinline__ int size(int v) const { return each + (v < extra); }
  __device__ __forceinline__ int range_of(int unit) const {
    const int wide = extra * (each + 1);
    return unit < wide ? unit / (each + 1) : extra + (unit - wide) / each;
  }
};

// All threads of a block find the line's length and where the first units of the block's ranges v0, v0 + step, .. lie.  Threads hold
// consecutive pairs.
template <int G> struct FindSmem {
  int warp[32];
  int place[G][6];
};
template <int ROWS, int EXTRA, int NT, int G>
__device__ __forceinline__ Cuts find_places(FindSmem<G>& sm, const Work<ROWS, EXTRA>& w, int ranges, int v0, int step) {
  const int tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  const int chunk = (w.pairs + NT - 1) / NT, p0 = min(w.pairs, tid * chunk), p1 = min(w.pairs, p0 + chunk);
  int len = 0, m = 0, per_head = 0, mine = 0;    // (of the last pair looked at: with no more pairs than threads, the only one)
  for (int p = p0; p < p1; p++) {
    w.lens(p, len, m);
    per_head = w.head_units(len, m);
    mine += per_head * w.n_kv;
  }
  int v = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += y;
  }
  if (lane == 31) sm.warp[wp] = v;
  __syncthreads();
  int before = v - mine, total = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; i++) {
    const int x = sm.warp[i];
    if (i < wp) before += x;
    total += x;
  }
  const Cuts cuts(total, ranges);
  if (mine > 0) {
#pragma unroll
    for (int g = 0; g < G; g++) {
      const int target = cuts.start(v0 + g * step);
      if (target < before || target >= before + mine) continue;
      int at = before, p = p0;
      if (chunk > 1)
        for (;; p++) {
          w.lens(p, len, m);
          per_head = w.head_units(len, m);
          if (target < at + per_head * w.n_kv) break;
          at += per_head * w.n_kv;
        }
      const int h = (target - at) / per_head;
      at += h * per_head;
      int rt = 0;
      while (target >= at + w.units(w.tiles(len, m, rt))) at += w.units(w.tiles(len, m, rt++));
      sm.place[g][0] = p; sm.place[g][1] = h; sm.place[g][2] = rt; sm.place[g][3] = target - at; sm.place[g][4] = len; sm.place[g][5] = m;
    }
  }
  __syncthreads();
  return cuts;
}
// the first tile of range v = v0 + g * step
template <int ROWS, int EXTRA, int G>
__device__ __forceinline__ Cursor<ROWS, EXTRA> place(const FindSmem<G>& sm, const Work<ROWS, EXTRA>& w, const Cuts& cuts, int v, int g) {
  Cursor<ROWS, EXTRA> c{};
  c.left = cuts.size(v);
  c.ok = c.left > 0;
  if (!c.ok) return c;
  c.pair = sm.place[g][0]; c.h = sm.place[g][1]; c.rt = sm.place[g][2]; c.tile = sm.place[g][3]; c.len = sm.place[g][4]; c.m = sm.place[g][5];
  c.li = w.layer_of(c.pair);
  c.b = c.pair - c.li * w.a.c.batch;
  c.nt = w.tiles(c.len, c.m, c.rt);
  if (c.tile >= c.nt) {   // behind an item's last tile
    c.left -= c.nt + EXTRA - c.tile;
    c.ok = c.left > 0;
    if (c.ok) c.next_item(w);
  }
  return c;
}

template <class T> __device__ __forceinline__ T* out_row(const AttnArgs& a, int li, int b, int h, int row) {
  const int qi = a.c.query_of(row);
  return static_cast<T*>(a.o.p) + li * a.o.s[0] + b * a.o.s[1] + (h * a.c.group + row - qi * a.c.group) * a.o.s[2] + qi * a.o.s[3];
}
template <class T> __device__ __forceinline__ const T* query_row(const AttnArgs& a, int li, int b, int h, int row) {
  const int qi = a.c.query_of(row);
  return static_cast<const T*>(a.q.p) + li * a.q.s[0] + b * a.q.s[1] + (h * a.c.group + row - qi * a.c.group) * a.q.s[2] + qi * a.q.s[3];
}

// What is left for the merge: the item goes on in the `more` ranges behind range v (0: its output is written).  Heads are numbered by
// item where there are no more items than ranges, by the range that the item begins in otherwise: as few as there can be to look at.
struct Head {
  int more, v, pair, h, rt;
  int unused[3];
};
template <int ROWS> struct Heads {
  int row_tiles, items;      // of every head; of the call
  bool by_item;
  __host__ __device__ Heads(int pairs, int n_kv, int group, int n_new, int ranges)
      : row_tiles((n_new * group + ROWS - 1) / ROWS), items(pairs * n_kv * row_tiles), by_item(items <= ranges) {}
  __host__ __device__ int count(int ranges) const { return by_item ? items : ranges; }
  __device__ int at(int v, int n_kv, int pair, int h, int rt) const { return by_item ? (pair * n_kv + h) * row_tiles + rt : v; }
};

// Zeros for the rows of items without tiles (queries that see nothing), and the heads of these items.  `who` of `n_who` warps.
template <class T, int ROWS, int EXTRA>
__device__ __forceinline__ void write_empty(const AttnArgs& a, const Work<ROWS, EXTRA>& w, const Heads<ROWS>& heads, int who, int n_who, int lane) {
  for (int pair = who; pair < w.pairs; pair += n_who) {
    int len, m;
    const int li = w.layer_of(pair), b = pair - li * a.c.batch;
    w.lens(li, b, len, m);
    for (int rt = 0; rt < heads.row_tiles; rt++) {
      const bool rows = rt < w.row_tiles(m);
      if (rows && w.tiles(len, m, rt) > 0) continue;
      if (heads.by_item)
        for (int h = lane; h < w.n_kv; h += 32) a.heads[heads.at(0, w.n_kv, pair, h, rt)].more = 0;
      if (!rows) continue;
      for (int row = rt * ROWS; row < min(m * w.group, (rt + 1) * ROWS); row++)
        for (int h = 0; h < w.n_kv; h++) *reinterpret_cast<uint2*>(out_row<T>(a, li, b, h, row) + 4 * lane) = make_uint2(0u, 0u);
    }
  }
}

constexpr int MERGE_NT = 512;

// Block (x, y): rows of the item of head x, if it is in parts.  WPR warps to a row, of which each has every WPR-th part, a lane four
// channels.  Bound by latency: a few megabytes of parts at most; all of a part is loaded at once, seven parts in flight.
template <class T, int ROWS, int WPR>
__global__ void __launch_bounds__(MERGE_NT) k_paged_merge(const AttnArgs a) {
  constexpr int WARPS = MERGE_NT / 32;
  __shared__ float4 sums[WARPS][32];
  __shared__ float2 stat[WARPS];
  depend_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = blockIdx.y * (WARPS / WPR) + warp / WPR, first = warp % WPR;
  const int4 h0 = __ldcg(reinterpret_cast<const int4*>(&a.heads[blockIdx.x]));
  const Head hd{h0.x, h0.y, h0.z, h0.w, __ldcg(&a.heads[blockIdx.x].rt), {}};
  if (hd.more == 0) return;
  constexpr size_t SLOT = (size_t)ROWS * (D + 2);
  const int n = hd.more + 1, row = hd.rt * ROWS + r;
  auto slot = [&](int k) { return a.slots + (size_t)(2 * (hd.v + k) + (k == 0)) * SLOT; };
  const Work<ROWS, 0> w(a);
  int len, m;
  const int li = w.layer_of(hd.pair), b = hd.pair - li * a.c.batch;
  w.lens(li, b, len, m);
  const bool there = row < m * w.group;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, l = 0.f;
  if (there) {
    for (int k0 = first; k0 < n; k0 += 7 * WPR) {
      float4 x[7];
      float tk[7], lk[7];
#pragma unroll
      for (int e = 0; e < 7; e++) {
        const int k = k0 + e * WPR;
        tk[e] = -INFINITY;
        if (k >= n) continue;
        const float* s = slot(k);
        x[e] = __ldcg(reinterpret_cast<const float4*>(s + (size_t)r * D) + lane);
        tk[e] = __ldcg(s + ROWS * D + r);
        lk[e] = __ldcg(s + ROWS * D + ROWS + r);
      }
      float mn = top;
#pragma unroll
      for (int e = 0; e < 7; e++) mn = fmaxf(mn, tk[e]);
      const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(top - ref);
      l *= f0;
      acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
      top = mn;
#pragma unroll
      for (int e = 0; e < 7; e++) {
        if (k0 + e * WPR >= n) continue;
        const float f = ex2(tk[e] - ref);
        l = fmaf(lk[e], f, l);
        acc.x = fmaf(x[e].x, f, acc.x); acc.y = fmaf(x[e].y, f, acc.y); acc.z = fmaf(x[e].z, f, acc.z); acc.w = fmaf(x[e].w, f, acc.w);
      }
    }
  }
  if (WPR > 1) {
    sums[warp][lane] = acc;
    if (lane == 0) stat[warp] = make_float2(top, l);
    __syncthreads();
    if (first != 0) return;
    float mn = top;
#pragma unroll
    for (int i = 1; i < WPR; i++) mn = fmaxf(mn, stat[warp + i].x);
    const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(top - ref);
    l *= f0;
    acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
#pragma unroll
    for (int i = 1; i < WPR; i++) {
      const float f = ex2(stat[warp + i].x - ref);
      const float4 x = sums[warp + i][lane];
      l = fmaf(stat[warp + i].y, f, l);
      acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y); acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
    }
  }
  if (!there) return;
  T o[4] = {from_f<T>(l == 0.f ? 0.f : acc.x / l), from_f<T>(l == 0.f ? 0.f : acc.y / l), from_f<T>(l == 0.f ? 0.f : acc.z / l),
            from_f<T>(l == 0.f ? 0.f : acc.w / l)};
  *reinterpret_cast<uint2*>(out_row<T>(a, li, b, hd.h, row) + 4 * lane) = *reinterpret_cast<const uint2*>(o);
}
template <class T, int ROWS, int WPR> inline cudaError_t launch_merge_by(const AttnArgs& a, int heads, cudaStream_t s) {
  const long long rows = (long long)a.n_new * a.c.group;
  const int most = (int)(rows < ROWS ? rows : ROWS), per = MERGE_NT / 32 / WPR;
  return launch_dependent(k_paged_merge<T, ROWS, WPR>, dim3(heads, (most + per - 1) / per), MERGE_NT, 0, s, 1, a);
}
template <class T, int ROWS> inline cudaError_t launch_merge(const AttnArgs& a, int ranges, cudaStream_t s) {
  const Heads<ROWS> heads(a.layer_count * a.c.batch, a.c.n_kv, a.c.group, a.n_new, ranges);
  const int n = heads.count(ranges), parts = heads.items < ranges ? ranges / heads.items : 1;   // (of an item, were all alike)
  if (ROWS <= 8) return launch_merge_by<T, ROWS, MERGE_NT / 32>(a, n, s);
  // Warps to a row: more where one would load parts several times in a row, as long as the GPU holds them all at once (1 sequence of 32768
  // tokens, 32 rows: 37 us with one warp to a row, 20 with sixteen; 16 heads of 8000 tokens, 256 rows: 52 with one, 60 with four).
  const long long room = 4ll * sm_count() * (MERGE_NT / 32) / n, rows = (long long)a.n_new * a.c.group, most = rows < ROWS ? rows : ROWS;
  if (parts >= 28 && 16 * most <= room) return launch_merge_by<T, ROWS, 16>(a, n, s);
  return parts >= 15 && 4 * most <= room ? launch_merge_by<T, ROWS, 4>(a, n, s) : launch_merge_by<T, ROWS, 1>(a, n, s);
}

// okq_paged_decode.cu: DECODE_ROWS rows to an item, DECODE_PIPES pipelines per block.  An item's own costs (queries, the first tile's
// latency, the output) in tiles, as measured: 64 sequences x 8 heads of up to 1500 tokens, 24 rows, 93 us with 1, 75 with 2, 71 with 3.
constexpr int DECODE_ROWS = 8, DECODE_PIPES = 3, DECODE_EXTRA = 3;
cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, int blocks, int cluster, cudaStream_t s);   // cluster 0: ranges of the line, merge
int decode_clusters(int size);   // clusters of so many blocks (at most eight) that run at once
// okq_paged_prompt.cu: PROMPT_ROWS rows to an item, one pipeline per block.  Own costs alike: 16 sequences x 4 heads of up to 12345 tokens,
// 35 rows 62 us with 3, 58 with 4, 55 with 6, 56 with 8; 64 x 8 of up to 1500, 1024 rows, 555, 511, 462, 482.
constexpr int PROMPT_ROWS = 256, PROMPT_EXTRA = 6;
cudaError_t launch_paged_prompt(const AttnArgs& a, int dtype, int grid, cudaStream_t s);

// the pool's codes as rows of 128 bytes, copied 32 at a time
inline bool codes_map(CUtensorMap& map, const PagedView& c, bool swizzled) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)c.n_layers * c.n_pages * c.n_kv * 2 * c.page}, str[1] = {(cuuint64_t)D};
  const cuuint32_t box[2] = {(cuuint32_t)D, (cuuint32_t)PB}, estr[2] = {1, 1};
  return enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c.codes, dims, str, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace okq
