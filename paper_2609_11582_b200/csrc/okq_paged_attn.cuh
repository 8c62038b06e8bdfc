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

// Which of the tokens up to its own a query sees: all; the last `window` and the first `sinks`; those before the drafted tree and the nodes
// that its bits name.  A template argument of the kernels, so that the first is what it would be without the others.
enum Sight { CAUSAL, WINDOW, TREE };

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
  int window, sinks;                    // WINDOW
  const unsigned long long* seen;       // TREE: [batch][n_new][words]
  int words;
};

// n lowest bits of 64
__device__ __forceinline__ unsigned long long low_bits(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

// Tiles that an item reads: those up to the last token that its last row sees, all of the sequence's for a tree (bits are in any order).  With
// a window those between the sinks and the first token that its first row sees by the window are left out: an item's tiles are numbered
// without them, `head` of them lie before the gap.
struct Span {
  int nt, head, gap;
};
template <int ROWS, int EXTRA, int SIGHT = CAUSAL> struct Work {
  int pairs, n_kv, group;
  uint32_t whole_at = 0;   // CAN_BE_WHOLE: place in shared memory of FindWhole's `whole`
  __device__ __forceinline__ bool whole() const {
    int x;
    asm volatile("ld.shared.s32 %0, [%1];\n" : "=r"(x) : "r"(whole_at) : "memory");
    return x != 0;
  }
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
  // first token that the item's first row sees by the window (or a negative number)
  __device__ __forceinline__ int window_from(int len, int m, int rt) const { return max(0, len - m + a.c.query_of(rt * ROWS)) - a.window + 1; }
  __device__ __forceinline__ Span span(int len, int m, int rt) const {
    const int last = a.c.query_of(min(m * group, (rt + 1) * ROWS) - 1), seen = SIGHT == TREE ? len : len - m + last + 1;
    Span s{seen <= 0 ? 0 : (seen + PT - 1) / PT, 0, 0};
    if (SIGHT == WINDOW && s.nt > 0) {
      s.head = (min(a.sinks, seen) + PT - 1) / PT;
      s.gap = max(0, max(0, window_from(len, m, rt)) / PT - s.head);
      s.nt -= s.gap;
    }
    return s;
  }
  __device__ __forceinline__ int tiles(int len, int m, int rt) const {
    if (SIGHT != CAUSAL) return span(len, m, rt).nt;
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

// Whether the line may be cut between items only: where many rows are put together by a merge that costs several tiles, and where the causal
// kernels' results would not change with it.
template <int ROWS, int SIGHT> constexpr bool CAN_BE_WHOLE = ROWS > 8 && SIGHT != CAUSAL;

// A walk over the tiles of a range.
template <int ROWS, int EXTRA, int SIGHT = CAUSAL> struct Cursor {
  int pair, h, rt, tile;     // item and tile inside it
  int li, b;                 // layer (of the call's) and sequence of the pair
  int len, m, nt;            // of the item: tokens, queries, tiles
  int head, gap;             // WINDOW: Span's
  int left;                  // units of the range from this tile on
  bool ok, ended;            // there is a tile here; the tile before was its item's last
  // number of the item's tile i among the sequence's
  __device__ __forceinline__ int at(int i) const { return SIGHT == WINDOW && i >= head ? i + gap : i; }
  __device__ __forceinline__ void measure(const Work<ROWS, EXTRA, SIGHT>& w) {
    if (SIGHT != WINDOW) {
      nt = w.tiles(len, m, rt);
    } else {
      const Span s = w.span(len, m, rt);
      nt = s.nt;
      head = s.head;
      gap = s.gap;
    }
  }
  __device__ __forceinline__ void next_item(const Work<ROWS, EXTRA, SIGHT>& w) {
    tile = 0;
    for (;;) {
      nt = 0;
      if (++rt < w.row_tiles(m)) measure(w);
      else if (rt = 0, ++h < w.n_kv) {
        if (m) measure(w);
      } else {
        h = 0;
        if (++pair >= w.pairs) { ok = false; return; }
        if (++b == w.a.c.batch) { b = 0; li++; }
        w.lens(li, b, len, m);
        if (m) measure(w);
      }
      if (nt > 0) return;
    }
  }
  __device__ __forceinline__ int piece(const Work<ROWS, EXTRA, SIGHT>& w) const {   // tiles of the item in the range, from this one on
    return CAN_BE_WHOLE<ROWS, SIGHT> && w.whole() ? nt - tile : min(nt - tile, left);
  }
  __device__ __forceinline__ void skip(const Work<ROWS, EXTRA, SIGHT>& w, int n) {       // no more than piece()
    tile += n;
    left -= n;
    ended = tile == nt;
    if (ended) left -= EXTRA;
    ok = left > 0 || (CAN_BE_WHOLE<ROWS, SIGHT> && w.whole() && !ended);
    if (ended && ok) next_item(w);
  }
  __device__ __forceinline__ void next(const Work<ROWS, EXTRA, SIGHT>& w) { skip(w, 1); }
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

// Units of a head's row tiles before tile `rt` that begin no later than `offset`, found by a warp, 32 row tiles at a time; all lanes get the
// same answer.  (With one thread and 56 row tiles finding the first tile took 10000 to 23000 cycles of a block's 170000.)
template <int ROWS, int EXTRA, int SIGHT>
__device__ __forceinline__ int warp_units(const Work<ROWS, EXTRA, SIGHT>& w, int len, int m, int lane) {   // of the whole head
  int s = 0;
  for (int rt = lane; rt < w.row_tiles(m); rt += 32) s += w.units(w.tiles(len, m, rt));
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;
}
template <int ROWS, int EXTRA, int SIGHT>
__device__ __forceinline__ void warp_row_tile(const Work<ROWS, EXTRA, SIGHT>& w, int len, int m, int offset, int lane, int& rt, int& tile) {
  for (int rt0 = 0, at = 0;; rt0 += 32) {
    int u = rt0 + lane < w.row_tiles(m) ? w.units(w.tiles(len, m, rt0 + lane)) : 0, end = u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, end, d);
      if (lane >= d) end += y;
    }
    const unsigned behind = __ballot_sync(0xffffffffu, offset < at + end);   // row tiles that end behind the unit
    if (behind) {
      const int l = __ffs(behind) - 1;
      rt = rt0 + l;
      tile = offset - (at + __shfl_sync(0xffffffffu, end - u, l));
      return;
    }
    at += __shfl_sync(0xffffffffu, end, 31);
    if (rt0 + 32 >= w.row_tiles(m)) { rt = tile = 0; return; }   // (cannot be: the unit is the head's)
  }
}

// All threads of a block find the line's length and where the first units of the block's ranges v0, v0 + step, .. lie.  Threads hold
// consecutive pairs.
constexpr float WHOLE_GAIN = 8.f;   // what a merge and its parts cost, in units
template <int G> struct FindSmem {
  int warp[16];   // units of a warp's pairs
  int place[G][6];
};
struct FindWhole : FindSmem<1> {     // CAN_BE_WHOLE
  int items[16], most[16];   // of a warp's pairs: items, the largest item's units
  int whole;
};
template <int ROWS, int EXTRA, int NT, int G, int SIGHT, class Smem>
__device__ __forceinline__ Cuts find_places(Smem& sm, const Work<ROWS, EXTRA, SIGHT>& w, int ranges, int v0, int step) {
  static_assert(NT <= 512, "a place for each warp");
  const int tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  const int chunk = (w.pairs + NT - 1) / NT, p0 = min(w.pairs, tid * chunk), p1 = min(w.pairs, p0 + chunk);
  int len = 0, m = 0, per_head = 0, mine = 0;    // (of the last pair looked at: with no more pairs than threads, the only one)
  // whether a warp goes through its pairs' row tiles together
  const int row_tiles = w.row_tiles(w.a.n_new), pairs_here = min(32, max(0, w.pairs - 32 * wp));
  const bool together = ROWS > 8 && chunk == 1 && pairs_here * ((row_tiles + 31) / 32) < row_tiles;
  if (together) {
    if (p0 < p1) w.lens(p0, len, m);
    for (int l = 0; l < pairs_here; l++) {
      const int s = warp_units(w, __shfl_sync(0xffffffffu, len, l), __shfl_sync(0xffffffffu, m, l), lane);
      if (lane == l) per_head = s;
    }
    mine = per_head * w.n_kv;
  } else {
    for (int p = p0; p < p1; p++) {
      w.lens(p, len, m);
      per_head = w.head_units(len, m);
      mine += per_head * w.n_kv;
    }
  }
  int v = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += y;
  }
  if (lane == 31) sm.warp[wp] = v;
  if constexpr (CAN_BE_WHOLE<ROWS, SIGHT>) {
    int items = 0, most = 0;
    for (int p = p0; p < p1; p++) {
      if (chunk > 1) w.lens(p, len, m);
      const int n = w.row_tiles(m);
      items += n * w.n_kv;
      if (n > 0) most = max(most, max(w.units(w.tiles(len, m, 0)), w.units(w.tiles(len, m, n - 1))));   // (those between are hardly longer)
    }
    items = __reduce_add_sync(0xffffffffu, items);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) { sm.items[wp] = items; sm.most[wp] = most; }
  }
  __syncthreads();
  int before = v - mine, total = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; i++) {
    const int x = sm.warp[i];
    if (i < wp) before += x;
    total += x;
  }
  const Cuts cuts(total, ranges);
  if constexpr (CAN_BE_WHOLE<ROWS, SIGHT>) {
    // Whole items, as many rounds of the largest as it takes, against even parts and their merge, in units (us, whole items and even parts,
    // windows of long sequences: 224 items of 6 tiles 67, 74; of 14 tiles 121, 119; 240 items of 7 tiles 74, 80; 180 of 19 tiles 141, 119;
    // 240 ragged ones of up to 12 tiles 92, 74).  It is an estimate, good for items that are alike: a range takes the items that begin in it, its
    // share and up to one item more.
    int items = 0, most = 0;
#pragma unroll
    for (int i = 0; i < NT / 32; i++) {
      items += sm.items[i];
      most = max(most, sm.most[i]);
    }
    const int rounds = (items + ranges - 1) / ranges;
    sm.whole = rounds > 1 && (float)rounds * (float)most <= (float)total / (float)ranges + WHOLE_GAIN;
  }
  if (together) {
#pragma unroll
    for (int g = 0; g < G; g++) {
      const int target = cuts.start(v0 + g * step);
      const unsigned owner = __ballot_sync(0xffffffffu, mine > 0 && target >= before && target < before + mine);
      if (owner == 0) continue;
      const int l = __ffs(owner) - 1, heads = __shfl_sync(0xffffffffu, per_head, l), offset = target - __shfl_sync(0xffffffffu, before, l);
      const int h = offset / heads, len_l = __shfl_sync(0xffffffffu, len, l), m_l = __shfl_sync(0xffffffffu, m, l);
      int rt, tile;
      warp_row_tile(w, len_l, m_l, offset - h * heads, lane, rt, tile);
      if (lane == l) {
        sm.place[g][0] = p0; sm.place[g][1] = h; sm.place[g][2] = rt; sm.place[g][3] = tile; sm.place[g][4] = len; sm.place[g][5] = m;
      }
    }
  } else if (mine > 0) {
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
template <int ROWS, int EXTRA, int G, int SIGHT>
__device__ __forceinline__ Cursor<ROWS, EXTRA, SIGHT> place(const FindSmem<G>& sm, const Work<ROWS, EXTRA, SIGHT>& w, const Cuts& cuts, int v, int g) {
  Cursor<ROWS, EXTRA, SIGHT> c{};
  c.left = cuts.size(v);
  c.ok = c.left > 0;
  if (!c.ok) return c;
  c.pair = sm.place[g][0]; c.h = sm.place[g][1]; c.rt = sm.place[g][2]; c.tile = sm.place[g][3]; c.len = sm.place[g][4]; c.m = sm.place[g][5];
  c.li = w.layer_of(c.pair);
  c.b = c.pair - c.li * w.a.c.batch;
  c.measure(w);
  if (c.tile >= c.nt || (CAN_BE_WHOLE<ROWS, SIGHT> && w.whole() && c.tile > 0)) {   // behind an item's last tile, or where the range before goes on
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
template <class T, int ROWS, int EXTRA, int SIGHT>
__device__ __forceinline__ void write_empty(const AttnArgs& a, const Work<ROWS, EXTRA, SIGHT>& w, const Heads<ROWS>& heads, int who, int n_who, int lane) {
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

// A sum that falls so far below a new maximum that 2^d leaves fp32's normal numbers (the row's largest weight may lie on a token without
// value) is multiplied by 2^-100 first, and its maximum raised by as much.
constexpr float FALL = -120.f, LATE_BITS = 100.f, LATE = 7.888609e-31f;
__device__ __forceinline__ bool falls(float top, float ref) { return top - ref < FALL && top != -INFINITY; }

constexpr int MERGE_NT = 512;

// Block (x, y): row y of the item of head x, if it is in parts, each warp has every sixteenth part, a lane four channels.  Bound by latency:
// a few megabytes of parts at most; all of a part is loaded at once, seven parts in flight.  (Of the decode kernel's parts.)
// Parts far below the maximum are looked for once and added by a loop of their own: with a branch at each part in the common one, 64
// sequences x 8 heads of 1500 tokens took 58.4 us and not 57.2.
struct MergeSum {
  float top, l;
  float4 x;
  __device__ __forceinline__ void times(float f) {
    l *= f;
    x.x *= f; x.y *= f; x.z *= f; x.w *= f;
  }
  __device__ __forceinline__ void late(float ref) {
    if (!falls(top, ref)) return;
    top += LATE_BITS;
    times(LATE);
  }
  __device__ __forceinline__ void add(const MergeSum& y, float ref) {
    const float f = ex2(y.top - ref);
    l = fmaf(y.l, f, l);
    x.x = fmaf(y.x.x, f, x.x); x.y = fmaf(y.x.y, f, x.y); x.z = fmaf(y.x.z, f, x.z); x.w = fmaf(y.x.w, f, x.w);
  }
};
template <class T, int ROWS>
__global__ void __launch_bounds__(MERGE_NT, 2) k_paged_merge(const AttnArgs a) {
  constexpr int WARPS = MERGE_NT / 32;
  __shared__ float4 sums[WARPS][32];
  __shared__ float2 stat[WARPS];
  depend_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = blockIdx.y;
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
  if (row >= m * w.group) return;
  MergeSum acc{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  // to the maximum `mn` of acc and of what is added next
  auto raise = [&](float mn, float ref) {
    acc.late(ref);
    acc.times(ex2(acc.top - ref));
    acc.top = mn;
  };
  for (int k0 = warp; k0 < n; k0 += 7 * WARPS) {
    MergeSum y[7];
#pragma unroll
    for (int e = 0; e < 7; e++) {
      const int k = k0 + e * WARPS;
      y[e].top = -INFINITY;
      if (k >= n) continue;
      const float* s = slot(k);
      y[e].x = __ldcg(reinterpret_cast<const float4*>(s + (size_t)r * D) + lane);
      y[e].top = __ldcg(s + ROWS * D + r);
      y[e].l = __ldcg(s + ROWS * D + ROWS + r);
    }
    float mn = acc.top;
#pragma unroll
    for (int e = 0; e < 7; e++) mn = fmaxf(mn, y[e].top);
    const float ref = mn == -INFINITY ? 0.f : mn;
    if (n > WARPS) {   // (else the warp has one part at most, and that is the maximum)
#pragma unroll
      for (int e = 0; e < 7; e++) y[e].late(ref);
    }
    raise(mn, ref);
#pragma unroll
    for (int e = 0; e < 7; e++)
      if (k0 + e * WARPS < n) acc.add(y[e], ref);
  }
  sums[warp][lane] = acc.x;
  if (lane == 0) stat[warp] = make_float2(acc.top, acc.l);
  __syncthreads();
  if (warp != 0) return;
  float mn = acc.top;
#pragma unroll
  for (int i = 1; i < WARPS; i++) mn = fmaxf(mn, stat[i].x);
  const float ref = mn == -INFINITY ? 0.f : mn;
  const bool far = __any_sync(0xffffffffu, falls(stat[lane % WARPS].x, ref));
  raise(mn, ref);
  auto part = [&](int i) { return MergeSum{stat[i].x, stat[i].y, sums[i][lane]}; };
  if (far) {
#pragma unroll 1
    for (int i = 1; i < WARPS; i++) {
      MergeSum y = part(i);
      y.late(ref);
      acc.add(y, ref);
    }
  } else {
#pragma unroll
    for (int i = 1; i < WARPS; i++) acc.add(part(i), ref);
  }
  const float l = acc.l;
  T o[4] = {from_f<T>(l == 0.f ? 0.f : acc.x.x / l), from_f<T>(l == 0.f ? 0.f : acc.x.y / l), from_f<T>(l == 0.f ? 0.f : acc.x.z / l),
            from_f<T>(l == 0.f ? 0.f : acc.x.w / l)};
  *reinterpret_cast<uint2*>(out_row<T>(a, li, b, hd.h, row) + 4 * lane) = *reinterpret_cast<const uint2*>(o);
}
// okq_paged_decode.cu: DECODE_ROWS rows to an item, DECODE_PIPES pipelines per block.  An item's own costs (queries, the first tile's
// latency, the output) in tiles, as measured: 64 sequences x 8 heads of up to 1500 tokens, 24 rows, 93 us with 1, 75 with 2, 71 with 3.
constexpr int DECODE_ROWS = 8, DECODE_PIPES = 3, DECODE_EXTRA = 3;
cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, Sight sight, int blocks, int cluster, cudaStream_t s);   // cluster 0: ranges of the line, merge
int decode_clusters(int size);   // clusters of so many blocks (at most eight) that run at once
// okq_paged_prompt.cu: PROMPT_ROWS rows to an item, one pipeline per block.  Own costs alike: 16 sequences x 4 heads of up to 12345 tokens,
// 35 rows 62 us with 3, 58 with 4, 55 with 6, 56 with 8; 64 x 8 of up to 1500, 1024 rows, 555, 511, 462, 482.
constexpr int PROMPT_ROWS = 256, PROMPT_EXTRA = 6;
cudaError_t launch_paged_prompt(const AttnArgs& a, int dtype, Sight sight, int grid, cudaStream_t s);

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
