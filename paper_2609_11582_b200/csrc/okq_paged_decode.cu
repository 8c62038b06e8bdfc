// Attention over the 8-bit paged cache for few query rows per (layer, sequence, KV head): single tokens, a few drafted ones, and short
// pieces of prompts.  An item has up to eight rows.  With a window the tiles between the sinks and the window are left out, and of the
// others the blocks that no row sees; where some row does not see a tile's token, its score is -inf (of a tree: by the bits, loaded while
// the products are waited for).
//
// All products are of 8-bit integers on tcgen05 (kind::i8), with the cache's codes as they lie in memory for one operand:
//   scores   S[token][row] = K[token][channel] Q[row][channel]: A = a tile of 128 tokens (K-major), B = the queries as three signed
//            limbs of a 24-bit fixed-point number (per row: q / max|q| * 127 * 2^16), exact sums in int32
//   values   O[channel][row] = V[token][channel] P[token][row]: A = the tile transposed by its descriptor (MN-major), B = the numerators
//            p * scale_v as the four bytes of a 32-bit fixed-point number, exact sums in int32
// so nothing is unpacked: a tile goes from memory to shared memory by TMA and from there into the tensor cores.  Fixed point is
// relative to the row's largest p * scale_v in the tile (up to a factor of 4): the power of two R next above the largest log2 of p and
// scale is taken off in the exponent and put back in the factor of the tile's sums.  What lies more than 2^-30
// below the largest of the same tile is lost, whatever other tiles hold; fp32 would keep 2^-24 of each.
//
// A block has three pipelines, each with a range of tiles and a ring of two of its own, so that one tile's chain of products, softmax
// and products hides behind those of the others.  A pipeline is a service warp (copies of 32-token blocks by page, products) and four
// worker warps (an item's queries: rotation, limbs; softmax with lane = token; then, with lane = channel, the item's sums in fp32
// registers), which meet at mbarriers.  Fifteen warps leave 128 registers to a thread; with six warps to a pipeline (a loader of
// its own) there are 96, and the queries prepared by one warp held an item up by 10 us.
//
// Bound by memory: 256 bytes per token and head; an SM's share of the copy rate is a tile in about 1400 cycles.  16 sequences of 32768
// tokens x 4 heads (538 MB) take 95 us a call, 5.6 TB/s with the merge and both ends (93 in a graph); 1 sequence of 131072 tokens (134 MB,
// partly in the second-level cache) 34; 1 head of 2048 tokens 7.2, which is latency: launch, table, copies, products, the cluster's merge.
// 16 sequences x 4 heads with a window of 4096 and 64 sinks (68 MB, 2 blocks to each head) 21 us, 10 of them latency at both ends.
// (The running maxima in every thread and not in one lane per row: 98 us and not 95, 128 registers and not 127.)
#include "okq_paged_attn.cuh"

namespace okq {

namespace {

constexpr int R = DECODE_ROWS, G = DECODE_PIPES, EXTRA = DECODE_EXTRA;
constexpr int NS = 2;                     // ring of a pipeline
constexpr int SIDE = PT * D;              // bytes of a tile's keys or values
constexpr int WARPS = 5, SERVICE = 4;     // of a pipeline; the service warp's number in it
constexpr int NT = G * WARPS * 32;
constexpr uint32_t S_COL = 0, O_COL = 32, PIPE_COLS = 64, COLS = 256;
constexpr size_t SLOT = (size_t)R * (D + 2);
constexpr int MOST_CLUSTER = 8;

struct Pipe {
  __align__(1024) int8_t k[NS][SIDE];
  __align__(1024) int8_t v[NS][SIDE];
  __align__(1024) int8_t q[24 * D];          // rows limb * 8 + row, 128-byte swizzle (the product takes 32 rows: what the last
                                             // eight columns hold is not read)
  __align__(1024) uint32_t p[2][PT * 4];     // [half of the rows][token][row of the half]
};
struct PipeSync {
  __align__(16) float wmax[2][4][R];
  __align__(16) float qscale[R];
  __align__(16) float sum[4][R];             // an item's normalisers, by worker warp
  __align__(16) float scale[NS][12];         // of the tile's four blocks: keys; values as a fraction of [1/2, 1), 2^32 times, and its exponent
  __align__(8) unsigned long long full[NS], s_full, p_full, o_full, q_full;
};
struct DecodeSmem {
  Pipe pipe[G];
  PipeSync sync[G];
  FindSmem<G> find;
  uint32_t tmem_slot;
  long long limit;
  volatile int abort;
  volatile int tmem_busy;
};

__device__ __forceinline__ uint64_t make_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {   // no swizzle
  return (uint64_t)((saddr >> 4) & 0x3fff) | ((uint64_t)((lbo >> 4) & 0x3fff) << 16) | ((uint64_t)((sbo >> 4) & 0x3fff) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, bool acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}\n"
               ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void commit(unsigned long long* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, int (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;\n" : "=f"(y) : "f"(x));
  return y;
}

// the loader's view of one 32-token block of a coming tile
struct Block {
  int row;        // row of its keys in the pool; -1: behind the sequence's end, -2: its page is missing
  float ks, vs;
};

// Sums over the lanes of eight rows at once, to `to` by row: bits 4 .. 2 of a lane choose its row, then the four lanes of a row.
__device__ __forceinline__ void lane_sums(const float (&x)[R], float* to, int lane) {
  float w[R];
#pragma unroll
  for (int r = 0; r < R; r++) w[r] = x[r];
#pragma unroll
  for (int d = 16, n = 4; d >= 4; d >>= 1, n >>= 1) {
    const bool upper = (lane & d) != 0;
#pragma unroll
    for (int r = 0; r < 4; r++)
      if (r < n) {
        const float give = upper ? w[r] : w[r + n], keep = upper ? w[r + n] : w[r];
        w[r] = keep + __shfl_xor_sync(0xffffffffu, give, d);
      }
  }
  w[0] += __shfl_xor_sync(0xffffffffu, w[0], 2);
  w[0] += __shfl_xor_sync(0xffffffffu, w[0], 1);
  if ((lane & 3) == 0) to[lane >> 2] = w[0];
}

// Two of an item's rows, r0 and r0 + 1: limbs (swizzled) and scales.  One warp, four channels per lane.  `turns`: cosines and sines of
// the item's queries, [query from the first on][64 pairs].
template <class T, class Cur>
__device__ __forceinline__ void prepare_queries(const AttnArgs& a, const Cur& cur, int r0, const uint2 (&raw)[2], const float2* turns, int8_t* qbuf,
                                                float* qscale, int lane) {
  const int step = a.rope.half >> 2;   // lanes from a channel to its partner
  const bool turned = a.rope.freq && lane < 2 * step, low = lane < step;
  const int other = !turned ? lane : low ? lane + step : lane - step, pair0 = 4 * (low ? lane : lane - step);
#pragma unroll
  for (int e = 0; e < 2; e++) {
    const int r = r0 + e;
    const T* y = reinterpret_cast<const T*>(&raw[e]);
    float x[4] = {to_f(y[0]), to_f(y[1]), to_f(y[2]), to_f(y[3])};
    if (a.rope.freq) {
      const float2* cs = turns + 64 * (a.c.query_of(R * cur.rt + r) - a.c.query_of(R * cur.rt)) + pair0;
#pragma unroll
      for (int z = 0; z < 4; z++) {
        const float o = __shfl_sync(0xffffffffu, x[z], other);
        if (turned) {
          float u = low ? x[z] : o, w = low ? o : x[z];
          rotate_pair(u, w, cs[z].x, cs[z].y);
          x[z] = to_f(from_f<T>(low ? u : w));
        }
      }
    }
    unsigned mx = 0;
#pragma unroll
    for (int z = 0; z < 4; z++) mx = max(mx, __float_as_uint(x[z]) & 0x7fffffffu);
    mx = __reduce_max_sync(0xffffffffu, mx);
    // fixed point: 127 * 2^16 for the largest; numbers too small for a quotient (and infinities, NaN) have limbs of 0
    const float big = __uint_as_float(mx);
    const bool fine = mx < 0x7f800000u && big > 1e-30f;
    const float f = fine ? __fdiv_rn(127.f * 65536.f, big) : 0.f;   // (__fdividef gives 0 for divisors above 2^126, which bf16 has)
    // signed digits to the base 256: with 128 added to each, the bytes of one sum
    uint32_t u[4];
#pragma unroll
    for (int z = 0; z < 4; z++) u[z] = (uint32_t)((fine ? __float2int_rn(x[z] * f) : 0) + 0x808080) ^ 0x808080u;
    const uint32_t lo = __byte_perm(u[0], u[1], 0x5140), hi = __byte_perm(u[2], u[3], 0x5140);   // bytes 0, 0, 1, 1
    const uint32_t limb[3] = {__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632),
                              __byte_perm(__byte_perm(u[0], u[1], 0x0062), __byte_perm(u[2], u[3], 0x0062), 0x5410)};
#pragma unroll
    for (int n = 0; n < 3; n++) {
      const int line = 8 * n + r;
      *reinterpret_cast<uint32_t*>(qbuf + line * D + (((lane >> 2) ^ (line & 7)) << 4) + ((4 * lane) & 15)) = limb[n];
    }
    if (lane == 0) qscale[r] = mx >= 0x7f800000u ? NAN : big / (127.f * 65536.f) * a.scale2;
  }
}

// CLUSTER: every (layer, sequence, KV head) has a cluster of `size` blocks, whose pipelines share its tiles evenly, and its parts are put
// together in the cluster's shared memory: one launch.  Otherwise pipelines have even ranges of the whole line and k_paged_merge follows.
template <class T, bool CLUSTER, int SIGHT>
__global__ void __launch_bounds__(NT, 1) k_paged_decode(const __grid_constant__ CUtensorMap map, const AttnArgs a, int size) {
  extern __shared__ unsigned char raw_smem[];
  DecodeSmem& sm = *reinterpret_cast<DecodeSmem*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, lane = tid & 31;
  // warps 0 .. 11 are the workers (so that a warp's number mod 4 is its quarter of tensor memory), then the service warps
  const int warp = tid >> 5, g = warp < 4 * G ? warp / 4 : warp - 4 * G, role = warp < 4 * G ? warp % 4 : SERVICE;
  Pipe& pipe = sm.pipe[g];
  PipeSync& sy = sm.sync[g];
  if (tid < G) {
    auto init = [](unsigned long long* b, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(b)), "r"(count)); };
    PipeSync& mine = sm.sync[tid];
    for (int i = 0; i < NS; i++) init(&mine.full[i], 2);   // copies, scales
    init(&mine.s_full, 1);
    init(&mine.p_full, 4);
    init(&mine.o_full, 1);
    init(&mine.q_full, 4);
    sm.abort = 0;
    sm.tmem_busy = 0;
    sm.limit = a.limit;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&sm.tmem_slot)), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (warp == 4 * G && lane == 0) asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = sm.tmem_slot + PIPE_COLS * g;
  depend_wait();

  const PagedView& c = a.c;
  const Work<R, EXTRA, SIGHT> work(a);
  const Heads<R> heads(work.pairs, c.n_kv, c.group, a.n_new, G * gridDim.x);
  Cuts cuts(0, 1);
  int v = 0, end = 0;            // this pipeline's range of the line, and the unit behind it
  Cursor<R, EXTRA, SIGHT> cur{};
  int rank = 0;
  if (CLUSTER) {   // (grid (size x row tiles, heads, pairs): a division on the way to the first tile is felt)
    asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    asm("mov.u32 %0, %%clusterid.x;\n" : "=r"(cur.rt));
    cur.h = blockIdx.y;
    cur.pair = blockIdx.z;
    cur.li = work.layer_of(cur.pair);
    cur.b = cur.pair - cur.li * c.batch;
    work.lens(cur.li, cur.b, cur.len, cur.m);
    if (cur.rt < work.row_tiles(cur.m)) cur.measure(work);   // (else none)
    const Cuts share(cur.nt, G * size);
    cur.tile = share.start(g * size + rank);
    cur.left = share.size(g * size + rank);
    cur.ok = cur.left > 0;
  } else {
    cuts = find_places<R, EXTRA, NT, G, SIGHT>(sm.find, work, G * gridDim.x, blockIdx.x, gridDim.x);
    v = blockIdx.x + g * gridDim.x;
    end = cuts.start(v) + cuts.size(v);
    cur = place<R, EXTRA, G, SIGHT>(sm.find, work, cuts, v, g);
  }
  const int rows = min(R, cur.m * c.group - R * cur.rt);   // (CLUSTER: of the item)

  if (role == SERVICE) {
    // ------------------------------------------------------------------ copies and products
    constexpr uint32_t shape = (2u << 4) | ((32u >> 3) << 17) | (((uint32_t)PT >> 4) << 24);   // D int32, N 32, M 128
    constexpr uint32_t id_s = shape | (1u << 7) | (1u << 10);                                  // A, B signed, K-major
    constexpr uint32_t id_o = shape | (1u << 7) | (1u << 15) | (1u << 16);                     // A signed, B unsigned, both MN-major
    // Blocks of the tiles to come, eight tiles at a time, a lane for each block: entries of the page table when the batch before
    // begins, their scales halfway through it, so that neither load is waited for.
    Cursor<R, EXTRA, SIGHT> ahead = cur;      // first tile that has not been looked up
    int n_now = 0, n_nx = 0;           // tiles of a batch
    int t_nx = 0, l_nx = 0, h_nx = 0, page_nx = -1;
    bool in_nx = false;
    Block now{-1, 0.f, 0.f}, nxt{-1, 0.f, 0.f};
    auto entries = [&] {
      int b = 0, len = 0, from = 0;
      for (n_nx = 0; n_nx < 8 && ahead.ok; n_nx++) {
        if (lane >> 2 == n_nx) {
          t_nx = ahead.at(ahead.tile) * PT + PB * (lane & 3); len = ahead.len; l_nx = a.layer + ahead.li; b = ahead.b; h_nx = ahead.h;
          if (SIGHT == WINDOW) from = work.window_from(len, ahead.m, ahead.rt);
        }
        ahead.next(work);
      }
      in_nx = lane >> 2 < n_nx && t_nx < len;
      if (SIGHT == WINDOW) in_nx = in_nx && (t_nx < a.sinks || t_nx + PB > from);   // (blocks that no row sees may have no page)
      if (in_nx) {
        const int j = t_nx >> c.page_shift;
        page_nx = __ldcg(&c.table[(size_t)b * c.max_pages + j]);   // (held() keeps j inside the row)
      }
    };
    auto scales = [&] {
      nxt = Block{-1, 0.f, 0.f};
      if (!in_nx) return;
      if ((unsigned)page_nx >= (unsigned)c.n_pages) {
        nxt = Block{-2, NAN, NAN};
        set_status(c.status, OKQ_ERR_INVALID_ARG);
      } else {
        const size_t row = c.code_row(l_nx, page_nx, h_nx, 0) + (t_nx & (c.page - 1));
        nxt = Block{(int)row, __ldcg(&c.scales[row / PB]), __ldcg(&c.scales[(row + c.page) / PB])};
      }
    };
    auto load = [&](int i) {   // tile i into the ring, whose place is free
      const int k = i & 7, s = i % NS;
      if (k == 0) {
        now = nxt;
        n_now = n_nx;
        entries();
      }
      const bool mine = lane >> 2 == k, there = mine && now.row >= 0;
      const int blocks = __popc(__ballot_sync(0xffffffffu, there));
      const uint32_t bar = smem_u32(&sy.full[s]);
      if (lane == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(blocks * 2 * PB * D) : "memory");
      __syncwarp();
      if (there) {
        const int j = lane & 3;
#pragma unroll
        for (int side = 0; side < 2; side++)
          asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                       ::"r"(smem_u32(side ? pipe.v[s] : pipe.k[s]) + j * PB * D), "l"(reinterpret_cast<uint64_t>(&map)), "r"(0),
                         "r"(now.row + side * c.page), "r"(bar) : "memory");
      }
      if (mine) {   // (may still be on their way: behind the copies)
        int e;
        const float m = frexpf(now.vs, &e);
        sy.scale[s][lane & 3] = now.ks;
        sy.scale[s][4 + (lane & 3)] = m * 4294967296.f;
        sy.scale[s][8 + (lane & 3)] = m > 0.f && m < 1.f ? (float)e : -INFINITY;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sy.full[s]);
      if (k == 4) scales();
    };
    int items = 0, armed = 0, scored = 0, done = 0;
    auto score = [&](int i, bool fresh) {
      const int s = i % NS;
      if (fresh && !bar_wait(sm, &sy.q_full, (uint32_t)(items++) & 1u)) return false;
      if (!bar_wait(sm, &sy.full[s], (uint32_t)(i / NS) & 1u)) return false;
      if (elect_one()) {
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        const uint64_t ad = make_desc_sw128(smem_u32(pipe.k[s])), bd = make_desc_sw128(smem_u32(pipe.q));
#pragma unroll
        for (int k = 0; k < 4; k++) mma_i8(tmem + S_COL, ad + 2u * k, bd + 2u * k, id_s, k != 0);   // 32 channels further
        commit(&sy.s_full);
      }
      __syncwarp();
      scored = i + 1;
      return true;
    };
    auto more = [&] { return (armed & 7) == 0 ? n_nx > 0 : (armed & 7) < n_now; };   // there is a tile `armed`
    bool go = cur.ok;
    if (go) {
      entries();
      scales();
      while (armed < NS && more() && !a.withhold) load(armed++);
      go = score(0, true);
      for (int i = 0; go; i++) {
        cur.next(work);
        if (!bar_wait(sm, &sy.p_full, (uint32_t)i & 1u)) { go = false; break; }
        const int s = i % NS;
        if (elect_one()) {
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint64_t ad = make_desc_sw128(smem_u32(pipe.v[s])), bd = make_desc(smem_u32(pipe.p), 128, PT * 16);
#pragma unroll
          for (int k = 0; k < 4; k++) mma_i8(tmem + O_COL, ad + 256u * k, bd + 32u * k, id_o, k != 0);   // 32 tokens further
          commit(&sy.o_full);
        }
        __syncwarp();
        done = i + 1;
        // (the workers have read the scores of tile i; the next item's queries are not ready before they have its sums too)
        if (cur.ok && !cur.ended) go = score(i + 1, false);
        if (go && more() && (go = bar_wait(sm, &sy.o_full, (uint32_t)i & 1u))) load(armed++);
        if (go && cur.ok && cur.ended) go = score(i + 1, true);
        if (!cur.ok) break;
      }
    }
    // Nothing may be in flight when the block ends or tensor memory is released; if the last products do not answer, it stays allocated.
    if (!go)
      for (int i = max(0, armed - NS); i < armed; i++) mbar_drain(&sy.full[i % NS], (uint32_t)(i / NS) & 1u);
    if (scored >= 1 && !mbar_drain(&sy.s_full, (uint32_t)(scored - 1) & 1u)) sm.tmem_busy = 1;
    if (done >= 1 && !mbar_drain(&sy.o_full, (uint32_t)(done - 1) & 1u)) sm.tmem_busy = 1;
    if (!CLUSTER) write_empty<T>(a, work, heads, v, G * gridDim.x, lane);
  } else {
    // ------------------------------------------------------------------ workers (after a timeout they run on, waits failing at once)
    const uint32_t lanes = (uint32_t)(32 * role) << 16;
    const int ch = 32 * role + lane;
    const int rl = lane & (R - 1);   // the lane's own row, whose running maximum and factors it works out for all
    float top = -INFINITY, sum[R], o[R];
    bool fresh = true, whole = cur.tile == 0, began = cur.tile != 0;   // the piece has its item's first tile; the item began in an earlier range
    if (CLUSTER) {
#pragma unroll
      for (int r = 0; r < R; r++) sum[r] = o[r] = 0.f;
    }
    if (!CLUSTER && !heads.by_item && tid == g * 128) a.heads[v].more = 0;
    for (int i = 0; cur.ok; i++) {
      const int s = i % NS, b = i & 1;
      // what is needed of this item when the cursor has gone on: its last tile's unit, its rows, and the token of the tile's first lane
      // counted from the first that the first query does not see
      const int li = cur.li, bq = cur.b, h = cur.h, rt = cur.rt, item_end = end - cur.left - cur.tile + cur.nt - 1;
      const int rows = cur.m * c.group - R * rt, late = cur.at(cur.tile) * PT - (cur.len - cur.m + 1);
      if (fresh) {   // (the products of the item before are through: their sums have been read)
        // rows, and the turns of the item's queries (at most eight) in the place of the numerators
        const int row = R * rt + 2 * role;
        uint2 raw[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
          raw[e] = make_uint2(0u, 0u);
          if (2 * role + e < rows) raw[e] = *reinterpret_cast<const uint2*>(query_row<T>(a, li, bq, h, row + e) + 4 * lane);
        }
        float2* turns = reinterpret_cast<float2*>(pipe.p);
        if (a.rope.freq) {
          const size_t st = (size_t)c.batch * a.n_new;
          const int q0 = c.query_of(R * rt), nq = c.query_of(R * rt + min(rows, R) - 1) - q0 + 1;
          const int pair = ch & 63;
          const double f = pair < a.rope.half ? a.rope.freq[pair] : 0.0;
          const int32_t* pos = a.rope.positions + a.rope.axis(pair) * st + (size_t)bq * a.n_new + q0;
#pragma unroll 1
          for (int qi = ch >> 6; qi < nq; qi += 2) {
            float2 y;
            turn((double)pos[qi] * f, y.x, y.y);
            turns[64 * qi + pair] = y;
          }
          asm volatile("bar.sync %0, 128;\n" ::"r"(1 + g) : "memory");
        }
        prepare_queries<T>(a, cur, 2 * role, raw, turns, pipe.q, sy.qscale, lane);
        fence_async_smem();
        asm volatile("bar.sync %0, 128;\n" ::"r"(1 + g) : "memory");
        if (lane == 0) mbar_arrive(&sy.q_full);
#pragma unroll
        for (int r = 0; r < R; r++) sum[r] = o[r] = 0.f;
        top = -INFINITY;
      }
      // the rows that see the lane's token, a bit each
      unsigned sees = 0xffu;
      if (SIGHT == WINDOW) {
        const int base = cur.len - cur.m, t0 = late + base + 1, own = t0 + 32 * role + lane;
        const int q0 = c.query_of(R * rt), q1 = c.query_of(R * rt + min(rows, R) - 1);
        if (t0 + PT - 1 > base + q0 || (t0 + PT > a.sinks && t0 <= base + q1 - a.window)) {   // some row may not see all of the tile
          sees = 0;
#pragma unroll
          for (int r = 0; r < R; r++) {
            const int p = base + c.query_of(R * rt + r);
            if (own <= p && (own < a.sinks || p - own < a.window)) sees |= 1u << r;
          }
        }
      }
      if (SIGHT == TREE && late + PT > -1) {   // the tile has nodes, or ends behind the sequence
        const int node = late + 1 + 32 * role + lane;
        if (node >= 0) {
          sees = 0;
          if (node < cur.m) {
            unsigned long long bits[R];
#pragma unroll
            for (int r = 0; r < R; r++)
              bits[r] = r < rows ? __ldcg(a.seen + ((size_t)bq * a.n_new + c.query_of(R * rt + r)) * a.words + (node >> 6)) : 0ull;
#pragma unroll
            for (int r = 0; r < R; r++) sees |= (unsigned)(bits[r] >> (node & 63) & 1ull) << r;
          }
        }
      }
      cur.next(work);
      const bool last = cur.ended || !cur.ok;
      bar_wait(sm, &sy.full[s], (uint32_t)(i / NS) & 1u);   // (long complete: for the loader's scales)
      // scales of this warp's block of 32 tokens; exponents of the tile's value scales
      const float ks = sy.scale[s][role], frac = sy.scale[s][4 + role], exp_own = sy.scale[s][8 + role];
      const float4 ev = *reinterpret_cast<const float4*>(&sy.scale[s][8]);
      const bool lost = !(frac <= 4294967296.f);
      bar_wait(sm, &sy.s_full, (uint32_t)i & 1u);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      float x[R];
      {
        int d0[8], d1[8], d2[8];
        tmem_ld8(tmem + S_COL + lanes, d0);
        tmem_ld8(tmem + S_COL + 8u + lanes, d1);
        tmem_ld8(tmem + S_COL + 16u + lanes, d2);
        tmem_wait_ld();
#pragma unroll
        for (int r = 0; r < R; r++) x[r] = fmaf((float)d2[r], 65536.f, (float)(d1[r] * 256 + d0[r])) * (sy.qscale[r] * ks);
      }
      if (SIGHT != CAUSAL) {
#pragma unroll
        for (int r = 0; r < R; r++)
          if (!(sees >> r & 1u)) x[r] = -INFINITY;
      } else if (late + PT > 0) {   // some row may not see all of the tile
#pragma unroll
        for (int r = 0; r < R; r++)
          if (late + 32 * role + lane >= c.query_of(R * rt + r)) x[r] = -INFINITY;
      }
      {
        float w[R];
#pragma unroll
        for (int r = 0; r < R; r++) w[r] = warp_max(x[r]);
        if (lane == 0) {
          float4* to = reinterpret_cast<float4*>(sy.wmax[b][role]);
          to[0] = make_float4(w[0], w[1], w[2], w[3]);
          to[1] = make_float4(w[4], w[5], w[6], w[7]);
        }
      }
      asm volatile("bar.sync %0, 128;\n" ::"r"(1 + g) : "memory");
      const float w0 = sy.wmax[b][0][rl], w1 = sy.wmax[b][1][rl], w2 = sy.wmax[b][2][rl], w3 = sy.wmax[b][3][rl];
      const float mn = fmaxf(fmaxf(fmaxf(w0, w1), fmaxf(w2, w3)), top);
      if (__any_sync(0xffffffffu, mn > top)) {   // (the same in all of the pipeline's workers)
        float d = mn > top ? top - mn : 0.f;
        const bool far = falls(d, 0.f);
        if (__any_sync(0xffffffffu, far)) {
          d += far ? LATE_BITS : 0.f;
#pragma unroll
          for (int r = 0; r < R; r++) {
            const float f = __shfl_sync(0xffffffffu, far ? LATE : 1.f, r);
            sum[r] *= f;
            o[r] *= f;
          }
        }
        const float keep = ex2(d);
#pragma unroll
        for (int r = 0; r < R; r++) {
          const float f = __shfl_sync(0xffffffffu, keep, r);
          sum[r] *= f;
          o[r] *= f;
        }
        top = mn;
      }
      // R, below the running maximum (differences of scores are exact where their sums with exponents are not: scores may have no digits behind the point)
      const float t = top == -INFINITY ? 0.f : top;
      const float level = fmaxf(ceilf(fmaxf(fmaxf((w0 - t) + ev.x, (w1 - t) + ev.y), fmaxf((w2 - t) + ev.z, (w3 - t) + ev.w))), -3e38f);
      uint32_t u[R];
#pragma unroll
      for (int r = 0; r < R; r++) {
        const float d = x[r] - __shfl_sync(0xffffffffu, t, r), p = ex2(d);
        // a NaN scale of the values reaches the rows that see one of its tokens through their sum
        sum[r] += lost && x[r] != -INFINITY ? NAN : p;
        // (R and the exponent are whole numbers: their difference is exact)
        u[r] = __float2uint_rn(ex2(d + (exp_own - __shfl_sync(0xffffffffu, level, r))) * frac);
      }
#pragma unroll
      for (int half = 0; half < 2; half++)
        *reinterpret_cast<uint4*>(&pipe.p[half][4 * (32 * role + lane)]) = make_uint4(u[4 * half], u[4 * half + 1], u[4 * half + 2], u[4 * half + 3]);
      fence_async_smem();
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sy.p_full);

      // what a row's sums are worth, 2^R, times 2^60 where that is a number in all rows: small weights of small values would be below fp32's
      // range, and zeros
      const bool large = __any_sync(0xffffffffu, level > 60.f);
      const float unit = ex2(large ? level : level + 60.f);
      const float part_hi = large ? 1.52587890625e-5f : 1.3234889800848443e-23f, part_lo = large ? 2.3283064365386963e-10f : 2.0194839173657902e-28f;   // 2^-16, 2^-32, and those times 2^-60
      // the tile's sums: lane = channel
      bar_wait(sm, &sy.o_full, (uint32_t)i & 1u);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      {
        int y[4][8];
#pragma unroll
        for (int z = 0; z < 4; z++) tmem_ld8(tmem + O_COL + 8u * z + lanes, y[z]);
        tmem_wait_ld();
#pragma unroll
        for (int r = 0; r < R; r++) {
          const int* d = &y[r >> 1][4 * (r & 1)];
          const float y2 = fmaf((float)(d[3] * 256 + d[2]), part_hi, (float)(d[1] * 256 + d[0]) * part_lo);
          o[r] = fmaf(y2, __shfl_sync(0xffffffffu, unit, r), o[r]);
        }
      }
      fresh = last;
      if (last && !CLUSTER) {
        lane_sums(sum, sy.sum[role], lane);
        asm volatile("bar.sync %0, 128;\n" ::"r"(1 + g) : "memory");
        const bool ends = cur.ended, direct = whole && ends;
        float* slot = a.slots + (size_t)(2 * v + (began ? 0 : 1)) * SLOT;
        if (!began && (heads.by_item || !ends) && tid == g * 128)   // (the same thread as above)
          a.heads[heads.at(v, c.n_kv, li * c.batch + bq, h, rt)] = Head{ends ? 0 : cuts.range_of(item_end) - v, v, li * c.batch + bq, h, rt, {}};
#pragma unroll
        for (int r = 0; r < R; r++) {
          float l = (sy.sum[0][r] + sy.sum[1][r]) + (sy.sum[2][r] + sy.sum[3][r]);
          if (sm.abort) l = NAN;
          if (direct) {
            if (r < rows) out_row<T>(a, li, bq, h, R * rt + r)[ch] = from_f<T>(l == 0.f ? 0.f : o[r] / l);
          } else {
            slot[r * D + ch] = o[r];
            if (ch == r) { slot[R * D + r] = top; slot[R * D + R + r] = l; }
          }
        }
        whole = true;
        began = false;
      }
    }
    if (CLUSTER) {   // this pipeline's part, in the place of its first tile: all of its copies and products are through
      lane_sums(sum, sy.sum[role], lane);
      asm volatile("bar.sync %0, 128;\n" ::"r"(1 + g) : "memory");
      float* part = reinterpret_cast<float*>(pipe.k[0]);
#pragma unroll
      for (int r = 0; r < R; r++) {
        part[r * D + ch] = o[r];
        if (ch == r) {
          const float l = (sy.sum[0][r] + sy.sum[1][r]) + (sy.sum[2][r] + sy.sum[3][r]);
          part[R * D + r] = top;
          part[R * D + R + r] = sm.abort ? NAN : l;
        }
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (tid == 0 && sm.abort) set_status(c.status, OKQ_ERR_TIMEOUT);
  if (warp == 0 && !sm.tmem_busy) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(sm.tmem_slot), "n"(COLS) : "memory");
  if (!CLUSTER) return;
  // the item's rows dealt over the cluster's blocks, 128 threads (channels) to a row
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  // (pipeline i of every block by threads 128 i .. 128 i + 127: all loads of a row in flight at once)
  const int ch = tid & 127, pi = tid >> 7;
  float* mine = reinterpret_cast<float*>(sm.pipe[pi < G ? pi : 0].p);
  bool arrived = false;
  for (int r = rank; r < rows; r += size) {
    if (pi < G) {
      float t[MOST_CLUSTER], l[MOST_CLUSTER], o[MOST_CLUSTER];
      const uint32_t here = smem_u32(sm.pipe[pi].k[0]);
#pragma unroll
      for (int k = 0; k < MOST_CLUSTER; k++) {
        t[k] = -INFINITY;
        l[k] = o[k] = 0.f;
        if (k < size) {
          uint32_t there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(there) : "r"(here), "r"(k));
          asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(t[k]) : "r"(there + 4 * (R * D + r)));
          asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(l[k]) : "r"(there + 4 * (R * D + R + r)));
          asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(o[k]) : "r"(there + 4 * (r * D + ch)));
        }
      }
      float top = t[0], ls = 0.f, os = 0.f;
#pragma unroll
      for (int k = 1; k < MOST_CLUSTER; k++) top = fmaxf(top, t[k]);
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int k = 0; k < MOST_CLUSTER; k++) {
        if (falls(t[k], ref)) { t[k] += LATE_BITS; l[k] *= LATE; o[k] *= LATE; }
        const float f = ex2(t[k] - ref);
        ls = fmaf(l[k], f, ls);
        os = fmaf(o[k], f, os);
      }
      mine[ch] = os;
      if (ch == 0) { mine[D] = top; mine[D + 1] = ls; }
    }
    __syncthreads();
    if (r + size >= rows) {   // this block has read all that it needs of the others
      asm volatile("barrier.cluster.arrive.aligned;\n" ::: "memory");
      arrived = true;
    }
    if (pi == 0) {
      float top = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
      for (int g2 = 0; g2 < G; g2++) top = fmaxf(top, reinterpret_cast<const float*>(sm.pipe[g2].p)[D]);
      if (top == -INFINITY) top = 0.f;
#pragma unroll
      for (int g2 = 0; g2 < G; g2++) {
        const float* y = reinterpret_cast<const float*>(sm.pipe[g2].p);
        const float late = falls(y[D], top) ? LATE : 1.f, f = ex2(y[D] - top + (late == LATE ? LATE_BITS : 0.f));
        l = fmaf(y[D + 1] * late, f, l);
        o = fmaf(y[ch] * late, f, o);
      }
      out_row<T>(a, cur.li, cur.b, cur.h, R * cur.rt + r)[ch] = from_f<T>(l == 0.f ? 0.f : o / l);
    }
    __syncthreads();
  }
  if (!arrived) asm volatile("barrier.cluster.arrive.aligned;\n" ::: "memory");
  asm volatile("barrier.cluster.wait.aligned;\n" ::: "memory");   // no block ends while its parts are read
}

template <class T, bool CLUSTER, int SIGHT> cudaError_t launch(const AttnArgs& a, const CUtensorMap& map, dim3 grid, int size, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  int dev = 0;
  constexpr int SMEM = (int)sizeof(DecodeSmem) + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory of one block");
  if (attr_needed(attr_mask, dev)) {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_decode<T, CLUSTER, SIGHT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    attr_done(attr_mask, dev);
  }
  cudaError_t e = launch_dependent(k_paged_decode<T, CLUSTER, SIGHT>, grid, NT, SMEM, s, CLUSTER ? size : 1, map, a, size);
  if (e != cudaSuccess || CLUSTER) return e;
  const int ranges = G * (int)grid.x, rows = a.n_new * a.c.group;
  const Heads<R> heads(a.layer_count * a.c.batch, a.c.n_kv, a.c.group, a.n_new, ranges);
  return launch_dependent(k_paged_merge<T, R>, dim3(heads.count(ranges), rows < R ? rows : R), MERGE_NT, 0, s, 1, a);
}

template <int SIGHT> cudaError_t launch_sight(const AttnArgs& a, const CUtensorMap& map, int dtype, int blocks, int cluster, cudaStream_t s) {
  if (cluster > 0) {
    const dim3 grid((unsigned)cluster * (unsigned)((a.n_new * a.c.group + R - 1) / R), (unsigned)a.c.n_kv, (unsigned)(a.layer_count * a.c.batch));
    return dtype == OKQ_FP16 ? launch<__half, true, SIGHT>(a, map, grid, cluster, s) : launch<__nv_bfloat16, true, SIGHT>(a, map, grid, cluster, s);
  }
  return dtype == OKQ_FP16 ? launch<__half, false, SIGHT>(a, map, dim3(blocks), 1, s) : launch<__nv_bfloat16, false, SIGHT>(a, map, dim3(blocks), 1, s);
}

}  // namespace

// clusters of `size` blocks that the current device holds at once
int decode_clusters(int size) {
  static thread_local int known_dev = -1, known[MOST_CLUSTER + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
  if (dev != known_dev) {
    for (int k = 1; k <= MOST_CLUSTER; k++) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(k);
      cfg.blockDim = dim3(NT);
      cfg.dynamicSmemBytes = sizeof(DecodeSmem) + 1024;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = k; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      known[k] = 0;
      if (cudaFuncSetAttribute(k_paged_decode<__half, true, CAUSAL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes) != cudaSuccess ||
          cudaOccupancyMaxActiveClusters(&known[k], k_paged_decode<__half, true, CAUSAL>, &cfg) != cudaSuccess)
        (void)cudaGetLastError();
    }
    known_dev = dev;
  }
  return known[size];
}

cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, Sight sight, int blocks, int cluster, cudaStream_t s) {
  CUtensorMap map;
  if (!codes_map(map, a.c, true)) return cudaErrorInvalidValue;
  if (sight == WINDOW) return launch_sight<WINDOW>(a, map, dtype, blocks, cluster, s);
  if (sight == TREE) return launch_sight<TREE>(a, map, dtype, blocks, cluster, s);
  return launch_sight<CAUSAL>(a, map, dtype, blocks, cluster, s);
}

}  // namespace okq
