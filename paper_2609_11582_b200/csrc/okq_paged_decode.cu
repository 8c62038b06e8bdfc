// Attention over the 8-bit paged cache for up to eight query rows per (layer, sequence, KV head): single tokens, and a few drafted
// ones where the GQA group is small.
//
// All products are of 8-bit integers on tcgen05 (kind::i8), with the cache's codes as they lie in memory for one operand:
//   scores   S[token][row] = K[token][channel] Q[row][channel]: A = a tile of 128 tokens (K-major), B = the queries as three signed
//            limbs of a 24-bit fixed-point number (per row: q / max|q| * 127 * 2^16), exact sums in int32
//   values   O[channel][row] = V[token][channel] P[token][row]: A = the tile transposed by its descriptor (MN-major), B = the numerators
//            p * scale_v as the four bytes of a 32-bit fixed-point number, exact sums in int32
// so nothing is unpacked: a tile goes from memory to shared memory by TMA and from there into the tensor cores.  Fixed point is
// relative to the largest numerator so far; what lies more than 2^-32 below it is lost, fp32 would keep 2^-24 of each.
//
// Roles, meeting at mbarriers: a loader warp (ring of NS tiles, 32-token blocks by page), an MMA warp, four softmax warps (lane =
// token: running maximum, numerators, sums), four output warps (lane = channel: the item's sums in fp32 registers), four query warps
// (rotation and limbs of the next item while this one runs).
//
// Bound by memory: 256 bytes per token and head; an SM's share of the copy rate is a tile in about 1400 cycles, the longest role
// needs about half of that.
#include "okq_paged_attn.cuh"
#include "okq_tc.cuh"

namespace okq {

namespace {

constexpr int R = DECODE_ROWS;
constexpr int NS = 6;                     // ring of tiles
constexpr int SIDE = PT * D;              // bytes of a tile's keys or values
constexpr int W_OUT = 4, W_Q = 8, W_LOAD = 12, W_MMA = 13;
constexpr int NT = 14 * 32;
constexpr uint32_t S_COL = 0, O_COL = 64, COLS = 128;   // two buffers of 32 columns each
constexpr size_t SLOT = (size_t)R * (D + 2);

struct Factors {
  float out;          // what a unit of the 32-bit numerators stands for
  float keep[R];      // what the sums so far are multiplied by
  int moved;          // whether any of them is not 1
};

struct DecodeSmem {
  __align__(1024) int8_t k[NS][SIDE];
  __align__(1024) int8_t v[NS][SIDE];
  __align__(1024) int8_t q[2][32 * D];         // rows limb * 8 + row, 128-byte swizzle
  __align__(1024) uint32_t p[2][2][PT * 4];    // [half of the rows][token][row of the half]
  __align__(16) float wmax[2][4][R];
  __align__(16) float qscale[2][R];
  __align__(16) float sum[2][4][R];            // an item's normalisers, by softmax warp
  __align__(16) float top[2][R];
  Factors fac[2];
  float scale[NS][8];                          // of the tile's four blocks: keys, values
  __align__(8) unsigned long long full[NS], empty[NS];
  __align__(8) unsigned long long s_full[2], s_free[2], p_full[2], o_full[2], o_free[2], q_full[2], q_free[2];
  FindSmem find;
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

template <class T>
__global__ void __launch_bounds__(NT, 1) k_paged_decode(const __grid_constant__ CUtensorMap map, const AttnArgs a, long long wait_limit) {
  extern __shared__ unsigned char raw_smem[];
  DecodeSmem& sm = *reinterpret_cast<DecodeSmem*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    auto init = [](unsigned long long* b, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(b)), "r"(count)); };
    for (int i = 0; i < NS; i++) { init(&sm.full[i], 1); init(&sm.empty[i], 1); }
    for (int i = 0; i < 2; i++) {
      init(&sm.s_full[i], 1); init(&sm.s_free[i], 4);
      init(&sm.p_full[i], 4);
      init(&sm.o_full[i], 1); init(&sm.o_free[i], 4);
      init(&sm.q_full[i], 4); init(&sm.q_free[i], 5);
    }
    sm.abort = 0;
    sm.tmem_busy = 0;
    sm.limit = wait_limit;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&sm.tmem_slot)), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  for (int i = tid; i < 2 * 32 * D / 16; i += NT) reinterpret_cast<uint4*>(sm.q)[i] = make_uint4(0u, 0u, 0u, 0u);   // (the fourth limb stays 0)
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = sm.tmem_slot;
  depend_wait();

  const PagedView& c = a.c;
  const Work<R> work(a);
  Cursor<R> cur;
  long long g0, per = 1;
  find_place<R, NT>(sm.find, work, [&](long long total) { per = tiles_per_block(total, gridDim.x); return (long long)blockIdx.x * per; }, cur, g0);
  const long long rest = sm.find.total - g0;
  const int n_my = cur.pair >= work.pairs ? 0 : (int)(rest < per ? rest : per);

  if (warp == W_LOAD) {
    // ------------------------------------------------------------------ loader: eight tiles' blocks at a time, a lane for each, one batch ahead
    auto look = [&](int n) {   // the next n tiles
      int t = 0, len = 0, pair = 0, h = 0;
      for (int i = 0; i < n; i++) {
        if (lane >> 2 == i) { t = cur.tile * PT + PB * (lane & 3); len = cur.len; pair = cur.pair; h = cur.h; }
        cur.next(work);
      }
      Block x{-1, 0.f, 0.f};
      if (lane >> 2 < n && t < len) {
        const int l = a.layer + pair / c.batch, page = c.page_of(pair % c.batch, t);
        if (page < 0) {
          x = Block{-2, NAN, NAN};
          set_status(c.status, OKQ_ERR_INVALID_ARG);
        } else {
          const size_t row = c.code_row(l, page, h, 0) + (t & (c.page - 1));
          x = Block{(int)row, __ldg(&c.scales[row / PB]), __ldg(&c.scales[(row + c.page) / PB])};
        }
      }
      return x;
    };
    int armed = 0;
    Block nxt{-1, 0.f, 0.f};
    if (n_my > 0) nxt = look(min(8, n_my));
    for (int i0 = 0; i0 < n_my; i0 += 8) {
      const Block x = nxt;
      const int n = min(8, n_my - i0);
      if (i0 + 8 < n_my) nxt = look(min(8, n_my - i0 - 8));
      bool out = false;
      for (int k = 0; k < n; k++) {
        const int i = i0 + k, s = i % NS;
        if (i >= NS && !mbar_wait(sm, &sm.empty[s], (uint32_t)(i / NS - 1) & 1u)) { out = true; break; }
        const bool mine = lane >> 2 == k, there = mine && x.row >= 0;
        if (mine) { sm.scale[s][lane & 3] = x.ks; sm.scale[s][4 + (lane & 3)] = x.vs; }
        const int blocks = __popc(__ballot_sync(0xffffffffu, there));
        const uint32_t bar = smem_u32(&sm.full[s]);
        __syncwarp();   // the scales are written before the arrival
        if (lane == 0)
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(blocks * 2 * PB * D) : "memory");
        __syncwarp();
        if (there) {
          const int j = lane & 3;
#pragma unroll
          for (int side = 0; side < 2; side++)
            asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                         ::"r"(smem_u32(side ? sm.v[s] : sm.k[s]) + j * PB * D), "l"(reinterpret_cast<uint64_t>(&map)), "r"(0),
                           "r"(x.row + side * c.page), "r"(bar) : "memory");
        }
        armed = i + 1;
      }
      if (out) break;
    }
    if (sm.abort || armed < n_my)   // no copy may still be landing when the block ends
      for (int i = max(0, armed - NS); i < armed; i++) mbar_drain(&sm.full[i % NS], (uint32_t)(i / NS) & 1u);
  } else if (warp == W_MMA) {
    // ------------------------------------------------------------------ products: scores of tile i, then values of tile i - 1
    constexpr uint32_t shape = (2u << 4) | ((32u >> 3) << 17) | (((uint32_t)PT >> 4) << 24);   // D int32, N 32, M 128
    constexpr uint32_t id_s = shape | (1u << 7) | (1u << 10);                                  // A, B signed, K-major
    constexpr uint32_t id_o = shape | (1u << 7) | (1u << 15) | (1u << 16);                     // A signed, B unsigned, both MN-major
    int items = 0, scored = 0, done = 0;
    for (int i = 0; i <= n_my; i++) {
      if (i < n_my) {
        const int s = i % NS, b = i & 1;
        const bool fresh = i == 0 || cur.tile == 0;
        if (fresh) {
          if (!mbar_wait(sm, &sm.q_full[items & 1], (uint32_t)(items >> 1) & 1u)) break;
          items++;
        }
        cur.next(work);
        const bool last = i + 1 == n_my || cur.tile == 0;
        if (!mbar_wait(sm, &sm.full[s], (uint32_t)(i / NS) & 1u)) break;
        if (i >= 2 && !mbar_wait(sm, &sm.s_free[b], (uint32_t)((i >> 1) - 1) & 1u)) break;
        if (elect_one()) {
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint64_t ad = make_desc_sw128(smem_u32(sm.k[s])), bd = make_desc_sw128(smem_u32(sm.q[(items - 1) & 1]));
#pragma unroll
          for (int k = 0; k < 4; k++) mma_i8(tmem + S_COL + 32u * b, ad + 2u * k, bd + 2u * k, id_s, k != 0);
          if (last) commit(&sm.q_free[(items - 1) & 1]);
          commit(&sm.s_full[b]);
        }
        __syncwarp();
        scored = i + 1;
      }
      if (i >= 1) {
        const int j = i - 1, s = j % NS, b = j & 1;
        if (!mbar_wait(sm, &sm.p_full[b], (uint32_t)(j >> 1) & 1u)) break;
        if (j >= 2 && !mbar_wait(sm, &sm.o_free[b], (uint32_t)((j >> 1) - 1) & 1u)) break;
        if (elect_one()) {
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint64_t ad = make_desc_sw128(smem_u32(sm.v[s])), bd = make_desc(smem_u32(sm.p[b]), 128, PT * 16);
#pragma unroll
          for (int k = 0; k < 4; k++) mma_i8(tmem + O_COL + 32u * b, ad + 256u * k, bd + 32u * k, id_o, k != 0);   // 32 tokens further
          commit(&sm.empty[s]);
          commit(&sm.o_full[b]);
        }
        __syncwarp();
        done = i;
      }
    }
    // nothing may be in flight when tensor memory is released; if the last products do not answer, it stays allocated
    if (scored >= 1 && !mbar_drain(&sm.s_full[(scored - 1) & 1], (uint32_t)((scored - 1) >> 1) & 1u)) sm.tmem_busy = 1;
    if (done >= 1 && !mbar_drain(&sm.o_full[(done - 1) & 1], (uint32_t)((done - 1) >> 1) & 1u)) sm.tmem_busy = 1;
  } else if (warp >= W_Q) {
    // ------------------------------------------------------------------ queries: two rows per warp, four channels per lane
    const int wq = warp - W_Q;
    write_empty<T>(a, work, blockIdx.x * 4 + wq, gridDim.x * 4, lane);
    int items = 0;
    for (int i = 0; i < n_my; items++) {
      const int qb = items & 1;
      if (items >= 2) mbar_wait(sm, &sm.q_free[qb], (uint32_t)((items >> 1) - 1) & 1u);
      const int li = cur.pair / c.batch, b = cur.pair % c.batch;
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const int r = 2 * wq + e, row = cur.rt * R + r, qi = row / c.group;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        const bool there = row < cur.m * c.group;
        if (there) {
          const T* src = static_cast<const T*>(a.q.p) + li * a.q.s[0] + b * a.q.s[1] + (cur.h * c.group + row % c.group) * a.q.s[2] + qi * a.q.s[3];
          const uint2 raw = *reinterpret_cast<const uint2*>(src + 4 * lane);
          const T* y = reinterpret_cast<const T*>(&raw);
#pragma unroll
          for (int z = 0; z < 4; z++) x[z] = to_f(y[z]);
        }
        if (a.rope.freq) {
          const int step = a.rope.half >> 2, turns = lane < 2 * step, low = lane < step;   // lanes from a channel to its partner
          const int other = !turns ? lane : low ? lane + step : lane - step, pair0 = 4 * (low ? lane : lane - step);
#pragma unroll
          for (int z = 0; z < 4; z++) {
            const float y = __shfl_sync(0xffffffffu, x[z], other);
            if (turns && there) {
              const size_t st = (size_t)c.batch * a.n_new;
              float cs, sn, u = low ? x[z] : y, w2 = low ? y : x[z];
              turn((double)a.rope.positions[a.rope.axis(pair0 + z) * st + (size_t)b * a.n_new + qi] * a.rope.freq[pair0 + z], cs, sn);
              rotate_pair(u, w2, cs, sn);
              x[z] = to_f(from_f<T>(low ? u : w2));
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
        const float f = fine ? 8323072.f / big : 0.f;
        uint32_t limb[3] = {0u, 0u, 0u};
#pragma unroll
        for (int z = 0; z < 4; z++) {
          int v = fine ? __float2int_rn(x[z] * f) : 0;
#pragma unroll
          for (int n = 0; n < 3; n++) {
            const int d = (int)(signed char)(v & 0xff);
            limb[n] |= (uint32_t)(d & 0xff) << (8 * z);
            v = (v - d) >> 8;
          }
        }
#pragma unroll
        for (int n = 0; n < 3; n++) {
          const int line = 8 * n + r;
          *reinterpret_cast<uint32_t*>(sm.q[qb] + line * D + (((lane >> 2) ^ (line & 7)) << 4) + ((4 * lane) & 15)) = limb[n];
        }
        if (lane == 0) sm.qscale[qb][r] = mx >= 0x7f800000u ? NAN : big / 8323072.f * a.scale2;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[qb]);
      i += cur.nt - cur.tile;
      cur.next_item(work);
    }
  } else if (warp < W_OUT) {
    // ------------------------------------------------------------------ softmax: lane = token
    const uint32_t lanes = (uint32_t)(32 * warp) << 16;
    float top[R], sum[R], qs[R];
    int items = 0;
    bool fresh = true;
    for (int i = 0; i < n_my; i++) {
      const int b = i & 1, s = i % NS;
      const int tile = cur.tile, len = cur.len, m = cur.m, rt = cur.rt;
      cur.next(work);
      const bool last = i + 1 == n_my || cur.tile == 0;
      mbar_wait(sm, &sm.full[s], (uint32_t)(i / NS) & 1u);   // (long complete: for the loader's scales and the query warps')
      if (fresh) mbar_wait(sm, &sm.q_full[items & 1], (uint32_t)(items >> 1) & 1u);
      mbar_wait(sm, &sm.s_full[b], (uint32_t)(i >> 1) & 1u);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      int d0[8], d1[8], d2[8];
      tmem_ld8(tmem + S_COL + 32u * b + lanes, d0);
      tmem_ld8(tmem + S_COL + 32u * b + 8u + lanes, d1);
      tmem_ld8(tmem + S_COL + 32u * b + 16u + lanes, d2);
      if (fresh) {
#pragma unroll
        for (int r = 0; r < R; r++) { qs[r] = sm.qscale[items & 1][r]; top[r] = -INFINITY; sum[r] = 0.f; }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.q_free[items & 1]);
      }
      // scales of this warp's block of 32 tokens; the largest value scale of the tile
      const float ks = sm.scale[s][warp], vs = sm.scale[s][4 + warp];
      const float vref = fmaxf(fmaxf(sm.scale[s][4], sm.scale[s][5]), fmaxf(sm.scale[s][6], sm.scale[s][7]));
      tmem_wait_ld();
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.s_free[b]);
      float x[R];
#pragma unroll
      for (int r = 0; r < R; r++) x[r] = fmaf((float)d2[r], 65536.f, (float)(d1[r] * 256 + d0[r])) * (qs[r] * ks);
      const int t = tile * PT + 32 * warp + lane;
      const bool edge = tile * PT + PT > len - m + 1;   // (some row does not see all of the tile)
      if (edge) {
#pragma unroll
        for (int r = 0; r < R; r++)
          if (t >= len - m + 1 + (rt * R + r) / c.group) x[r] = -INFINITY;
      }
      {
        float4* to = reinterpret_cast<float4*>(sm.wmax[b][warp]);
        float w[R];
#pragma unroll
        for (int r = 0; r < R; r++) w[r] = warp_max(x[r]);
        if (lane == 0) {
          to[0] = make_float4(w[0], w[1], w[2], w[3]);
          to[1] = make_float4(w[4], w[5], w[6], w[7]);
        }
      }
      asm volatile("bar.sync 1, 128;\n" ::: "memory");
      bool moved = false;
      float keep[R];
#pragma unroll
      for (int r = 0; r < R; r++) {
        const float mn = fmaxf(fmaxf(fmaxf(sm.wmax[b][0][r], sm.wmax[b][1][r]), fmaxf(sm.wmax[b][2][r], sm.wmax[b][3][r])), top[r]);
        moved |= mn > top[r];
        keep[r] = mn > top[r] ? ex2(top[r] - mn) : 1.f;
        top[r] = mn;
      }
      const float ratio = vref > 0.f ? vs / vref : 0.f;
      uint32_t u[R];
#pragma unroll
      for (int r = 0; r < R; r++) {
        float p = ex2(x[r] - (top[r] == -INFINITY ? 0.f : top[r]));
        // a NaN scale of the values reaches the rows that see one of its tokens through their sum
        const float ps = vs != vs && x[r] != -INFINITY ? NAN : p;
        sum[r] = moved ? fmaf(sum[r], keep[r], ps) : sum[r] + ps;
        u[r] = __float2uint_rn(p * ratio * 4294967040.f);   // (largest fp32 number below 2^32)
      }
      // numerators and factors of two tiles ago: read by their product and by the output warps
      if (i >= 2) mbar_wait(sm, &sm.o_free[b], (uint32_t)((i >> 1) - 1) & 1u);
#pragma unroll
      for (int half = 0; half < 2; half++)
        *reinterpret_cast<uint4*>(&sm.p[b][half][4 * (32 * warp + lane)]) = make_uint4(u[4 * half], u[4 * half + 1], u[4 * half + 2], u[4 * half + 3]);
      if (tid == 0) {
        Factors& f = sm.fac[b];
        f.out = vref > 0.f ? vref * (1.f / 4294967040.f) : 0.f;
        f.moved = moved && !fresh;
#pragma unroll
        for (int r = 0; r < R; r++) f.keep[r] = keep[r];
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.p_full[b]);
      fresh = last;
      if (last) {
#pragma unroll
        for (int r = 0; r < R; r++) {
          float v = sum[r];
#pragma unroll
          for (int w = 16; w >= 1; w >>= 1) v += __shfl_xor_sync(0xffffffffu, v, w);
          if (lane == r) { sm.sum[items & 1][warp][r] = v; if (warp == 0) sm.top[items & 1][r] = top[r]; }
        }
        asm volatile("bar.sync 2, 256;\n" ::: "memory");   // the output warps may read them; they are written again two items later
        items++;
      }
    }
  } else {
    // ------------------------------------------------------------------ sums: lane = channel
    const int wo = warp - W_OUT, ch = 32 * wo + lane;
    const uint32_t lanes = (uint32_t)(32 * wo) << 16;
    float o[R];
#pragma unroll
    for (int r = 0; r < R; r++) o[r] = 0.f;
    int items = 0;
    bool whole = cur.tile == 0, began = cur.tile != 0;   // the piece has its item's first tile; the item began in an earlier block
    for (int i = 0; i < n_my; i++) {
      const int b = i & 1;
      const int pair = cur.pair, h = cur.h, rt = cur.rt, m = cur.m;
      cur.next(work);
      const bool last = i + 1 == n_my || cur.tile == 0, ends = cur.tile == 0;
      mbar_wait(sm, &sm.p_full[b], (uint32_t)(i >> 1) & 1u);
      const float f = sm.fac[b].out;
      if (sm.fac[b].moved) {
#pragma unroll
        for (int r = 0; r < R; r++) o[r] *= sm.fac[b].keep[r];
      }
      mbar_wait(sm, &sm.o_full[b], (uint32_t)(i >> 1) & 1u);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      int y[4][8];
#pragma unroll
      for (int z = 0; z < 4; z++) tmem_ld8(tmem + O_COL + 32u * b + 8u * z + lanes, y[z]);
      tmem_wait_ld();
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.o_free[b]);
#pragma unroll
      for (int r = 0; r < R; r++) {
        const int* d = &y[r >> 1][4 * (r & 1)];
        o[r] = fmaf(fmaf((float)(d[3] * 256 + d[2]), 65536.f, (float)(d[1] * 256 + d[0])), f, o[r]);
      }
      if (last) {
        asm volatile("bar.sync 2, 256;\n" ::: "memory");
        const int ib = items & 1;
        const bool direct = whole && ends;
        float* slot = a.slots + (size_t)(2 * blockIdx.x + (began ? 0 : 1)) * SLOT;
#pragma unroll
        for (int r = 0; r < R; r++) {
          float l = (sm.sum[ib][0][r] + sm.sum[ib][1][r]) + (sm.sum[ib][2][r] + sm.sum[ib][3][r]);
          if (sm.abort) l = NAN;
          if (direct) {
            if (rt * R + r < m * c.group) out_row<T>(a, pair, h, rt * R + r)[ch] = from_f<T>(l == 0.f ? 0.f : o[r] / l);
          } else {
            slot[r * D + ch] = o[r];
            if (ch == 0) { slot[R * D + r] = sm.top[ib][r]; slot[R * D + R + r] = l; }
          }
          o[r] = 0.f;
        }
        items++;
        whole = true;
        began = false;
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (tid == 0 && sm.abort) set_status(c.status, OKQ_ERR_TIMEOUT);
  if (warp == 0 && !sm.tmem_busy) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(COLS) : "memory");
}

constexpr int MERGE_NT = 256;

template <class T> cudaError_t launch(const AttnArgs& a, const CUtensorMap& map, int grid, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  int dev = 0;
  constexpr int SMEM = (int)sizeof(DecodeSmem) + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory of one block");
  if (attr_needed(attr_mask, dev)) {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_decode<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    attr_done(attr_mask, dev);
  }
  cudaError_t e = launch_dependent(k_paged_decode<T>, dim3(grid), NT, SMEM, s, 1, map, a, WAIT_LIMIT_CLOCKS);
  if (e == cudaSuccess && grid > 1) e = launch_dependent(k_paged_merge<T, R, MERGE_NT>, dim3(grid - 1), MERGE_NT, 0, s, 1, a, grid);
  return e;
}

}  // namespace

cudaError_t launch_paged_decode(const AttnArgs& a, int dtype, int grid, cudaStream_t s) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return cudaErrorInvalidValue;
  CUtensorMap map;
  const PagedView& c = a.c;
  const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)c.n_layers * c.n_pages * c.n_kv * 2 * c.page}, str[1] = {(cuuint64_t)D};
  const cuuint32_t box[2] = {(cuuint32_t)D, (cuuint32_t)PB}, estr[2] = {1, 1};
  if (enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c.codes, dims, str, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  return dtype == OKQ_FP16 ? launch<__half>(a, map, grid, s) : launch<__nv_bfloat16>(a, map, grid, s);
}

}  // namespace okq
