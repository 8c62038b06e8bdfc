// Attention over the 8-bit paged cache for many query rows per (layer, sequence, KV head): prompts, pieces of prompts,
// drafted tokens.  Causal against the end of the sequence.
//
// Both products are fp16 on tcgen05 (kind::f16, fp32 accumulation in tensor memory):
//   S[row][token] = Q[row][channel] K[token][channel]   the cache's codes are fp16 numbers as they are (|code| <= 127); queries are scaled
//                                                       to a power of two per row, so that bf16 ones are fp16 numbers too
//   O[row][channel] += P[row][token] V[token][channel]  P = 2^14 p w in fp16, in place of the scores in tensor memory, with
//                                                       w the value scale of the token's block
// and the scales of the blocks enter where they cost nothing: those of the keys in the factor of the exponent, those of the values as
// log2(w) in its offset; the normaliser takes a block's sum divided by w.
// The reference m of the exponent is that of p w, row by row, not of p: fp16 numbers have room for what a row multiplies, whatever the
// weights of tokens without value and the values of tokens that it does not see.  m is set 6 above a step's maximum and moves when one
// passes it (log2 units): O is multiplied then, by the row's own threads (3 above: every other step of a drifting sequence).  It moves
// down, too, to 6 above the maximum of a step that lies 20 below it or more (14: three times as many multiplications where scores spread
// by 3, 306 us and not 284): sums in fp32 have room for that, numerators in fp16 have not.  So the largest numerator of a step is 2^-6 or
// more; 11 bits down to 2^-14, below that rounded to 2^-24.
//
// A block of threads has 256 rows, in two streams A and B of 128, and walks the tokens in steps of 64: a loader warp (32-token blocks
// by page, two tiles of 128 tokens ahead), four warps that turn codes into fp16 (0x6400 | (code + 128) is 1024 + 128 + code; the rest is
// one subtraction per two) in the layout of the products, to each stream an MMA warp (one for both was busy with waits and issue) and four
// softmax warps (lane = row).  A stream has two places for scores, so that the next step's are there when a softmax ends.  Where an item
// has no more than 128 rows (a dual item), both streams have the same ones: A takes the first 64 tokens of every tile, B the others, and
// their sums are put together at the end.
//
// At best bound by the exponentials (16 per cycle and SM: 2048 cycles for 256 x 128 scores) and the products (2048 cycles at fp16's
// rate).  What it takes is about 4200 (2048 queries x 28 heads on 8192 tokens 286 us a call, 736 TFLOP/s of products): a softmax warp's own
// chain of waits, tensor memory, maximum, exponentials and roundings, with two such warps on a scheduler and 128 registers to each (the
// maximum beside the exponentials, by last step's reference: 390 us, spills).
// Few rows (a dual item) are bound by the conversion, a step in 1500 cycles, a third of it waits and fences: 35 rows, 16 sequences x 4
// heads of up to 12345 tokens 50 us a call (a converting warp to every other step, with half of those waits but a ring that is then too
// short: 61).
#include "okq_paged_attn.cuh"

namespace okq {

namespace {

constexpr int R = PROMPT_ROWS, EXTRA = PROMPT_EXTRA, M = 128;         // rows of a block, of a stream
constexpr int PH = PT / 2;                      // tokens of a step
constexpr int SIDE = PT * D;                    // bytes of a tile's keys or values as codes
constexpr int Q_HALF = M * 128, KV_HALF = PH * 128;   // 64 channels in fp16, of a stream's queries and of a step's keys or values
constexpr int NR = 3;                           // ring of steps' keys, and values, in fp16
constexpr int W_CONV = 8, W_MMA = 12, W_LOAD = 14;   // (an MMA warp to each stream)
constexpr int NT = 15 * 32;
constexpr uint32_t S_COL = 0, O_COL = 256;      // + 128 per stream, + 64 per place for scores; numerators lie on its first half
constexpr size_t SLOT = (size_t)R * (D + 2);
constexpr float P_SHIFT = 14.f, LEAD = 6.f, DROP = 20.f;
// The reference stays above 2^-FALL of the row's largest numerator: with 127 * 2^14 and 2^20 tokens O stays below 2^126.
constexpr float FALL = 76.f;
constexpr float WIDE = 65536.f;                 // references beyond which a product's rounding shows
constexpr float NO_VALUE = -112.f;              // log2(w) of blocks without a value: they move m where nothing else is near
constexpr float LEAST_W = 1.9259299e-34f;       // 2^-112: scales below that count as 0 (the normaliser, tokens / w, is no number)

struct Info {            // of a tile, by block
  float ks[4];           // key scales
  float lw[4];           // log2 of w, and the shift
  float iw[4];           // 2^-14 / w
  int lost;              // blocks whose value scale is NaN, a bit for each; from bit 4 on those without a value
};

struct PromptSmem {
  __align__(1024) unsigned char q[2][2][Q_HALF];   // [stream][channels / 64]
  __align__(1024) unsigned char k[NR][2][KV_HALF];
  __align__(1024) unsigned char v[NR][2][KV_HALF];
  __align__(1024) int8_t code[2][2][SIDE];         // [keys, values][tile mod 2]
  __align__(16) Info info[4];
  __align__(8) unsigned long long code_full[2][2], code_free[2][2], info_full[4], k_free[NR], v_free[NR];
  __align__(8) unsigned long long s_full[2][2], p_full[2][2], o_full[2], q_full[2];   // [stream][place]
  // steps of keys, and values, that are in fp16, by converting warp: numbers and not phases, since a stream of a dual item looks at every
  // other step only and could take a phase for the one after the next
  __align__(8) volatile int done[2][2];
  float peak[2 * M];                               // [stream][row] maximum of the numerators so far, LEAD below the highest reference
  FindSmem<1> find;
  uint32_t tmem_slot;
  long long limit;
  volatile int abort;
  volatile int tmem_busy;
};

// MN-major operand, 128-byte swizzle: 64 channels by 8 tokens are 1024 bytes, the other 64 channels lie KV_HALF further
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3fff) | ((uint64_t)(KV_HALF >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, bool acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
               ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t at, uint64_t bd, uint32_t idesc, bool acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n"
               ::"r"(d), "r"(at), "l"(bd), "r"(idesc), "r"(acc ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void commit(unsigned long long* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
               : "=f"(r[0]),"=f"(r[1]),"=f"(r[2]),"=f"(r[3]),"=f"(r[4]),"=f"(r[5]),"=f"(r[6]),"=f"(r[7]),"=f"(r[8]),"=f"(r[9]),"=f"(r[10]),"=f"(r[11]),"=f"(r[12]),"=f"(r[13]),"=f"(r[14]),"=f"(r[15]),
                 "=f"(r[16]),"=f"(r[17]),"=f"(r[18]),"=f"(r[19]),"=f"(r[20]),"=f"(r[21]),"=f"(r[22]),"=f"(r[23]),"=f"(r[24]),"=f"(r[25]),"=f"(r[26]),"=f"(r[27]),"=f"(r[28]),"=f"(r[29]),"=f"(r[30]),"=f"(r[31])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n"
               ::"r"(taddr), "r"(r[0]),"r"(r[1]),"r"(r[2]),"r"(r[3]),"r"(r[4]),"r"(r[5]),"r"(r[6]),"r"(r[7]),"r"(r[8]),"r"(r[9]),"r"(r[10]),"r"(r[11]),"r"(r[12]),"r"(r[13]),"r"(r[14]),"r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
               : "=f"(r[0]),"=f"(r[1]),"=f"(r[2]),"=f"(r[3]),"=f"(r[4]),"=f"(r[5]),"=f"(r[6]),"=f"(r[7]),"=f"(r[8]),"=f"(r[9]),"=f"(r[10]),"=f"(r[11]),"=f"(r[12]),"=f"(r[13]),"=f"(r[14]),"=f"(r[15])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }

// four codes as two pairs of fp16 numbers
__device__ __forceinline__ uint2 codes_to_half(uint32_t w) {
  w ^= 0x80808080u;
  const __half2 bias = __floats2half2_rn(1152.f, 1152.f);
  uint32_t lo = __byte_perm(w, 0x64646464u, 0x4140), hi = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 a = __hsub2(*reinterpret_cast<__half2*>(&lo), bias), b = __hsub2(*reinterpret_cast<__half2*>(&hi), bias);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// The warps of streams A and B that share a scheduler work out their numerators in turn (both have equally many steps).  Left alone they
// fall into step, and each waits for the other's exponentials in that stretch and leaves the unit idle in the others.
__device__ __forceinline__ void take_turn(int id) { asm volatile("bar.sync %0, 64;\n" ::"r"(id) : "memory"); }
__device__ __forceinline__ void pass_turn(int id) { asm volatile("bar.arrive %0, 64;\n" ::"r"(id) : "memory"); }

// Wait of a warp until both converting warps have done step x, with the limit of every wait.
__device__ __forceinline__ bool step_ready(PromptSmem& sm, const volatile int* done, int x) {
  const uint32_t at = smem_u32(const_cast<const int*>(done));
  const long long t0 = clock64();
  bool ok = true;
  for (;;) {
    int a, b;
    asm volatile("ld.volatile.shared.v2.s32 {%0, %1}, [%2];\n" : "=r"(a), "=r"(b) : "r"(at) : "memory");
    if (a > x && b > x) break;
    if (sm.abort || clock64() - t0 > sm.limit) {
      ok = false;
      break;
    }
  }
  if (!ok) sm.abort = 1;
  __threadfence_block();
  return __all_sync(0xffffffffu, ok);
}

// The 32 rows of a warp in a row tile: rotated, scaled by a power of two, swizzled; returns the factor of the exponent that undoes the
// scaling for the lane's own row (times the softmax scale, whose sign goes to the queries).  Eight lanes to a row, sixteen channels each.
template <class T>
__device__ __forceinline__ float prepare_queries(const AttnArgs& a, const Cursor<R, EXTRA>& cur, int row0, unsigned char* q, bool store, int lane) {
  const PagedView& c = a.c;
  const int rows = cur.m * c.group;
  const int j = lane & 7, nc = a.rope.half >> 3;
  const bool turns = a.rope.freq && j < nc;
  const int c0 = !a.rope.freq || j < nc ? 8 * j : 2 * a.rope.half + 16 * (j - nc);
  const int c1 = !a.rope.freq ? c0 + 64 : j < nc ? c0 + a.rope.half : c0 + 8;
  float mine = 0.f;
#pragma unroll 2
  for (int it = 0; it < 8; it++) {
    const int rl = 4 * it + (lane >> 3), row = cur.rt * R + row0 + rl;    // row inside the warp, of the item's queries
    Vec8<T> x[2] = {};
    if (row < rows) {
      const T* src = query_row<T>(a, cur.li, cur.b, cur.h, row);
      x[0] = *reinterpret_cast<const Vec8<T>*>(src + c0);
      x[1] = *reinterpret_cast<const Vec8<T>*>(src + c1);
      if (turns) {
        float cs[8], sn[8];
        turns8(a.rope, a.rope.positions + (size_t)cur.b * a.n_new + c.query_of(row), (size_t)c.batch * a.n_new, c0, cs, sn);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          float u = to_f(x[0].v[e]), w = to_f(x[1].v[e]);
          rotate_pair(u, w, cs[e], sn[e]);
          x[0].v[e] = from_f<T>(u);
          x[1].v[e] = from_f<T>(w);
        }
      }
    }
    unsigned mx = 0;
#pragma unroll
    for (int e = 0; e < 16; e++) mx = max(mx, __float_as_uint(to_f(x[e >> 3].v[e & 7])) & 0x7fffffffu);
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    // 2^-e brings the largest magnitude to [1, 2) (4 at the end of the range); rows too small for that, and those with an infinity or NaN, are zeros here
    const int e2 = min((int)(mx >> 23) - 127, 126);
    const bool fine = mx < 0x7f800000u && e2 > -100;
    const float up = fine ? __uint_as_float((uint32_t)(127 - e2) << 23) * (a.scale2 < 0.f ? -1.f : 1.f) : 0.f;
    const float back = mx >= 0x7f800000u ? NAN : fine ? __uint_as_float((uint32_t)(127 + e2) << 23) * fabsf(a.scale2) : 0.f;
#pragma unroll
    for (int z = 0; z < 2; z++) {
      const int ch = z ? c1 : c0;
      __half2 y[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float u = to_f(x[z].v[2 * e]), w = to_f(x[z].v[2 * e + 1]);
        y[e] = __floats2half2_rn(fine ? u * up : 0.f, fine ? w * up : 0.f);
      }
      const int r = (row0 & (M - 1)) + rl;
      if (store) *reinterpret_cast<uint4*>(q + (ch >> 6) * Q_HALF + r * 128 + ((((ch & 63) >> 3) ^ (r & 7)) << 4)) = *reinterpret_cast<const uint4*>(y);
    }
    const float got = __shfl_sync(0xffffffffu, back, 8 * (lane & 3));    // rows 4 it .. 4 it + 3 are in lanes 0, 8, 16, 24
    if (lane >> 2 == it) mine = got;
  }
  return mine;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// The lane's row of a step's scores, two blocks of 32 tokens, b0 the tile's number of the first; `seen`: last column that the row sees.
// The largest log2 of p w, 2^P_SHIFT times.
template <bool EDGE>
__device__ __forceinline__ float row_max(float (&x)[2][32], const Info& info, int b0, float back, int seen) {
  float mx = -INFINITY;
#pragma unroll
  for (int b = 0; b < 2; b++) {
    if (EDGE) {
#pragma unroll
      for (int e = 0; e < 32; e++)
        if (32 * b + e > seen) x[b][e] = -INFINITY;
    }
    float y[4] = {x[b][0], x[b][1], x[b][2], x[b][3]};
#pragma unroll
    for (int e = 4; e < 28; e += 2) y[(e >> 1) & 3] = max3(y[(e >> 1) & 3], x[b][e], x[b][e + 1]);
    const float top = max3(max3(y[0], y[1], x[b][28]), max3(y[2], y[3], x[b][29]), fmaxf(x[b][30], x[b][31]));
    mx = fmaxf(mx, EDGE && top == -INFINITY ? top : EDGE ? __fadd_rn(__fmul_rn(top, back * info.ks[b0 + b]), info.lw[b0 + b]) : fmaf(top, back * info.ks[b0 + b], info.lw[b0 + b]));
  }
  return mx;
}
// EDGE also rounds a score once before the reference is taken off, as the maximum is: the difference is exact then, where scores are so
// large that an unrounded one could lie far above it (not by packed pairs: their product and sum were contracted to one rounding).  Blocks
// without a value count in the normaliser alone.
template <bool EDGE>
__device__ __forceinline__ float numerators(const float (&x)[2][32], uint32_t s_at, const Info& info, int b0, float back, float ref, int seen, float l) {
#pragma unroll
  for (int b = 0; b < 2; b++) {
    const bool none = EDGE && (info.lost >> (4 + b0 + b) & 1);
    const float cb = back * info.ks[b0 + b], lw = none ? 0.f : info.lw[b0 + b], off = lw - ref;
    const F2 cb2 = f2(cb, cb), off2 = f2(off, off);
    F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
    uint32_t u[16];
#pragma unroll
    for (int e = 0; e < 16; e++) {
      float2 z;
      if (EDGE) {
        const float most = none ? 127.f : P_SHIFT + 1.f;   // (lw may have no digit in the reference)
        z = make_float2(__fadd_rn(__fsub_rn(__fmul_rn(x[b][2 * e], cb), ref), lw), __fadd_rn(__fsub_rn(__fmul_rn(x[b][2 * e + 1], cb), ref), lw));
        z = make_float2(z.x > most ? most : z.x, z.y > most ? most : z.y);
      } else {
        z = un2(fma2(f2(x[b][2 * e], x[b][2 * e + 1]), cb2, off2));
      }
      float p0 = ex2(z.x), p1 = ex2(z.y);
      if (EDGE) {   // (-inf times a scale of zero is NaN)
        if (32 * b + 2 * e > seen) p0 = 0.f;
        if (32 * b + 2 * e + 1 > seen) p1 = 0.f;
      }
      sum[e & 1] = add2(sum[e & 1], f2(p0, p1));
      const __half2 h = __floats2half2_rn(p0, p1);
      u[e] = none ? 0u : *reinterpret_cast<const uint32_t*>(&h);
    }
    const float2 total = un2(add2(sum[0], sum[1]));
    l = fmaf(total.x + total.y, info.iw[b0 + b], l);
    if (EDGE && (info.lost >> (b0 + b) & 1) && 32 * b <= seen) l = NAN;
    tmem_st16(s_at + 16u * b, u);
  }
  return l;
}

template <class T>
__global__ void __launch_bounds__(NT, 1) k_paged_prompt(const __grid_constant__ CUtensorMap map, const AttnArgs a) {
  extern __shared__ unsigned char raw_smem[];
  PromptSmem& sm = *reinterpret_cast<PromptSmem*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    auto init = [](unsigned long long* b, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(b)), "r"(count)); };
    for (int i = 0; i < 4; i++) {
      init(&sm.code_full[0][0] + i, 1); init(&sm.code_free[0][0] + i, 2); init(&sm.info_full[i], 1);
      init(&sm.s_full[0][0] + i, 1); init(&sm.p_full[0][0] + i, 4);
    }
    for (int i = 0; i < NR; i++) { init(&sm.k_free[i], 2); init(&sm.v_free[i], 2); }
    for (int i = 0; i < 4; i++) sm.done[i >> 1][i & 1] = 0;
    for (int i = 0; i < 2; i++) { init(&sm.o_full[i], 1); init(&sm.q_full[i], 4); }
    sm.abort = 0;
    sm.tmem_busy = 0;
    sm.limit = a.limit;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&sm.tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  before_sync();
  __syncthreads();
  after_sync();
  const uint32_t tmem = sm.tmem_slot;
  depend_wait();

  const PagedView& c = a.c;
  const Work<R, EXTRA> work(a);
  const int v = blockIdx.x;                     // this block's range
  const Cuts cuts = find_places<R, EXTRA, NT, 1>(sm.find, work, gridDim.x, v, 0);
  const int end = cuts.start(v) + cuts.size(v); // the unit behind it
  const Heads<R> heads(work.pairs, c.n_kv, c.group, a.n_new, gridDim.x);
  Cursor<R, EXTRA> cur = place<R, EXTRA, 1>(sm.find, work, cuts, v, 0);

  if (warp == W_LOAD) {
    // ------------------------------------------------------------------ loader: blocks of the tiles to come, as in the decode kernel
    Cursor<R, EXTRA> ahead = cur;
    int n_now = 0, n_nx = 0;
    int t_nx = 0, l_nx = 0, h_nx = 0, page_nx = -1;
    bool in_nx = false;
    int row_now = -1, row_nx = -1;               // -1: nothing to copy
    float ks_now = 0.f, vs_now = 0.f, ks_nx = 0.f, vs_nx = 0.f;
    auto entries = [&] {
      int b = 0, len = 0;
      for (n_nx = 0; n_nx < 8 && ahead.ok; n_nx++) {
        if (lane >> 2 == n_nx) { t_nx = ahead.tile * PT + PB * (lane & 3); len = ahead.len; l_nx = a.layer + ahead.li; b = ahead.b; h_nx = ahead.h; }
        ahead.next(work);
      }
      in_nx = lane >> 2 < n_nx && t_nx < len;
      if (in_nx) page_nx = __ldcg(&c.table[(size_t)b * c.max_pages + (t_nx >> c.page_shift)]);
    };
    auto scales = [&] {
      row_nx = -1;
      ks_nx = vs_nx = 0.f;
      if (!in_nx) return;
      if ((unsigned)page_nx >= (unsigned)c.n_pages) {
        ks_nx = vs_nx = NAN;
        set_status(c.status, OKQ_ERR_INVALID_ARG);
      } else {
        const size_t row = c.code_row(l_nx, page_nx, h_nx, 0) + (t_nx & (c.page - 1));
        row_nx = (int)row;
        ks_nx = __ldcg(&c.scales[row / PB]);
        vs_nx = __ldcg(&c.scales[(row + c.page) / PB]);
      }
    };
    int armed[2] = {0, 0};
    bool out = a.withhold != 0;
    entries();
    scales();
    for (int i = 0; !out; i++) {
      const int k = i & 7;
      if (k == 0) {
        n_now = n_nx;
        row_now = row_nx; ks_now = ks_nx; vs_now = vs_nx;
        entries();
      }
      if (k >= n_now) break;
      const bool mine = lane >> 2 == k, there = mine && row_now >= 0;
      const int blocks = __popc(__ballot_sync(0xffffffffu, there)), j = lane & 3;
#pragma unroll
      for (int side = 0; side < 2; side++) {
        if (i >= 2 && !bar_wait(sm, &sm.code_free[side][i & 1], (uint32_t)((i >> 1) - 1) & 1u)) { out = true; break; }
        const uint32_t bar = smem_u32(&sm.code_full[side][i & 1]);
        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(blocks * PB * D) : "memory");
        __syncwarp();
        if (there)
          asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                       ::"r"(smem_u32(sm.code[side][i & 1]) + j * PB * D), "l"(reinterpret_cast<uint64_t>(&map)), "r"(0), "r"(row_now + side * c.page), "r"(bar) : "memory");
        armed[side] = i + 1;
      }
      if (out) break;
      // what the other roles need to know of the tile (tile i - 4, whose place it takes, is through: the values of tile i - 2 are in fp16,
      // so those of tile i - 4 have been used)
      const float vs = __shfl_sync(0xffffffffu, vs_now, 4 * k + j), ks = __shfl_sync(0xffffffffu, ks_now, 4 * k + j);
      Info& info = sm.info[i & 3];
      if (lane < 4) {
        info.ks[lane] = ks;
        info.lw[lane] = (vs >= LEAST_W ? log2f(vs) : NO_VALUE) + P_SHIFT;
        info.iw[lane] = vs >= LEAST_W ? 1.f / (vs * 16384.f) : 1.f;
      }
      const unsigned lost = __ballot_sync(0xffffffffu, lane < 4 && vs != vs), none = __ballot_sync(0xffffffffu, lane < 4 && !(vs >= LEAST_W));
      if (lane == 0) info.lost = (int)(lost | none << 4);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.info_full[i & 3]);
      if (k == 4) scales();
    }
    if (sm.abort || out)   // no copy may still be landing when the block ends
      for (int side = 0; side < 2; side++)
        for (int i = max(0, armed[side] - 2); i < armed[side]; i++) mbar_drain(&sm.code_full[side][i & 1], (uint32_t)(i >> 1) & 1u);
    write_empty<T>(a, work, heads, v, gridDim.x, lane);
  } else if (warp >= W_MMA) {
    // ------------------------------------------------------------------ products of stream t
    const int t = warp - W_MMA;
    constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(PH >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
    constexpr uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(M >> 4) << 24);   // B MN-major
    const uint32_t s_at = tmem + S_COL + 128u * t, o_at = tmem + O_COL + 128u * t;
    int items = 0, n_o = 0;                       // items so far, steps through
    uint32_t scored = 0, ph_s = 0, ph_p = 0;      // by place for scores, a bit each: whether any were issued; phases to come
    bool go = true;
    // A step's buffers are free when both streams are through with them; the one stream that uses a step of a dual item says so twice.
    auto score = [&](int x, int place, uint64_t ad, bool dual) {
      const int s = x % NR;
      if (!(go = go && step_ready(sm, sm.done[0], x))) return;
      if (elect_one()) {
        after_sync();
        const uint64_t bd = make_desc_sw128(smem_u32(sm.k[s][0]));
#pragma unroll
        for (int k = 0; k < 8; k++)
          mma_ss(s_at + 64u * place, ad + (uint64_t)(((k & 3) * 32 + (k >> 2) * Q_HALF) >> 4), bd + (uint64_t)(((k & 3) * 32 + (k >> 2) * KV_HALF) >> 4), id_s, k != 0);
        commit(&sm.s_full[t][place]);
        commit(&sm.k_free[s]);
        if (dual) commit(&sm.k_free[s]);
      }
      __syncwarp();
      scored |= 1u << place;
      ph_s ^= 1u << place;
    };
    for (int i = 0; cur.ok && go;) {
      const bool dual = cur.m * c.group - cur.rt * R <= M;        // both streams have the same rows
      const int n = cur.piece(), steps = dual ? n : 2 * n;
      const int x0 = 2 * i + (dual ? t : 0), dx = dual ? 2 : 1;   // step y is step x0 + dx y of the range
      const uint64_t ad = make_desc_sw128(smem_u32(sm.q[dual ? 0 : t][0]));
      go = bar_wait(sm, &sm.q_full[t], (uint32_t)(items++) & 1u);
      for (int y = 0; y < min(2, steps); y++) score(x0 + dx * y, y, ad, dual);
      for (int y = 0; y < steps && go; y++) {
        const int x = x0 + dx * y, s = x % NR, place = y & 1;
        if (!(go = go && bar_wait(sm, &sm.p_full[t][place], ph_p >> place & 1u) && step_ready(sm, sm.done[1], x))) break;
        ph_p ^= 1u << place;
        if (elect_one()) {
          after_sync();
          const uint64_t bd = make_desc_mn(smem_u32(sm.v[s][0]));
#pragma unroll
          for (int k = 0; k < 4; k++)   // 16 tokens further
            mma_ts(o_at, s_at + 64u * place + 8u * k, bd + (uint64_t)(k * 2048 >> 4), id_o, y > 0 || k != 0);
          commit(&sm.o_full[t]);
          commit(&sm.v_free[s]);
          if (dual) commit(&sm.v_free[s]);
        }
        __syncwarp();
        n_o++;
        if (y + 2 < steps) score(x + 2 * dx, place, ad, dual);
      }
      i += n;
      cur.skip(work, n);
    }
#pragma unroll
    for (int p = 0; p < 2; p++)
      if ((scored >> p & 1u) && !mbar_drain(&sm.s_full[t][p], (ph_s >> p & 1u) ^ 1u)) sm.tmem_busy = 1;
    if (n_o > 0 && !mbar_drain(&sm.o_full[t], (uint32_t)(n_o - 1) & 1u)) sm.tmem_busy = 1;
  } else if (warp >= W_CONV) {
    // ------------------------------------------------------------------ codes to fp16: eight lanes to a token, sixteen channels each
    // Two warps have the keys, two the values.  (Loads a step ahead: the moves between the registers cost a draft 5 %, a prompt gains 0.5.)
    // (of eight lanes four have the first 64 channels of token t and four the others of token t ^ 1, so that each store has all banks)
    const int side = (warp - W_CONV) >> 1, who = (warp - W_CONV) & 1, j = lane & 7, tok = ((32 * who + lane) >> 3) ^ (j >> 2);
    const uint32_t at = (uint32_t)((j >> 2) * KV_HALF + tok * 128), a0 = at + (((2 * (j & 3)) ^ tok) << 4), a1 = at + (((2 * (j & 3) + 1) ^ tok) << 4);
    int end_x = 0;
    auto there = [&](int x) {   // whether step x is the range's
      if (x == end_x && cur.ok) {
        const int n = cur.piece();
        end_x += 2 * n;
        cur.skip(work, n);
      }
      return x < end_x;
    };
    auto codes_of = [&](int x) { return sm.code[side][x >> 1 & 1] + ((x & 1) * PH + tok) * D + 16 * j; };
    uint4 w[8];
    auto fetch = [&](int x, uint4 (&to)[8]) {
      if (!(x & 1)) bar_wait(sm, &sm.code_full[side][x >> 1 & 1], (uint32_t)(x >> 2) & 1u);
#pragma unroll
      for (int z = 0; z < 8; z++) to[z] = *reinterpret_cast<const uint4*>(codes_of(x) + 8 * z * D);
    };
    for (int x = 0; there(x); x++) {
      const int i = x >> 1, half = x & 1, s = x % NR;
      fetch(x, w);
      if (x >= NR) bar_wait(sm, side ? &sm.v_free[s] : &sm.k_free[s], (uint32_t)(x / NR - 1) & 1u);
      unsigned char* to = side ? sm.v[s][0] : sm.k[s][0];
#pragma unroll
      for (int z = 0; z < 8; z++) {   // (no branch between the rows, so that their conversions overlap)
        const uint2 h[4] = {codes_to_half(w[z].x), codes_to_half(w[z].y), codes_to_half(w[z].z), codes_to_half(w[z].w)};
        *reinterpret_cast<uint4*>(to + a0 + 1024 * z) = make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
        *reinterpret_cast<uint4*>(to + a1 + 1024 * z) = make_uint4(h[2].x, h[2].y, h[3].x, h[3].y);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        asm volatile("st.release.cta.shared.s32 [%0], %1;\n" ::"r"(smem_u32(const_cast<const int*>(&sm.done[side][who]))), "r"(x + 1) : "memory");
        if (half) mbar_arrive(&sm.code_free[side][i & 1]);
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax: lane = row (after a timeout they run on, waits failing at once)
    const int t = warp >> 2, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16, s_at = tmem + S_COL + 128u * t + lanes, o_at = tmem + O_COL + 128u * t + lanes;
    uint32_t ph_s = 0;   // phases of s_full to come, by place
    int n_o = 0;
    bool whole = cur.tile == 0, began = cur.tile != 0;
    if (!heads.by_item && tid == 0) a.heads[v].more = 0;
    if (t) pass_turn(2 + quarter);   // stream A begins
    for (int i = 0; cur.ok;) {
      const int n = cur.piece(), rows = cur.m * c.group - cur.rt * R, item0 = end - cur.left - cur.tile;   // (the item's first unit)
      const bool ends = cur.tile + n == cur.nt, dual = rows <= M;
      const int row0 = (dual ? 0 : M * t) + 32 * quarter, row = row0 + lane, steps = dual ? n : 2 * n;
      // (the stream's own products of the item before are through)
      // (stream B of a dual item takes its rows' factors only: its place holds the item's statistics in the end)
      const float back = prepare_queries<T>(a, cur, row0, sm.q[t][0], !dual || t == 0, lane);
      fence_async_smem();
      if (dual) asm volatile("bar.sync 1, 256;\n" ::: "memory");   // stream A's queries are B's too
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[t]);
      float m = -INFINITY, l = 0.f;
      sm.peak[M * t + 32 * quarter + lane] = -INFINITY;
      {
        // (what the loop keeps in registers besides 64 scores: as little as can be)
        int seen = cur.len - cur.m + c.query_of(cur.rt * R + row) - cur.tile * PT - (dual ? PH * t : 0);   // last column of the step that the row sees
        int half = dual ? t : 0, tile = i;
        bool wide = false;
        for (int y = 0; y < steps; y++) {
          const uint32_t p_at = s_at + 64u * (y & 1);
          if (dual || !half) bar_wait(sm, &sm.info_full[tile & 3], (uint32_t)(tile >> 2) & 1u);
          const Info& info = sm.info[tile & 3];
          bar_wait(sm, &sm.s_full[t][y & 1], ph_s >> (y & 1) & 1u);
          ph_s ^= 1u << (y & 1);
          after_sync();
          float x[2][32];
          tmem_ld32(p_at, x[0]);
          tmem_ld32(p_at + 32u, x[1]);
          const bool edge = __any_sync(0xffffffffu, seen < PH - 1) || info.lost;
          tmem_wait_ld();
          const float mx = edge ? row_max<true>(x, info, 2 * half, back, seen) : row_max<false>(x, info, 2 * half, back, seen);
          // a new reference: the row's sums so far are multiplied, once their last product is through
          const float below = m - mx;   // (-inf for the first; inf or NaN for steps that the row does not see)
          if (__any_sync(0xffffffffu, fabsf(below - (DROP / 2 - P_SHIFT)) > DROP / 2 && below < FALL)) {
            float& peak = sm.peak[M * t + 32 * quarter + lane];
            const bool up = below < -P_SHIFT;
            if (l > 4e37f) l = 4e37f;   // (not infinite: weights of tokens without value, 2^100 above all others)
            float mn = up || (below > DROP - P_SHIFT && below < FALL && peak - mx < FALL) ? mx + (LEAD - P_SHIFT) : m;
            if (!up && !(l * ex2(m - mn) < 1e36f)) mn = m;
            const float g = mn != m ? ex2(0.5f * (m - mn)) : 1.f, f = g * g;   // (0 for the first)
            m = mn;
            if (up) peak = fmaxf(peak, mx);
            wide = __any_sync(0xffffffffu, fabsf(m) > WIDE && m > -INFINITY);   // (scores so large that their products' rounding shows)
            l = l * g * g;   // (in two steps: it may be as large as the square is small)
            if (y > 0) {
              bar_wait(sm, &sm.o_full[t], (uint32_t)(n_o + y - 1) & 1u);
              after_sync();
#pragma unroll 1
              for (int b = 0; b < 8; b++) {
                float o[16];
                tmem_ld16(o_at + 16u * b, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; e++) o[e] *= f;
                tmem_st16(o_at + 16u * b, reinterpret_cast<const uint32_t(&)[16]>(o));
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          if (!dual) take_turn(2 + 4 * t + quarter);
          l = edge || wide ? numerators<true>(x, p_at, info, 2 * half, back, ref, seen, l) : numerators<false>(x, p_at, info, 2 * half, back, ref, seen, l);
          if (!dual) pass_turn(2 + 4 * (t ^ 1) + quarter);
          tmem_wait_st();
          before_sync();
          __syncwarp();
          // Phases of o_full are told apart by one bit: the last but one is waited for while the last cannot be complete, since all that is
          // known without a wait is that the third last is.
          if (y > 0 && y + 1 == steps) bar_wait(sm, &sm.o_full[t], (uint32_t)(n_o + y - 1) & 1u);
          if (lane == 0) mbar_arrive(&sm.p_full[t][y & 1]);
          if (dual) {
            tile++;
            seen -= PT;
          } else {
            tile += half;
            half ^= 1;
            seen -= PH;
          }
        }
      }
      n_o += steps;
      bar_wait(sm, &sm.o_full[t], (uint32_t)(n_o - 1) & 1u);
      if (sm.abort) l = NAN;
      float f = 1.f, f_other = 0.f;
      if (dual) {
        const int r = 32 * quarter + lane;
        float2* stat = reinterpret_cast<float2*>(sm.q[1][0]);
        stat[M * t + r] = make_float2(m, l);
        before_sync();
        asm volatile("bar.sync 1, 256;\n" ::: "memory");   // both streams' sums are complete
        const float2 y = stat[M * (t ^ 1) + r];
        const float mn = fmaxf(m, y.x), at = mn == -INFINITY ? 0.f : mn;
        const float g = ex2(0.5f * (m - at)), g_other = ex2(0.5f * (y.x - at));
        f = g * g;
        f_other = g_other * g_other;
        l = l * g * g + y.y * g_other * g_other;
        m = mn;
      }
      after_sync();
      const bool direct = whole && ends;
      float* slot = a.slots + (size_t)(2 * v + (began ? 0 : 1)) * SLOT;
      // divided by the normaliser, or by a power of two near it: it is large where weight lies on tokens of little value
      if (l > 4e37f) l = 4e37f;
      float unit = 1.f, late = 1.f;
      if (direct) {
        if (l > 1.2379400e27f) { unit = 1.1529215e18f; late = 8.6736174e-19f; }   // 2^90; 2^60 and back, so that the factor stays a normal number
        unit = l == 0.f ? 0.f : unit / l;
      } else if (l > 0.f && l < INFINITY) {
        const int e = (int)(__float_as_uint(l) >> 23) - 127;
        if (m + (float)e - m == (float)e) {
          const float down = __uint_as_float((uint32_t)(127 - e) << 23);
          unit *= down;
          m += (float)e;
          l *= down;
        }
      }
      unit *= 1.f / 16384.f;   // (not one factor with f: both may be small where the stream's sums are large)
      const bool there = row < rows;
      T* dst = there && direct ? out_row<T>(a, cur.li, cur.b, cur.h, cur.rt * R + row) : nullptr;
      // (a dual item's streams have 64 channels each)
      const uint32_t o_own = tmem + O_COL + lanes;
#pragma unroll 1
      for (int b = dual ? 4 * t : 0; b < (dual ? 4 * t + 4 : 8); b++) {
        float x[16];
        tmem_ld16(o_at + 16u * b, x);
        tmem_wait_ld();
        if (dual) {
          float y[16];
          tmem_ld16(o_own + 128u * (t ^ 1) + 16u * b, y);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e++) x[e] = fmaf(y[e], f_other, x[e] * f);
        }
        if (!there) continue;
#pragma unroll
        for (int e = 0; e < 16; e++) x[e] *= unit;
        if (late != 1.f) {
#pragma unroll
          for (int e = 0; e < 16; e++) x[e] *= late;
        }
        if (direct) {
#pragma unroll
          for (int e = 0; e < 2; e++) {
            Vec8<T> y;
#pragma unroll
            for (int z = 0; z < 8; z++) y.v[z] = from_f<T>(x[8 * e + z]);
            *reinterpret_cast<Vec8<T>*>(dst + 16 * b + 8 * e) = y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; e++)
            *reinterpret_cast<float4*>(slot + (size_t)row * D + 16 * b + 4 * e) = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
        }
      }
      before_sync();
      if (there && !direct && (!dual || t == 0)) { slot[(size_t)R * D + row] = m; slot[(size_t)R * D + R + row] = l; }
      if (dual) asm volatile("bar.sync 1, 256;\n" ::: "memory");   // the next item's products may replace the sums
      if (!began && (heads.by_item || !ends) && tid == 0)
        a.heads[heads.at(v, c.n_kv, cur.pair, cur.h, cur.rt)] =
            Head{ends ? 0 : cuts.range_of(item0 + cur.nt - 1) - v, v, cur.pair, cur.h, cur.rt, {}};
      whole = true;
      began = false;
      i += n;
      cur.skip(work, n);
    }
    if (!t) take_turn(2 + quarter);
  }
  before_sync();
  __syncthreads();
  if (tid == 0 && sm.abort) set_status(c.status, OKQ_ERR_TIMEOUT);
  if (warp == 0 && !sm.tmem_busy) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

template <class T> cudaError_t launch(const AttnArgs& a, const CUtensorMap& map, int grid, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  int dev = 0;
  constexpr int SMEM = (int)sizeof(PromptSmem) + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory of one block");
  if (attr_needed(attr_mask, dev)) {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_prompt<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    attr_done(attr_mask, dev);
  }
  cudaError_t e = launch_dependent(k_paged_prompt<T>, dim3(grid), NT, SMEM, s, 1, map, a);
  return e == cudaSuccess ? launch_merge<T, R>(a, grid, s) : e;
}

}  // namespace

cudaError_t launch_paged_prompt(const AttnArgs& a, int dtype, int grid, cudaStream_t s) {
  CUtensorMap map;
  if (!codes_map(map, a.c, false)) return cudaErrorInvalidValue;
  return dtype == OKQ_FP16 ? launch<__half>(a, map, grid, s) : launch<__nv_bfloat16>(a, map, grid, s);
}

}  // namespace okq
