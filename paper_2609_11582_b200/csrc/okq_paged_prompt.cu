// Attention over the 8-bit paged cache for many query rows per (layer, sequence, KV head): prompts, pieces of prompts,
// drafted tokens.  Causal against the end of the sequence, with a window and sinks, or by the bits of a tree of drafted tokens.
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
// With a window and for a tree a numerator is two fp16 numbers, the rounded one and what is left, each multiplied with the same values: 22
// bits.  (The causal call has one: its results are what they were.)  The second products cost 1 %; the second numbers, some 100 instructions
// of a softmax warp's step, 11: 2048 queries x 28 heads with a window of 1400 110 -> 123 us.
//
// A block of threads has 256 rows, in two streams A and B of 128, and walks the tokens in steps of 64: a loader warp (32-token blocks
// by page, two tiles of 128 tokens ahead), four warps that turn codes into fp16 (0x6400 | (code + 128) is 1024 + 128 + code; the rest is
// one subtraction per two) in the layout of the products, to each stream an MMA warp (one for both was busy with waits and issue) and four
// softmax warps (lane = row).  A stream has two places for scores, so that the next step's are there when a softmax ends.  Where an item
// has no more than 128 rows (a dual item), both streams have the same ones: A takes the first 64 tokens of every tile, B the others, and
// their sums are put together at the end.
//
// What a row sees of a step is one number where the kernel is causal, and 64 bits otherwise, worked out while the products are waited for.
// Steps that some row does not see all of have -inf put in and go the same way as the others: of a window or a tree such steps are a large
// part, and a copy of the loop for them took 4000 to 5000 cycles a step for its code's size, where this took 2600 to 2900.  (The causal
// kernel keeps its copy, which rounds otherwise, for the step or two at the end.)
//
// At best bound by the exponentials (16 per cycle and SM: 2048 cycles for 256 x 128 scores) and the products (2048 cycles at fp16's
// rate).  What it takes is about 4200 (2048 queries x 28 heads on 8192 tokens 260 us a call, 810 TFLOP/s of products): a softmax warp's own
// chain of waits, tensor memory, maximum, exponentials and roundings, with two such warps on a scheduler and 128 registers to each (the
// maximum beside the exponentials, by last step's reference: 390 us, spills).  A multiplication of O is another 1000 cycles in its step.
// A window's items are short, and their ends show: of 93000 cycles of 256 rows with a window of 1400 (26 steps) the queries take 5000, the
// first scores 2500, the last products and the output 7000; 2048 queries x 28 heads 123 us.  (Cycles as counted with one number to a
// numerator, here and below, and 300 more for a step.)  Queries are copied to their place as they are
// while the item before ends (loaded there and then they took 11000 to 17000 cycles).
// Few rows (a dual item) are bound by the conversion, a step in 1500 to 1700 cycles, a third of it waits and fences: 35 rows, 16 sequences x 4
// heads of up to 12345 tokens 47 us a causal call (a converting warp to every other step, with half of those waits but a ring that is then too
// short: 61).  Calls whose items are all dual have a kernel of their own (NARROW).
#include "okq_paged_attn.cuh"

namespace okq {

namespace {

constexpr int R = PROMPT_ROWS, EXTRA = PROMPT_EXTRA, M = 128;         // rows of a block, of a stream
constexpr int PH = PT / 2;                      // tokens of a step
constexpr int SIDE = PT * D;                    // bytes of a tile's keys or values as codes
constexpr int Q_HALF = M * 128, KV_HALF = PH * 128;   // 64 channels in fp16, of a stream's queries and of a step's keys or values
constexpr int W_CONV = 8, W_MMA = 12, W_LOAD = 14;   // (an MMA warp to each stream)
constexpr int NT = 15 * 32;
constexpr uint32_t S_COL = 0, O_COL = 256;      // + 128 per stream, + 64 per place for scores; numerators lie on its first half,
constexpr uint32_t REST = 32;                   // of a window and a tree what their rounding left on the second
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

// NARROW: a call with no more than 128 rows to a head, whose items are all dual: no queries for stream B, and a longer ring in their place.
template <bool NARROW> struct PromptSmem {
  static constexpr int NR = NARROW ? 4 : 3;        // ring of steps' keys, and values, in fp16
  __align__(1024) unsigned char q[NARROW ? 1 : 2][2][Q_HALF];   // [stream][channels / 64]
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
  signed char row_exp[2 * M];                      // of the item's rows
  FindWhole find;
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
__device__ __forceinline__ void tmem_st2(uint32_t taddr, float a, float b) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};\n" ::"r"(taddr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ float2 tmem_ld2(uint32_t taddr) {
  float2 r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];\ntcgen05.wait::ld.sync.aligned;\n" : "=f"(r.x), "=f"(r.y) : "r"(taddr) : "memory");
  return r;
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
template <class SM> __device__ __forceinline__ bool step_ready(SM& sm, const volatile int* done, int x) {
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

// A warp's rows of a row tile, four times ROUNDS from row0 on, eight lanes to a row and sixteen channels each.  Their numbers are copied, as they are, into the places that
// the fp16 ones will have (both have 16 bits); a lane copies what it will turn itself, so that its own wait is enough.  All of it is in
// flight at once, behind the end of the item before (loaded into registers two rows at a time the queries took 11000 to 17000 cycles of an
// item's 40000).
struct QueryPlace {
  int c0, c1;      // first channels of both eights
  bool turns;
  __device__ __forceinline__ QueryPlace(const RopeView& rope, int lane) {
    const int j = lane & 7, nc = rope.half >> 3;
    turns = rope.freq && j < nc;
    c0 = !rope.freq || j < nc ? 8 * j : 2 * rope.half + 16 * (j - nc);
    c1 = !rope.freq ? c0 + 64 : j < nc ? c0 + rope.half : c0 + 8;
  }
  // of row r of the stream
  __device__ __forceinline__ unsigned char* at(unsigned char* q, int r, int ch) const { return q + (ch >> 6) * Q_HALF + r * 128 + ((((ch & 63) >> 3) ^ (r & 7)) << 4); }
};
template <class T, int ROUNDS, class Cur>
__device__ __forceinline__ void fetch_queries(const AttnArgs& a, const Cur& cur, int row0, unsigned char* q, int lane) {
  const QueryPlace pl(a.rope, lane);
  const int rows = cur.m * a.c.group;
#pragma unroll 2
  for (int it = 0; it < ROUNDS; it++) {
    const int rl = 4 * it + (lane >> 3), row = cur.rt * R + row0 + rl, r = (row0 & (M - 1)) + rl;
    const int bytes = row < rows ? 16 : 0;   // (zeros for rows that the item does not have)
    const T* src = query_row<T>(a, cur.li, cur.b, cur.h, bytes ? row : 0);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(smem_u32(pl.at(q, r, pl.c0))), "l"(src + pl.c0), "r"(bytes) : "memory");
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(smem_u32(pl.at(q, r, pl.c1))), "l"(src + pl.c1), "r"(bytes) : "memory");
  }
}

// The rows that fetch_queries copied: rotated, scaled by a power of two, whose exponents go to row_exp (the softmax scale's sign goes to the
// queries).
constexpr int ROW_ZERO = -128, ROW_NAN = 127;   // rows that are zeros here; with an infinity or NaN
// the factor of the exponent that undoes the scaling, times the softmax scale
__device__ __forceinline__ float back_of(int e2, float scale2) {
  return e2 == ROW_NAN ? NAN : e2 == ROW_ZERO ? 0.f : __uint_as_float((uint32_t)(127 + e2) << 23) * fabsf(scale2);
}
template <class T, int ROUNDS, class Cur>
__device__ __forceinline__ void prepare_queries(const AttnArgs& a, const Cur& cur, int row0, unsigned char* q, signed char* row_exp, int lane) {
  const PagedView& c = a.c;
  const QueryPlace pl(a.rope, lane);
  const int rows = cur.m * c.group;
  if (lane < 4 * ROUNDS) row_exp[row0 + lane] = (signed char)ROW_ZERO;
  __syncwarp();
  asm volatile("cp.async.wait_all;\n" ::: "memory");
#pragma unroll 1
  for (int it = 0; it < ROUNDS; it++) {
    if (cur.rt * R + row0 + 4 * it >= rows) break;   // (the same in all lanes)
    const int rl = 4 * it + (lane >> 3), row = cur.rt * R + row0 + rl, r = (row0 & (M - 1)) + rl;    // row inside the warp, of the item's queries, of the stream
    Vec8<T> x[2] = {*reinterpret_cast<const Vec8<T>*>(pl.at(q, r, pl.c0)), *reinterpret_cast<const Vec8<T>*>(pl.at(q, r, pl.c1))};
    if (pl.turns && row < rows) {
      float cs[8], sn[8];
      turns8(a.rope, a.rope.positions + (size_t)cur.b * a.n_new + c.query_of(row), (size_t)c.batch * a.n_new, pl.c0, cs, sn);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        float u = to_f(x[0].v[e]), w = to_f(x[1].v[e]);
        rotate_pair(u, w, cs[e], sn[e]);
        x[0].v[e] = from_f<T>(u);
        x[1].v[e] = from_f<T>(w);
      }
    }
    // the largest magnitude, of two numbers at a time: without the sign they are in the order of their bits
    const uint32_t* bits = reinterpret_cast<const uint32_t*>(x);
    uint32_t top2 = bits[0] & 0x7fff7fffu;
#pragma unroll
    for (int e = 1; e < 8; e++) top2 = __vmaxu2(top2, bits[e] & 0x7fff7fffu);
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, d));
    const unsigned short top1 = (unsigned short)max(top2 & 0xffffu, top2 >> 16);
    const unsigned mx = __float_as_uint(to_f(*reinterpret_cast<const T*>(&top1)));
    // 2^-e brings the largest magnitude to [1, 2) (4 at the end of the range); rows too small for that, and those with an infinity or NaN, are zeros here
    const int e2 = min((int)(mx >> 23) - 127, 126);
    const bool fine = mx < 0x7f800000u && e2 > -100;
    const float up = fine ? __uint_as_float((uint32_t)(127 - e2) << 23) * (a.scale2 < 0.f ? -1.f : 1.f) : 0.f;
#pragma unroll
    for (int z = 0; z < 2; z++) {
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const __half2 h = __floats2half2_rn(to_f(x[z].v[2 * e]) * up, to_f(x[z].v[2 * e + 1]) * up);
        y[e] = fine ? *reinterpret_cast<const uint32_t*>(&h) : 0u;
      }
      *reinterpret_cast<uint4*>(pl.at(q, r, z ? pl.c1 : pl.c0)) = make_uint4(y[0], y[1], y[2], y[3]);
    }
    if ((lane & 7) == 0) row_exp[row0 + rl] = (signed char)(mx >= 0x7f800000u ? ROW_NAN : fine ? e2 : ROW_ZERO);
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Columns of a step that a row sees: up to one of them, or a bit for each.
struct UpTo {
  static constexpr bool all_ways = true;   // steps that some row does not see all of take the long way
  int last;
  __device__ __forceinline__ bool sees(int col) const { return col <= last; }
  __device__ __forceinline__ bool none_of(int block) const { return 32 * block > last; }
  __device__ __forceinline__ bool all() const { return last >= PH - 1; }
};
struct Bits {
  static constexpr bool all_ways = false;
  uint32_t half[2];
  __device__ __forceinline__ Bits(unsigned long long b) : half{(uint32_t)b, (uint32_t)(b >> 32)} {}
  __device__ __forceinline__ bool sees(int col) const { return half[col >> 5] >> (col & 31) & 1u; }
  __device__ __forceinline__ bool none_of(int block) const { return half[block] == 0u; }
  __device__ __forceinline__ bool all() const { return (half[0] & half[1]) == 0xffffffffu; }
};

// Of the step whose first token is t0.  `own`: the row's token; of a tree: the first node's.
template <int SIGHT>
__device__ __forceinline__ unsigned long long sight_bits(const AttnArgs& a, int t0, int own, const unsigned long long* row_bits, int len) {
  if (SIGHT == WINDOW) {
    const int last = own - t0, first = last - a.window + 1, sinks = a.sinks - t0;
    if (last >= PH - 1 && (first <= 0 || sinks >= PH)) return ~0ull;
    return low_bits(last + 1) & (~low_bits(first) | low_bits(sinks));
  }
  const int first = own - t0;
  if (first >= PH) return ~0ull;
  unsigned long long nodes = 0;
  if (row_bits) {
    if (first >= 0) {
      nodes = __ldcg(row_bits) << first;
    } else {
      const int w = -first >> 6, s = -first & 63;
      if (w < a.words) nodes = __ldcg(row_bits + w) >> s;
      if (s && w + 1 < a.words) nodes |= __ldcg(row_bits + w + 1) << (64 - s);
    }
  }
  return (low_bits(first) | nodes) & low_bits(len - t0);
}

// The factor of a block's scores.  Where -inf stands in the columns that a row does not see: one that makes no NaN of it (a zero is none for
// scores that are finite; a NaN is kept where the row sees any of the block).
template <class Seen> __device__ __forceinline__ float factor_of(const Info& info, int b0, int b, float back, const Seen& seen) {
  const float cb = back * info.ks[b0 + b];
  if (Seen::all_ways) return cb;
  return seen.none_of(b) ? 1.f : cb == 0.f ? 1e-38f : cb;
}

template <class Seen> __device__ __forceinline__ void mask(float (&x)[2][32], const Seen& seen) {
#pragma unroll
  for (int b = 0; b < 2; b++) {
#pragma unroll
    for (int e = 0; e < 32; e++)
      if (!seen.sees(32 * b + e)) x[b][e] = -INFINITY;
  }
}

// The lane's row of a step's scores, two blocks of 32 tokens, b0 the tile's number of the first; `seen`: the columns that the row sees.
// The largest log2 of p w, 2^P_SHIFT times.
template <bool EDGE, class Seen>
__device__ __forceinline__ float row_max(float (&x)[2][32], const Info& info, int b0, float back, const Seen& seen) {
  float mx = -INFINITY;
  if (EDGE) mask(x, seen);
#pragma unroll
  for (int b = 0; b < 2; b++) {
    float y[4] = {x[b][0], x[b][1], x[b][2], x[b][3]};
#pragma unroll
    for (int e = 4; e < 28; e += 2) y[(e >> 1) & 3] = max3(y[(e >> 1) & 3], x[b][e], x[b][e + 1]);
    const float top = max3(max3(y[0], y[1], x[b][28]), max3(y[2], y[3], x[b][29]), fmaxf(x[b][30], x[b][31]));
    mx = fmaxf(mx, EDGE && top == -INFINITY ? top : EDGE ? __fadd_rn(__fmul_rn(top, back * info.ks[b0 + b]), info.lw[b0 + b]) : fmaf(top, factor_of(info, b0, b, back, seen), info.lw[b0 + b]));
  }
  return mx;
}
// EDGE also rounds a score once before the reference is taken off, as the maximum is: the difference is exact then, where scores are so
// large that an unrounded one could lie far above it (not by packed pairs: their product and sum were contracted to one rounding).  Blocks
// without a value count in the normaliser alone.
// Of a window and a tree the numerators stay in x, for store_numerators.
template <bool EDGE, class Seen>
__device__ __forceinline__ float numerators(float (&x)[2][32], uint32_t s_at, const Info& info, int b0, float back, float ref, const Seen& seen, float l) {
#pragma unroll
  for (int b = 0; b < 2; b++) {
    const bool none = EDGE && (info.lost >> (4 + b0 + b) & 1);
    const float cb = EDGE ? back * info.ks[b0 + b] : factor_of(info, b0, b, back, seen), lw = none ? 0.f : info.lw[b0 + b], off = lw - ref;
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
        if (!seen.sees(32 * b + 2 * e)) p0 = 0.f;
        if (!seen.sees(32 * b + 2 * e + 1)) p1 = 0.f;
      }
      sum[e & 1] = add2(sum[e & 1], f2(p0, p1));
      if (Seen::all_ways) {
        const __half2 h = __floats2half2_rn(p0, p1);
        u[e] = none ? 0u : *reinterpret_cast<const uint32_t*>(&h);
      } else {
        x[b][2 * e] = none ? 0.f : p0;
        x[b][2 * e + 1] = none ? 0.f : p1;
      }
    }
    const float2 total = un2(add2(sum[0], sum[1]));
    l = fmaf(total.x + total.y, info.iw[b0 + b], l);
    if (EDGE && (info.lost >> (b0 + b) & 1) && !seen.none_of(b)) l = NAN;
    if (Seen::all_ways) tmem_st16(s_at + 16u * b, u);
  }
  return l;
}
// Numerators as two fp16 numbers, the rounded one and what the rounding left (exact in fp32; a multiply-add that takes fp16 numbers as they
// are: with the upper bits cut out and taken off, 2048 queries with a window of 1400 128 us and not 123).
__device__ __forceinline__ void store_numerators(const float (&x)[2][32], uint32_t s_at) {
#pragma unroll
  for (int b = 0; b < 2; b++) {
    uint32_t u[16], rest[16];
#pragma unroll
    for (int e = 0; e < 16; e++) {
      const float p0 = x[b][2 * e], p1 = x[b][2 * e + 1];
      const __half2 h = __floats2half2_rn(p0, p1);
      u[e] = *reinterpret_cast<const uint32_t*>(&h);
      float r0, r1;   // p - h
      asm("{\n\t.reg .b16 a, b, minus;\n\tmov.b32 {a, b}, %2;\n\tmov.b16 minus, 0xbc00;\n\tfma.rn.f32.f16 %0, a, minus, %3;\n\tfma.rn.f32.f16 %1, b, minus, %4;\n\t}\n"
          : "=f"(r0), "=f"(r1) : "r"(u[e]), "f"(p0), "f"(p1));
      const __half2 g = __floats2half2_rn(r0, r1);
      rest[e] = *reinterpret_cast<const uint32_t*>(&g);
    }
    tmem_st16(s_at + 16u * b, u);
    tmem_st16(s_at + REST + 16u * b, rest);
  }
}

// NARROW: all items are dual, and the code for the others is left out.
template <class T, int SIGHT, bool NARROW>
__global__ void __launch_bounds__(NT, 1) k_paged_prompt(const __grid_constant__ CUtensorMap map, const AttnArgs a) {
  extern __shared__ unsigned char raw_smem[];
  using Smem = PromptSmem<NARROW>;
  constexpr int NR = Smem::NR;
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
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
  Work<R, EXTRA, SIGHT> work(a);
  const int v = blockIdx.x;                     // this block's range
  const Cuts cuts = find_places<R, EXTRA, NT, 1, SIGHT>(sm.find, work, gridDim.x, v, 0);
  work.whole_at = smem_u32(&sm.find.whole);
  const int end = cuts.start(v) + cuts.size(v); // the unit behind it
  const Heads<R> heads(work.pairs, c.n_kv, c.group, a.n_new, gridDim.x);
  Cursor<R, EXTRA, SIGHT> cur = place<R, EXTRA, 1, SIGHT>(sm.find, work, cuts, v, 0);

  if (warp == W_LOAD) {
    // ------------------------------------------------------------------ loader: blocks of the tiles to come, as in the decode kernel
    Cursor<R, EXTRA, SIGHT> ahead = cur;
    int n_now = 0, n_nx = 0;
    int t_nx = 0, l_nx = 0, h_nx = 0, page_nx = -1;
    bool in_nx = false;
    int row_now = -1, row_nx = -1;               // -1: nothing to copy
    float ks_now = 0.f, vs_now = 0.f, ks_nx = 0.f, vs_nx = 0.f;
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
      if (in_nx) page_nx = __ldcg(&c.table[(size_t)b * c.max_pages + (t_nx >> c.page_shift)]);
    };
    auto scales = [&] {
      row_nx = -1;
      ks_nx = 0.f;
      vs_nx = SIGHT == CAUSAL ? 0.f : 1.f;   // (of a block that nobody sees: one that needs no care)
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
      const bool dual = NARROW || cur.m * c.group - cur.rt * R <= M;        // both streams have the same rows
      const int n = cur.piece(work), steps = dual ? n : 2 * n;
      const int x0 = 2 * i + (dual ? t : 0), dx = dual ? 2 : 1;   // step y is step x0 + dx y of the range
      const uint64_t ad = make_desc_sw128(smem_u32(sm.q[NARROW || dual ? 0 : t][0]));
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
          for (int k = 0; k < (SIGHT == CAUSAL ? 4 : 8); k++)   // 16 tokens further; then what the rounding left
            mma_ts(o_at, s_at + 64u * place + 8u * k, bd + (uint64_t)((k & 3) * 2048 >> 4), id_o, y > 0 || k != 0);
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
        const int n = cur.piece(work);
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
    if (!NARROW && t) pass_turn(2 + quarter);   // stream A begins
    bool first_item = true;
    for (int i = 0; cur.ok;) {
      const int n = cur.piece(work), rows = cur.m * c.group - cur.rt * R, item0 = end - cur.left - cur.tile;   // (the item's first unit)
      const bool ends = cur.tile + n == cur.nt, dual = NARROW || rows <= M;
      const int row0 = (dual ? 0 : M * t) + 32 * quarter, row = row0 + lane, steps = dual ? n : 2 * n;
      // (the stream's own products of the item before are through)
      // A dual item's queries lie in A's place and are prepared by A, or, where all items are dual, by both.
      constexpr int ROUNDS = NARROW ? 4 : 8;
      if (NARROW || !dual || t == 0) {
        const int first = NARROW ? 32 * quarter + 16 * t : row0;
        unsigned char* place = sm.q[NARROW || dual ? 0 : t][0];
        if (first_item) fetch_queries<T, ROUNDS>(a, cur, first, place, lane);
        prepare_queries<T, ROUNDS>(a, cur, first, place, sm.row_exp, lane);
        fence_async_smem();
      }
      if (dual) asm volatile("bar.sync 1, 256;\n" ::: "memory");
      __syncwarp();
      const float back = back_of(sm.row_exp[row], a.scale2);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[t]);
      float m = -INFINITY, l = 0.f;
      sm.peak[M * t + 32 * quarter + lane] = -INFINITY;
      {
        // (what the loop keeps in registers besides 64 scores: as little as can be)
        int seen = cur.len - cur.m + c.query_of(cur.rt * R + row) - cur.tile * PT - (dual ? PH * t : 0);   // last column of the step that the row sees
        const unsigned long long* row_bits = nullptr;
        if (SIGHT == TREE && row < rows) row_bits = a.seen + ((size_t)cur.b * a.n_new + c.query_of(cur.rt * R + row)) * a.words;
        if (SIGHT == WINDOW) seen = cur.len - cur.m + c.query_of(cur.rt * R + row);   // (the row's token)
        int half = dual ? t : 0, tile = i;
        bool wide = false;
        for (int y = 0; y < steps; y++) {
          const uint32_t p_at = s_at + 64u * (y & 1);
          if (dual || !half) bar_wait(sm, &sm.info_full[tile & 3], (uint32_t)(tile >> 2) & 1u);
          const Info& info = sm.info[tile & 3];
          const auto sight = [&] {
            if constexpr (SIGHT == CAUSAL) return UpTo{seen};
            else return Bits(sight_bits<SIGHT>(a, cur.at(cur.tile + tile - i) * PT + PH * half, SIGHT == TREE ? cur.len - cur.m : seen, row_bits, cur.len));
          }();
          bar_wait(sm, &sm.s_full[t][y & 1], ph_s >> (y & 1) & 1u);
          ph_s ^= 1u << (y & 1);
          after_sync();
          float x[2][32];
          tmem_ld32(p_at, x[0]);
          tmem_ld32(p_at + 32u, x[1]);
          // (of a window and a tree many steps are masked, and their scores are set to -inf for the short way; it is the code's size that
          // counts: a masked copy of the short way took 4000 cycles a step)
          const bool masked = __any_sync(0xffffffffu, !sight.all()), edge = info.lost || (SIGHT == CAUSAL && masked);
          tmem_wait_ld();
          if (SIGHT != CAUSAL && masked) mask(x, sight);
          const float mx = edge ? row_max<true>(x, info, 2 * half, back, sight) : row_max<false>(x, info, 2 * half, back, sight);
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
          l = edge || wide ? numerators<true>(x, p_at, info, 2 * half, back, ref, sight, l) : numerators<false>(x, p_at, info, 2 * half, back, ref, sight, l);
          if (!dual) pass_turn(2 + 4 * (t ^ 1) + quarter);
          if (SIGHT != CAUSAL) store_numerators(x, p_at);
          tmem_wait_st();
          before_sync();
          __syncwarp();
          // Phases of o_full are told apart by one bit: the last but one is waited for while the last cannot be complete, since all that is
          // known without a wait is that the third last is.
          if (y > 0 && y + 1 == steps) bar_wait(sm, &sm.o_full[t], (uint32_t)(n_o + y - 1) & 1u);
          if (lane == 0) mbar_arrive(&sm.p_full[t][y & 1]);
          if (dual) {
            tile++;
            if (SIGHT == CAUSAL) seen -= PT;
          } else {
            tile += half;
            half ^= 1;
            if (SIGHT == CAUSAL) seen -= PH;
          }
        }
      }
      n_o += steps;
      // The next item's queries, from here on: this stream's scores are through, and those of a dual item when both streams meet.
      auto next = cur;
      next.skip(work, n);
      auto fetch_next = [&] {
        const bool next_dual = NARROW || next.m * c.group - next.rt * R <= M;
        if (next.ok && (NARROW || t == 0 || !next_dual))
          fetch_queries<T, ROUNDS>(a, next, NARROW ? 32 * quarter + 16 * t : (next_dual ? 0 : M * t) + 32 * quarter, sm.q[NARROW || next_dual ? 0 : t][0], lane);
      };
      first_item = false;
      if (!dual) fetch_next();
      bar_wait(sm, &sm.o_full[t], (uint32_t)(n_o - 1) & 1u);
      if (sm.abort) l = NAN;
      float f = 1.f, f_other = 0.f;
      if (dual) {
        // statistics in the place of the first scores
        const uint32_t stat = tmem + S_COL + lanes;
        tmem_st2(stat + 128u * t, m, l);
        tmem_wait_st();
        before_sync();
        asm volatile("bar.sync 1, 256;\n" ::: "memory");   // both streams' sums are complete
        after_sync();
        fetch_next();
        const float2 y = tmem_ld2(stat + 128u * (t ^ 1));
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
          for (int e = 0; e < 16; e++) slot[(16 * b + e) * R + row] = x[e];
        }
      }
      before_sync();
      if (there && !direct && (!dual || t == 0)) { slot[(size_t)R * D + row] = m; slot[(size_t)R * D + R + row] = l; }
      if (dual) asm volatile("bar.sync 1, 256;\n" ::: "memory");   // the next item's products may replace the sums and statistics
      if (!began && (heads.by_item || !ends) && tid == 0)
        a.heads[heads.at(v, c.n_kv, cur.pair, cur.h, cur.rt)] =
            Head{ends ? 0 : cuts.range_of(item0 + cur.nt - 1) - v, v, cur.pair, cur.h, cur.rt, {}};
      whole = true;
      began = false;
      i += n;
      cur = next;
    }
    if (!NARROW && !t) take_turn(2 + quarter);
  }
  before_sync();
  __syncthreads();
  if (tid == 0 && sm.abort) set_status(c.status, OKQ_ERR_TIMEOUT);
  if (warp == 0 && !sm.tmem_busy) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
}

__device__ __forceinline__ void late(float& top, float& l, float (&x)[8]) {
  top += LATE_BITS;
  l *= LATE;
#pragma unroll
  for (int z = 0; z < 8; z++) x[z] *= LATE;
}
// Parts put together, in order.  A part's reference may lie 2^76 below its largest numerator, and its sums above as much: factors go down to
// 2^-226, in two steps where one would leave fp32's normal numbers (calls with 9 to 37 parts to a row 0.2 to 1.1 us longer for it; a look
// at all parts before the one at each was no shorter).  A part has its sums channel by channel, R rows each, as the lanes that hold rows write and read whole lines of
// them (row by row the stores took 8000 cycles of a piece's 90000, and this kernel 23 us of 135 for 2048 queries x 28 heads with a window).
// A warp has 32 rows and eight channels, WPR warps have every WPR-th part each; unit u of a block's 16 / WPR is rows u / 16, channels u % 16.
// FLIGHT parts are loaded at once: two, so that two blocks fit an SM, or seven where there are no more blocks than SMs.
template <class T, int WPR, int FLIGHT>
__global__ void __launch_bounds__(MERGE_NT, FLIGHT > 2 ? 1 : 2) k_prompt_merge(const AttnArgs a) {
  constexpr int WARPS = MERGE_NT / 32;
  __shared__ float sums[WPR > 1 ? WARPS : 1][8][32];
  __shared__ float2 stat[WPR > 1 ? WARPS : 1][32];
  depend_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = blockIdx.y * (WARPS / WPR) + warp / WPR, first = warp % WPR;
  const int r = 32 * (unit >> 4) + lane, ch = 8 * (unit & 15);
  const int4 h0 = __ldcg(reinterpret_cast<const int4*>(&a.heads[blockIdx.x]));
  const Head hd{h0.x, h0.y, h0.z, h0.w, __ldcg(&a.heads[blockIdx.x].rt), {}};
  if (hd.more == 0) return;
  const int n = hd.more + 1, row = hd.rt * R + r;
  auto slot = [&](int k) { return a.slots + (size_t)(2 * (hd.v + k) + (k == 0)) * SLOT; };
  const Work<R, 0> w(a);
  int len, m;
  const int li = w.layer_of(hd.pair), b = hd.pair - li * a.c.batch;
  w.lens(li, b, len, m);
  const bool there = row < m * w.group;
  float acc[8] = {}, top = -INFINITY, l = 0.f;
  if (there) {
    for (int k0 = first; k0 < n; k0 += 7 * WPR) {
      float tk[7], lk[7];
      float mn = top;
#pragma unroll
      for (int e = 0; e < 7; e++) {
        const int k = k0 + e * WPR;
        const float* s = slot(k) + R * D + r;
        tk[e] = k < n ? __ldcg(s) : -INFINITY;
        lk[e] = k < n ? __ldcg(s + R) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 7; e++) mn = fmaxf(mn, tk[e]);
      const float ref = mn == -INFINITY ? 0.f : mn;
      if (falls(top, ref)) late(top, l, acc);
      const float f0 = ex2(top - ref);
      l *= f0;
#pragma unroll
      for (int z = 0; z < 8; z++) acc[z] *= f0;
      top = mn;
#pragma unroll
      for (int e0 = 0; e0 < 7; e0 += FLIGHT) {
        float x[FLIGHT][8];
#pragma unroll
        for (int e = e0; e < min(7, e0 + FLIGHT); e++) {
          const int k = k0 + e * WPR;
          const float* s = slot(k) + (size_t)ch * R + r;
#pragma unroll
          for (int z = 0; z < 8; z++) x[e - e0][z] = k < n ? __ldcg(s + z * R) : 0.f;
        }
#pragma unroll
        for (int e = e0; e < min(7, e0 + FLIGHT); e++) {
          if (falls(tk[e], ref)) late(tk[e], lk[e], x[e - e0]);
          const float f = ex2(tk[e] - ref);   // (0 where there is none)
          l = fmaf(lk[e], f, l);
#pragma unroll
          for (int z = 0; z < 8; z++) acc[z] = fmaf(x[e - e0][z], f, acc[z]);
        }
      }
    }
  }
  if (WPR > 1) {
#pragma unroll
    for (int z = 0; z < 8; z++) sums[warp][z][lane] = acc[z];
    stat[warp][lane] = make_float2(top, l);
    __syncthreads();
    if (first != 0) return;
    float mn = top;
#pragma unroll
    for (int i = 1; i < WPR; i++) mn = fmaxf(mn, stat[warp + i][lane].x);
    const float ref = mn == -INFINITY ? 0.f : mn;
    if (falls(top, ref)) late(top, l, acc);
    const float f0 = ex2(top - ref);
    l *= f0;
#pragma unroll
    for (int z = 0; z < 8; z++) acc[z] *= f0;
#pragma unroll
    for (int i = 1; i < WPR; i++) {
      float2 y = stat[warp + i][lane];
      float x[8];
#pragma unroll
      for (int z = 0; z < 8; z++) x[z] = sums[warp + i][z][lane];
      if (falls(y.x, ref)) late(y.x, y.y, x);
      const float f = ex2(y.x - ref);
      l = fmaf(y.y, f, l);
#pragma unroll
      for (int z = 0; z < 8; z++) acc[z] = fmaf(x[z], f, acc[z]);
    }
  }
  if (!there) return;
  Vec8<T> o;
#pragma unroll
  for (int z = 0; z < 8; z++) o.v[z] = from_f<T>(l == 0.f ? 0.f : acc[z] / l);
  *reinterpret_cast<Vec8<T>*>(out_row<T>(a, li, b, hd.h, row) + ch) = o;
}
template <class T, int WPR, int FLIGHT> cudaError_t launch_merge_by(const AttnArgs& a, int heads, int rows, cudaStream_t s) {
  const int units = (rows + 31) / 32 * 16, per = MERGE_NT / 32 / WPR;
  return launch_dependent(k_prompt_merge<T, WPR, FLIGHT>, dim3(heads, (units + per - 1) / per), MERGE_NT, 0, s, 1, a);
}
template <class T> cudaError_t launch_merge(const AttnArgs& a, int ranges, cudaStream_t s) {
  const Heads<R> heads(a.layer_count * a.c.batch, a.c.n_kv, a.c.group, a.n_new, ranges);
  const int n = heads.count(ranges), parts = heads.items < ranges ? ranges / heads.items : 1;   // (of an item, were all alike)
  const long long rows = (long long)a.n_new * a.c.group, most = rows < R ? rows : R, blocks = n * ((most + 31) / 32), sms = sm_count();
  // Warps to a row: more where one would load parts several times in a row, as long as the GPU holds them all at once.  A call in us with one,
  // four, sixteen: 1 x 4 heads of 32768 tokens, 64 rows (37 parts, 8 blocks with one) 49, 41, 37; 16 heads of 4096, 112 rows (9 parts, 64
  // blocks) 37, 33, 39; 16 heads of 8000, 256 rows (9 parts, 128 blocks) 51, 53, 66.
  if (parts >= 16 && 16 * blocks <= sms) return launch_merge_by<T, 16, 2>(a, n, (int)most, s);
  if (parts >= 4 && 4 * blocks <= 2 * sms) return launch_merge_by<T, 4, 2>(a, n, (int)most, s);
  return blocks <= sms ? launch_merge_by<T, 1, 7>(a, n, (int)most, s) : launch_merge_by<T, 1, 2>(a, n, (int)most, s);
}

template <class T, int SIGHT, bool NARROW> cudaError_t launch(const AttnArgs& a, const CUtensorMap& map, int grid, cudaStream_t s) {
  static thread_local unsigned long long attr_mask = 0;
  int dev = 0;
  constexpr int SMEM = (int)sizeof(PromptSmem<NARROW>) + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory of one block");
  if (attr_needed(attr_mask, dev)) {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_prompt<T, SIGHT, NARROW>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    attr_done(attr_mask, dev);
  }
  cudaError_t e = launch_dependent(k_paged_prompt<T, SIGHT, NARROW>, dim3(grid), NT, SMEM, s, 1, map, a);
  return e == cudaSuccess ? launch_merge<T>(a, grid, s) : e;
}

template <int SIGHT> cudaError_t launch_sight(const AttnArgs& a, const CUtensorMap& map, int dtype, int grid, cudaStream_t s) {
  if ((long long)a.n_new * a.c.group <= M)
    return dtype == OKQ_FP16 ? launch<__half, SIGHT, true>(a, map, grid, s) : launch<__nv_bfloat16, SIGHT, true>(a, map, grid, s);
  return dtype == OKQ_FP16 ? launch<__half, SIGHT, false>(a, map, grid, s) : launch<__nv_bfloat16, SIGHT, false>(a, map, grid, s);
}

}  // namespace

cudaError_t launch_paged_prompt(const AttnArgs& a, int dtype, Sight sight, int grid, cudaStream_t s) {
  CUtensorMap map;
  if (!codes_map(map, a.c, false)) return cudaErrorInvalidValue;
  if (sight == WINDOW) return launch_sight<WINDOW>(a, map, dtype, grid, s);
  if (sight == TREE) return launch_sight<TREE>(a, map, dtype, grid, s);
  return launch_sight<CAUSAL>(a, map, dtype, grid, s);
}

}  // namespace okq
