// Pages of the 8-bit paged cache: handing out, sharing, giving back, copying and moving them, all on the device.
//
// The tables and counts are a few hundred kilobytes at most and every decision depends on the ones before it (which page is free next),
// so one thread block of 1024 takes them, 4096 entries at a time; what moves (codes, scales, raw tokens) is left in a list and
// copied by a second kernel on the whole GPU, bound by memory: bytes read and written once.  Tables and counts are read past the first
// cache: a kernel placed before its predecessor's end may find there what its predecessor read.
#include "okq_paged.cuh"

namespace okq {

namespace {

constexpr int NT = 1024, PER = 4, CHUNK = NT * PER;

struct Scan {
  int warp[NT / 32];
  int total;
};

// exclusive sum of x over the block; sc.total is the sum of all.  Ends with a barrier behind it.
__device__ __forceinline__ int block_scan(Scan& sc, int x) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int v = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += y;
  }
  if (lane == 31) sc.warp[w] = v;
  __syncthreads();
  if (w == 0) {
    int s = sc.warp[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += y;
    }
    sc.warp[lane] = s;
    if (lane == 31) sc.total = s;
  }
  __syncthreads();
  const int before = (w ? sc.warp[w - 1] : 0) + v - x;
  return before;
}

// Free pages in ascending order, found as they are asked for: a queue of up to CHUNK page numbers in shared memory.
struct FreePages {
  Scan sc;
  int queue[CHUNK];
  int head, count, next;   // first unused, filled, first page not looked at yet
};
__device__ __forceinline__ void free_init(FreePages& f) {
  if (threadIdx.x == 0) f.head = f.count = f.next = 0;
  __syncthreads();
}
// refills the queue when it is empty; afterwards f.head < f.count unless no page is free any more.  All threads call it.
__device__ __forceinline__ void free_refill(FreePages& f, const PagedView& c) {
  while (f.head == f.count && f.next < c.n_pages) {
    const int p0 = f.next + PER * threadIdx.x;
    int is[PER], n = 0;
#pragma unroll
    for (int e = 0; e < PER; e++) {
      is[e] = p0 + e < c.n_pages && __ldcg(&c.refs[p0 + e]) == 0;
      n += is[e];
    }
    __syncthreads();
    int at = block_scan(f.sc, n);
#pragma unroll
    for (int e = 0; e < PER; e++)
      if (is[e]) f.queue[at++] = p0 + e;
    __syncthreads();
    if (threadIdx.x == 0) { f.head = 0; f.count = f.sc.total; f.next += CHUNK; }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(NT) k_pages_reserve(const PagedView c, const int32_t* tokens) {
  __shared__ FreePages f;
  depend_wait();
  const int tid = threadIdx.x;
  const long long entries = (long long)c.batch * c.max_pages;
  auto wanted = [&](long long e) -> bool {   // entry e = (sequence, place) lacks a page that the call asks for
    if (e >= entries) return false;
    const int b = (int)(e / c.max_pages), j = (int)(e - (long long)b * c.max_pages);
    return (long long)j << c.page_shift < __ldcg(&tokens[b]) && __ldcg(&c.table[e]) < 0;
  };
  // all or nothing: what is asked for, then what is free
  long long need = 0, have = 0;
  int over = 0;
  for (int b = tid; b < c.batch; b += NT) over |= __ldcg(&tokens[b]) > c.room();
  if (__syncthreads_or(over)) {
    if (tid == 0) set_status(c.status, OKQ_ERR_CAPACITY);
    return;
  }
  for (long long e0 = 0; e0 < entries; e0 += CHUNK) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < PER; e++) n += wanted(e0 + e * NT + tid);
    need += n;
  }
  for (int p0 = 0; p0 < c.n_pages; p0 += CHUNK) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < PER; e++) n += p0 + e * NT + tid < c.n_pages && __ldcg(&c.refs[p0 + e * NT + tid]) == 0;
    have += n;
  }
  block_scan(f.sc, (int)need);   // (both fit 32 bits: entries and pages do)
  const int need_all = f.sc.total;
  __syncthreads();
  block_scan(f.sc, (int)have);
  const int have_all = f.sc.total;
  __syncthreads();
  if (need_all > have_all) {
    if (tid == 0) set_status(c.status, OKQ_ERR_CAPACITY);
    return;
  }
  free_init(f);
  for (long long e0 = 0, given = 0; given < need_all; e0 += CHUNK) {
    bool want[PER];
    int n = 0;
#pragma unroll
    for (int e = 0; e < PER; e++) { want[e] = wanted(e0 + PER * tid + e); n += want[e]; }
    const int rank0 = block_scan(f.sc, n), total = f.sc.total;
    __syncthreads();
    given += total;
    for (int done = 0; done < total;) {   // the queue may hold fewer than the chunk wants
      free_refill(f, c);
      const int head = f.head, take = min(total - done, f.count - head);
      if (take <= 0) break;               // (cannot be: they were counted)
      int rank = rank0;
#pragma unroll
      for (int e = 0; e < PER; e++) {
        if (!want[e]) continue;
        if (rank >= done && rank < done + take) {
          const int p = f.queue[head + rank - done];
          c.table[e0 + PER * tid + e] = p;
          c.refs[p] = 1;
        }
        rank++;
      }
      done += take;
      __syncthreads();
      if (tid == 0) f.head = head + take;
      __syncthreads();
    }
  }
}

// Whether pair (a, d) can be forked, by the `n` threads that call it (lane t of them): 0, or a bit set in some of their answers.
__device__ __forceinline__ int fork_wrong(const PagedView& c, int a, int d, int len, int t, int n) {
  int wrong = 0;
  for (int l = t; l < c.n_layers; l += n) wrong |= c.held(l, a) != len;
  for (int j = t; j < c.max_pages; j += n) {
    wrong |= __ldcg(&c.table[(size_t)d * c.max_pages + j]) >= 0;                                   // the destination has pages
    wrong |= (long long)j << c.page_shift < len && c.page_of(a, j << c.page_shift) < 0;   // the source lacks one
  }
  return wrong;
}
// full pages and lengths of a pair
__device__ __forceinline__ void fork_share(const PagedView& c, int a, int d, int len, int t, int n) {
  for (int j = t; j < len >> c.page_shift; j += n) {
    const int p = __ldcg(&c.table[(size_t)a * c.max_pages + j]);
    c.table[(size_t)d * c.max_pages + j] = p;
    atomicAdd(&c.refs[p], 1);
  }
  for (int l = t; l < c.n_layers; l += n) c.seq_len[(size_t)l * c.batch + d] = len;
}

// list[i] = pair i's (page to copy from, page to copy to, sequence to copy raw tokens from, sequence to copy them to), -1 where there is
// nothing to copy.  Pairs that do not touch one another's sequences are taken together, a warp to each (8 pairs 20 -> 8 us); others one
// after the other, and then a source that this call itself forked is replaced by the one it came from, so that no copy waits for another.
__global__ void __launch_bounds__(NT) k_pages_fork(const PagedView c, const int32_t* src, const int32_t* dst, int count, int4* list) {
  __shared__ FreePages f;
  __shared__ int2 root;           // page and sequence that the source's own came from
  __shared__ int bad_of[NT];      // by pair: status; length
  __shared__ int len_of[NT];
  depend_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  free_init(f);
  bool apart = count <= NT;
  if (apart) {
    int meet = 0;
    for (int i = warp; i < count; i += NT / 32) {
      const int a = __ldcg(&src[i]), d = __ldcg(&dst[i]);
      int bad = (unsigned)a >= (unsigned)c.batch || (unsigned)d >= (unsigned)c.batch || a == d ? OKQ_ERR_INVALID_ARG : 0;
      for (int k = lane; k < count; k += 32) meet |= k != i && (__ldcg(&dst[k]) == d || __ldcg(&dst[k]) == a);
      const int len = bad ? 0 : c.held(0, a);
      if (!bad && __any_sync(0xffffffffu, fork_wrong(c, a, d, len, lane, 32))) bad = OKQ_ERR_INVALID_ARG;
      if (lane == 0) { bad_of[i] = bad; len_of[i] = len; }
    }
    apart = !__syncthreads_or(meet);
  }
  if (apart) {
    // free pages for the unfinished ones, in the pairs' order
    const bool mine = tid < count;
    int bad = mine ? bad_of[tid] : 0, fresh = -1;
    const int len = mine ? len_of[tid] : 0;
    const bool part = mine && !bad && (len & (c.page - 1)) != 0;
    const int rank = block_scan(f.sc, part), total = f.sc.total;
    __syncthreads();
    for (int done = 0; done < total;) {
      free_refill(f, c);
      const int head = f.head, take = min(total - done, f.count - head);
      if (take <= 0) break;
      if (part && rank >= done && rank < done + take) fresh = f.queue[head + rank - done];
      done += take;
      __syncthreads();
      if (tid == 0) f.head = head + take;
      __syncthreads();
    }
    if (part && fresh < 0) bad = OKQ_ERR_CAPACITY;
    if (mine) {
      int4 todo = make_int4(-1, -1, -1, -1);
      const int a = __ldcg(&src[tid]), d = __ldcg(&dst[tid]), full = len >> c.page_shift;
      if (!bad && len > 0) { todo.z = a; todo.w = d; }
      if (!bad && part) {
        todo.x = __ldcg(&c.table[(size_t)a * c.max_pages + full]);
        todo.y = fresh;
        c.table[(size_t)d * c.max_pages + full] = fresh;
        c.refs[fresh] = 1;
      }
      if (bad) set_status(c.status, bad);
      list[tid] = todo;
      bad_of[tid] = bad;
    }
    __syncthreads();
    for (int i = warp; i < count; i += NT / 32)
      if (!bad_of[i]) fork_share(c, __ldcg(&src[i]), __ldcg(&dst[i]), len_of[i], lane, 32);
    return;
  }
  for (int i = 0; i < count; i++) {
    const int a = __ldcg(&src[i]), d = __ldcg(&dst[i]);
    int bad = (unsigned)a >= (unsigned)c.batch || (unsigned)d >= (unsigned)c.batch || a == d ? OKQ_ERR_INVALID_ARG : 0;
    int len = 0;
    if (tid == 0) root = make_int2(-1, a);
    if (!bad) {
      len = c.held(0, a);
      if (__syncthreads_or(fork_wrong(c, a, d, len, tid, NT))) bad = OKQ_ERR_INVALID_ARG;
    }
    const int full = len >> c.page_shift;
    const bool part = (len & (c.page - 1)) != 0;
    if (!bad && part) {
      free_refill(f, c);
      if (f.head == f.count) bad = OKQ_ERR_CAPACITY;
    }
    if (!bad) {
      for (int k = tid; k < i; k += NT)
        if (list[k].w == a) root = make_int2(list[k].x, list[k].z);
      fork_share(c, a, d, len, tid, NT);
    }
    __syncthreads();
    if (tid == 0) {
      int4 todo = make_int4(-1, -1, -1, -1);
      if (!bad && len > 0) { todo.z = root.y; todo.w = d; }
      if (!bad && part) {
        const int fresh = f.queue[f.head++];
        todo.x = root.x >= 0 ? root.x : __ldcg(&c.table[(size_t)a * c.max_pages + full]);
        todo.y = fresh;
        c.table[(size_t)d * c.max_pages + full] = fresh;
        c.refs[fresh] = 1;
      }
      if (bad) set_status(c.status, bad);
      list[i] = todo;
    }
    __syncthreads();
  }
}

// 16-byte pieces of `n` bytes, dealt over the threads of `parts` blocks
__device__ __forceinline__ void copy_bytes(void* dst, const void* src, size_t bytes, int part, int parts, int tid, int nt) {
  const int4* a = static_cast<const int4*>(src);
  int4* b = static_cast<int4*>(dst);
  const size_t n = bytes / 16, step = (size_t)parts * nt;
  size_t i = (size_t)part * nt + tid;
  for (; i + 3 * step < n; i += 4 * step) {
    const int4 x0 = a[i], x1 = a[i + step], x2 = a[i + 2 * step], x3 = a[i + 3 * step];
    b[i] = x0; b[i + step] = x1; b[i + 2 * step] = x2; b[i + 3 * step] = x3;
  }
  for (; i < n; i += step) b[i] = a[i];
}

// codes and scales of a page in one layer
__device__ __forceinline__ void copy_page(const PagedView& c, int l, int from, int to, int part, int parts, int tid, int nt) {
  const size_t rows = (size_t)c.n_kv * 2 * c.page, a = c.code_row(l, from, 0, 0), b = c.code_row(l, to, 0, 0);
  copy_bytes(c.codes + b * D, c.codes + a * D, rows * D, part, parts, tid, nt);
  if (part == 0)
    for (int i = tid; i < (int)(rows / PB); i += nt) c.scales[b / PB + i] = c.scales[a / PB + i];
}

constexpr int CT = 256;   // threads of a copying block

// grid (pairs, layers, parts): the unfinished page and the raw tokens of every forked pair
__global__ void __launch_bounds__(CT) k_fork_copy(const PagedView c, const int4* list) {
  depend_wait();
  const int l = blockIdx.y, part = blockIdx.z, parts = gridDim.z, tid = threadIdx.x;
  const int4 p = list[blockIdx.x];
  if (p.x >= 0) copy_page(c, l, p.x, p.y, part, parts, tid, CT);
  const size_t raw = (size_t)c.n_kv * 2 * PB * D * 2;
  if (p.z >= 0)
    copy_bytes(static_cast<char*>(c.raw) + ((size_t)l * c.batch + p.w) * raw, static_cast<char*>(c.raw) + ((size_t)l * c.batch + p.z) * raw, raw,
               part, parts, tid, CT);
}

// one block per named sequence
__global__ void __launch_bounds__(CT) k_pages_release(const PagedView c, const int32_t* seqs) {
  depend_wait();
  const int b = __ldcg(&seqs[blockIdx.x]);
  if ((unsigned)b >= (unsigned)c.batch) {
    if (threadIdx.x == 0) set_status(c.status, OKQ_ERR_INVALID_ARG);
    return;
  }
  for (int j = threadIdx.x; j < c.max_pages; j += CT) {
    const int p = atomicExch(&c.table[(size_t)b * c.max_pages + j], -1);   // one of two blocks that name the sequence gets the page
    if (p < 0) continue;
    if (p >= c.n_pages) { set_status(c.status, OKQ_ERR_INVALID_ARG); continue; }
    if (atomicSub(&c.refs[p], 1) <= 0) {                                   // counts that do not match the tables
      atomicAdd(&c.refs[p], 1);
      set_status(c.status, OKQ_ERR_INVALID_ARG);
    }
  }
  for (int l = threadIdx.x; l < c.n_layers; l += CT) c.seq_len[(size_t)l * c.batch + b] = 0;
}

// grid (pairs, layers, parts)
__global__ void __launch_bounds__(CT) k_pages_copy(const PagedView c, const int32_t* src, const int32_t* dst, int count) {
  depend_wait();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int a = __ldcg(&src[i]), d = __ldcg(&dst[i]);
  int bad = (unsigned)a >= (unsigned)c.n_pages || (unsigned)d >= (unsigned)c.n_pages;
  for (int k = tid; k < count; k += CT) bad |= k != i && (__ldcg(&dst[k]) == d || __ldcg(&src[k]) == d);
  if (__syncthreads_or(bad)) {
    if (tid == 0) set_status(c.status, OKQ_ERR_INVALID_ARG);
    return;
  }
  if (a != d) copy_page(c, blockIdx.y, a, d, blockIdx.z, gridDim.z, tid, CT);
}

// What compaction moves: to[p] = page p's new place, pairs[k] = (from, to) of the k-th move, head[0] = moves
__global__ void __launch_bounds__(NT) k_compact_plan(const PagedView c, int32_t* n_live, int32_t* head, int2* pairs, int32_t* to) {
  __shared__ Scan sc;
  depend_wait();
  const int tid = threadIdx.x;
  int live = 0;
  for (int p = tid; p < c.n_pages; p += NT) live += __ldcg(&c.refs[p]) > 0;
  block_scan(sc, live);
  const int n = sc.total;
  __syncthreads();
  // k-th hole among the first n pages and k-th page in use behind them; equally many of both
  int holes = 0, movers = 0;
  for (int q0 = 0; q0 < c.n_pages; q0 += CHUNK) {
    bool hole[PER], mover[PER];
    int nh = 0, nm = 0;
#pragma unroll
    for (int e = 0; e < PER; e++) {
      const int p = q0 + PER * tid + e;
      const bool in = p < c.n_pages, used = in && __ldcg(&c.refs[p]) > 0;
      hole[e] = in && !used && p < n;
      mover[e] = used && p >= n;
      nh += hole[e];
      nm += mover[e];
      if (in) to[p] = p;
    }
    // both counts in one scan: at most 4096 of each in a chunk
    const int r = block_scan(sc, nh | nm << 16), total = sc.total;
    int ah = holes + (r & 0xffff), am = movers + (r >> 16);
#pragma unroll
    for (int e = 0; e < PER; e++) {
      const int p = q0 + PER * tid + e;
      if (hole[e]) pairs[ah++].y = p;
      if (mover[e]) pairs[am++].x = p;
    }
    holes += total & 0xffff;
    movers += total >> 16;
    __syncthreads();
  }
  for (int k = tid; k < movers; k += NT) {   // (written by this block: visible behind the barrier)
    const int2 m = pairs[k];
    to[m.x] = m.y;
    c.refs[m.y] = __ldcg(&c.refs[m.x]);
    c.refs[m.x] = 0;
  }
  if (tid == 0) {
    head[0] = movers;
    if (n_live) n_live[0] = n;
  }
}

// the moves (pair by pair, every layer) and the tables
__global__ void __launch_bounds__(CT) k_compact_move(const PagedView c, const int32_t* head, const int2* pairs, const int32_t* to) {
  depend_wait();
  const int tid = threadIdx.x;
  const long long n = (long long)head[0] * c.n_layers;
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const int2 m = pairs[u / c.n_layers];
    copy_page(c, (int)(u % c.n_layers), m.x, m.y, 0, 1, tid, CT);
  }
  const long long entries = (long long)c.batch * c.max_pages;
  for (long long e = (long long)blockIdx.x * CT + tid; e < entries; e += (long long)gridDim.x * CT) {
    const int p = __ldcg(&c.table[e]);
    if ((unsigned)p < (unsigned)c.n_pages) c.table[e] = to[p];
  }
}

okq_status failed(cudaError_t e) {
  set_last_cuda_error((int)e);
  (void)cudaGetLastError();
  return OKQ_ERR_CUDA;
}

// blocks that a page of one layer is dealt over: enough to fill the GPU, at least 8 KB each
int parts_of(const PagedView& c, long long pages) {
  const long long bytes = (long long)c.n_kv * 2 * c.page * D, most = bytes / 8192;
  const long long want = (8ll * sm_count() + pages - 1) / pages;
  const long long p = want < most ? want : most;
  return (int)(p < 1 ? 1 : p > 64 ? 64 : p);
}

}  // namespace

}  // namespace okq

extern "C" {

okq_status okq_pages_reserve(const okq_paged* cache, const int32_t* tokens, void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if (!tokens) return OKQ_ERR_INVALID_ARG;
  if (!aligned16(tokens)) return OKQ_ERR_ALIGNMENT;
  const cudaError_t e = launch_dependent(k_pages_reserve, dim3(1), NT, 0, static_cast<cudaStream_t>(stream), 1, paged_view(cache), tokens);
  return e != cudaSuccess ? failed(e) : launch_status();
}

okq_status okq_pages_fork(const okq_paged* cache, const int32_t* src, const int32_t* dst, int32_t count, void* workspace, size_t workspace_bytes,
                          void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if (count < 0 || (count > 0 && (!src || !dst))) return OKQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(src) & 3) || (reinterpret_cast<uintptr_t>(dst) & 3) || !aligned16(workspace)) return OKQ_ERR_ALIGNMENT;
  if (count == 0) return OKQ_OK;
  if (!workspace || workspace_bytes < (size_t)count * sizeof(int4)) return OKQ_ERR_WORKSPACE;
  if (cache->n_layers > 65535) return OKQ_ERR_UNSUPPORTED;
  const PagedView c = paged_view(cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int4* list = static_cast<int4*>(workspace);
  cudaError_t e = launch_dependent(k_pages_fork, dim3(1), NT, 0, s, 1, c, src, dst, count, list);
  if (e != cudaSuccess) return failed(e);
  e = launch_dependent(k_fork_copy, dim3(count, c.n_layers, parts_of(c, (long long)count * c.n_layers)), CT, 0, s, 1, c, list);
  return e != cudaSuccess ? failed(e) : launch_status();
}

okq_status okq_pages_release(const okq_paged* cache, const int32_t* seqs, int32_t count, void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if (count < 0 || (count > 0 && !seqs)) return OKQ_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(seqs) & 3) return OKQ_ERR_ALIGNMENT;
  if (count == 0) return OKQ_OK;
  const cudaError_t e = launch_dependent(k_pages_release, dim3(count), CT, 0, static_cast<cudaStream_t>(stream), 1, paged_view(cache), seqs);
  return e != cudaSuccess ? failed(e) : launch_status();
}

okq_status okq_pages_copy(const okq_paged* cache, const int32_t* src, const int32_t* dst, int32_t count, void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if (count < 0 || (count > 0 && (!src || !dst))) return OKQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(src) & 3) || (reinterpret_cast<uintptr_t>(dst) & 3)) return OKQ_ERR_ALIGNMENT;
  if (count == 0) return OKQ_OK;
  if (cache->n_layers > 65535) return OKQ_ERR_UNSUPPORTED;
  const PagedView c = paged_view(cache);
  const cudaError_t e = launch_dependent(k_pages_copy, dim3(count, c.n_layers, parts_of(c, (long long)count * c.n_layers)), CT, 0,
                                         static_cast<cudaStream_t>(stream), 1, c, src, dst, count);
  return e != cudaSuccess ? failed(e) : launch_status();
}

okq_status okq_pages_compact(const okq_paged* cache, int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if ((reinterpret_cast<uintptr_t>(n_live) & 3) || !aligned16(workspace)) return OKQ_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < pages_workspace(cache)) return OKQ_ERR_WORKSPACE;
  const PagedView c = paged_view(cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t* head = static_cast<int32_t*>(workspace);
  int2* pairs = reinterpret_cast<int2*>(head + 4);
  int32_t* to = reinterpret_cast<int32_t*>(pairs + c.n_pages / 2 + 1);
  cudaError_t e = launch_dependent(k_compact_plan, dim3(1), NT, 0, s, 1, c, n_live, head, pairs, to);
  if (e != cudaSuccess) return failed(e);
  e = launch_dependent(k_compact_move, dim3(8 * sm_count()), CT, 0, s, 1, c, head, pairs, to);
  return e != cudaSuccess ? failed(e) : launch_status();
}

}  // extern "C"
