// The pages of a K/V cache as a pool that sequences share: copy, take, fork, free, compact (sva.h).
//
// What is decided (which free page goes where) is decided by one CTA that scans refs in the order of the ids, so that it does not depend on
// which thread comes first; what is moved is moved by a grid.  Counters (refs) are integers, whose sums are the same in any order.
#include "common.cuh"

namespace sva {

static constexpr int PLAN_THREADS = 1024, PLAN_EACH = 4;      // a scanning step looks at 4096 pages
static constexpr int MOVE_THREADS = 256;

struct PoolParams {
  uint8_t* arrays[6];                       // codes, scales, scale factors of K, then of V
  long long bytes[3];                       // of one page in each (0: the format has none)
  int32_t *refs, *table, *lengths;
  long long table_stride;
  int pages, page, rows, max_pages, n;
  const int32_t *from, *to, *keep;
  int32_t* status;
};

__device__ __forceinline__ void report(const PoolParams& prm, int bit) {
  if (prm.status) atomicOr(prm.status, bit);
}

// Exclusive prefix sum over the CTA's threads; every thread gets the total.
__device__ __forceinline__ int block_scan(int v, int* sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();                                            // (sums of the call before have been read)
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  int s = sums[lane];                                         // (32 warps)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  total = __shfl_sync(0xffffffffu, s, 31);
  const int before = __shfl_sync(0xffffffffu, s, max(warp - 1, 0));
  return (warp ? before : 0) + inc - v;
}

// Thread t asks for need >= 0 pages; the free ones of the lowest ids from `cursor` on go to the threads in order: assign(t, which of its own, id),
// id -1 where the pool has run out.  Called by all threads of the CTA; cursor is the same for all.
template <typename Assign>
__device__ void give_pages(const PoolParams& prm, int need, int& cursor, int* sums, int* prefix, int* next, Assign assign) {
  int total;
  prefix[threadIdx.x] = block_scan(need, sums, total);
  __syncthreads();
  auto owner = [&](int r) {                                   // the last thread whose first page comes at or before r
    int t = 0;
#pragma unroll
    for (int o = PLAN_THREADS / 2; o; o >>= 1)
      if (prefix[t + o] <= r) t += o;
    return t;
  };
  int got = 0;
  while (got < total && cursor < prm.pages) {
    int free[PLAN_EACH], mine = 0;
    const int p0 = cursor + (int)threadIdx.x * PLAN_EACH;
#pragma unroll
    for (int e = 0; e < PLAN_EACH; ++e) {
      free[e] = p0 + e < prm.pages && p0 + e >= 0 && prm.refs[p0 + e] <= 0;
      mine += free[e];
    }
    int found;
    int r = got + block_scan(mine, sums, found);
#pragma unroll
    for (int e = 0; e < PLAN_EACH; ++e)
      if (free[e]) {
        if (r < total) {
          const int t = owner(r);
          prm.refs[p0 + e] = 1;
          assign(t, r - prefix[t], p0 + e);
          if (r == total - 1) *next = p0 + e + 1;
        }
        ++r;
      }
    got += found;
    __syncthreads();
    cursor = got >= total ? *next : cursor > prm.pages - PLAN_THREADS * PLAN_EACH ? prm.pages : cursor + PLAN_THREADS * PLAN_EACH;
  }
  if (got < total) {
    if (threadIdx.x == 0) report(prm, SVA_DEV_NO_PAGES);
    for (int r = got + (int)threadIdx.x; r < total; r += PLAN_THREADS) {
      const int t = owner(r);
      assign(t, r - prefix[t], -1);
    }
  }
  __syncthreads();
}

__global__ void __launch_bounds__(PLAN_THREADS) pages_take_kernel(const PoolParams prm) {
  __shared__ int sums[32], prefix[PLAN_THREADS], first[PLAN_THREADS], next;
  const int zero = grid_dep_wait();
  int cursor = zero;
  for (int row0 = 0; row0 < prm.rows; row0 += PLAN_THREADS) {
    const int row = row0 + (int)threadIdx.x;
    int need = 0;
    if (row < prm.rows) {
      const long long held = max(prm.lengths[row], 0), after = held + max(prm.keep[row], 0);
      const long long from = (held + prm.page - 1) / prm.page;
      long long to = (after + prm.page - 1) / prm.page;
      if (to > prm.max_pages) {
        report(prm, SVA_DEV_BAD_INDEX);
        to = prm.max_pages;
      }
      need = (int)max(to - from, 0LL);
      first[threadIdx.x] = (int)min(from, (long long)prm.max_pages);
    }
    give_pages(prm, need, cursor, sums, prefix, &next, [&](int t, int k, int id) {
      prm.table[(row0 + t) * prm.table_stride + first[t] + k] = id;
    });
  }
}

// A slice of a page: of the codes a step of 32 KB or less, all of whose loads are in flight before the first store; with the first slice go the scales.
// 24 heads of 64 tokens x 128, 600 of 2 417 pages moved, with the plan: 88.7 us in slices of 16 KB of K and then of V with four loads in flight, now 84.5 = 5.6 TB/s.
static constexpr int COPY_EACH = 8;                          // 16-byte pieces per thread and step
__device__ __forceinline__ void copy_words(uint8_t* base, long long bytes, int src, int dst) {
  const uint32_t* from = reinterpret_cast<const uint32_t*>(base + src * bytes);
  uint32_t* to = reinterpret_cast<uint32_t*>(base + dst * bytes);
  for (long long i = threadIdx.x; i < bytes / 4; i += MOVE_THREADS) to[i] = from[i];
}
// parts: of K and V together (even ones K's)
__device__ __forceinline__ void copy_page(const PoolParams& prm, int src, int dst, int part, int parts) {
  const int tensor = part & 1, mine = part >> 1, of = parts >> 1;
  uint8_t* base = prm.arrays[3 * tensor];
  const uint4* from = reinterpret_cast<const uint4*>(base + src * prm.bytes[0]);
  uint4* to = reinterpret_cast<uint4*>(base + dst * prm.bytes[0]);
  const long long pieces = prm.bytes[0] / 16, lo = pieces * mine / of, hi = pieces * (mine + 1) / of;
  for (long long i = lo + threadIdx.x; i < hi; i += COPY_EACH * MOVE_THREADS) {
    uint4 x[COPY_EACH];
#pragma unroll
    for (int e = 0; e < COPY_EACH; ++e)
      if (i + e * MOVE_THREADS < hi) x[e] = from[i + e * MOVE_THREADS];
#pragma unroll
    for (int e = 0; e < COPY_EACH; ++e)
      if (i + e * MOVE_THREADS < hi) to[i + e * MOVE_THREADS] = x[e];
  }
  if (mine == 0) {
    copy_words(prm.arrays[3 * tensor + 1], prm.bytes[1], src, dst);
    if (prm.bytes[2]) copy_words(prm.arrays[3 * tensor + 2], prm.bytes[2], src, dst);
  }
}
__device__ __forceinline__ bool page_named(const PoolParams& prm, int id) { return id >= 0 && id < prm.pages; }

// grid (parts, n)
__global__ void __launch_bounds__(MOVE_THREADS) pages_copy_kernel(const PoolParams prm) {
  const int zero = grid_dep_wait();
  for (int i = (int)blockIdx.y + zero; i < prm.n; i += (int)gridDim.y) {
    const int src = prm.from[i], dst = prm.to[i];
    if (src < 0 || dst < 0) continue;
    if (!page_named(prm, src) || !page_named(prm, dst)) {
      if (threadIdx.x == 0 && blockIdx.x == 0) report(prm, SVA_DEV_BAD_INDEX);
      continue;
    }
    copy_page(prm, src, dst, (int)blockIdx.x, (int)gridDim.x);
  }
}

// A pair of a fork: what the child takes over.
struct Fork {
  int parent, child, length, full;          // full: pages shared
  bool good, partial;
};
__device__ __forceinline__ Fork fork_pair(const PoolParams& prm, int i) {
  Fork f;
  f.parent = prm.from[i];
  f.child = prm.to[i];
  f.good = f.parent >= 0 && f.parent < prm.rows && f.child >= 0 && f.child < prm.rows && f.parent != f.child;
  f.length = f.full = 0;
  f.partial = false;
  if (f.good) {
    const long long most = (long long)prm.max_pages * prm.page;
    f.length = (int)min((long long)max(prm.lengths[f.parent], 0), most);
    f.full = f.length / prm.page;
    f.partial = f.length % prm.page != 0;
  }
  return f;
}

__global__ void __launch_bounds__(PLAN_THREADS) pages_fork_plan_kernel(const PoolParams prm) {
  __shared__ int sums[32], prefix[PLAN_THREADS], next;
  const int zero = grid_dep_wait();
  int cursor = zero;
  for (int i0 = 0; i0 < prm.n; i0 += PLAN_THREADS) {
    Fork f = {};
    if (i0 + (int)threadIdx.x < prm.n) {
      f = fork_pair(prm, i0 + (int)threadIdx.x);
      if (!f.good) report(prm, SVA_DEV_BAD_INDEX);
      if (f.partial && !page_named(prm, prm.table[f.parent * prm.table_stride + f.full])) {
        report(prm, SVA_DEV_BAD_INDEX);
        prm.table[f.child * prm.table_stride + f.full] = -1;
        f.length = f.full * prm.page;
        f.partial = false;
      }
      if (f.good) prm.lengths[f.child] = f.length;
    }
    give_pages(prm, f.partial ? 1 : 0, cursor, sums, prefix, &next, [&](int t, int, int id) {
      const Fork g = fork_pair(prm, i0 + t);
      prm.table[g.child * prm.table_stride + g.full] = id;
      if (id < 0) prm.lengths[g.child] = g.full * prm.page;
    });
  }
}

// grid (parts + 1, n): the table's row, and slices of the last page
__global__ void __launch_bounds__(MOVE_THREADS) pages_fork_kernel(const PoolParams prm) {
  const int zero = grid_dep_wait();
  for (int i = (int)blockIdx.y + zero; i < prm.n; i += (int)gridDim.y) {
    const Fork f = fork_pair(prm, i);
    if (!f.good) continue;
    int32_t *from = prm.table + f.parent * prm.table_stride, *to = prm.table + f.child * prm.table_stride;
    if (blockIdx.x == gridDim.x - 1) {
      for (int e = (int)threadIdx.x; e < prm.max_pages; e += MOVE_THREADS) {
        if (f.partial && e == f.full) continue;                // (written by the plan)
        int id = -1;
        if (e < f.full) {
          id = from[e];
          if (page_named(prm, id)) {
            atomicAdd(prm.refs + id, 1);
          } else {
            report(prm, SVA_DEV_BAD_INDEX);
            id = -1;
          }
        }
        to[e] = id;
      }
    } else if (f.partial) {
      const int src = from[f.full], dst = to[f.full];
      if (page_named(prm, src) && page_named(prm, dst)) copy_page(prm, src, dst, (int)blockIdx.x, (int)gridDim.x - 1);
    }
  }
}

// grid (1, n).  An entry is taken out by an exchange: a row that is named twice gives its pages back once.
__global__ void __launch_bounds__(MOVE_THREADS) pages_free_kernel(const PoolParams prm) {
  const int zero = grid_dep_wait();
  for (int i = (int)blockIdx.y + zero; i < prm.n; i += (int)gridDim.y) {
    const int row = prm.to[i];
    if (row < 0 || row >= prm.rows) {
      if (threadIdx.x == 0) report(prm, SVA_DEV_BAD_INDEX);
      continue;
    }
    const int keep = prm.keep ? max(prm.keep[i], 0) : 0;
    const int first = (int)min(((long long)keep + prm.page - 1) / prm.page, (long long)prm.max_pages);
    for (int e = first + (int)threadIdx.x; e < prm.max_pages; e += MOVE_THREADS) {
      const int id = atomicExch(prm.table + row * prm.table_stride + e, -1);
      if (id < 0) continue;
      if (id >= prm.pages) {
        report(prm, SVA_DEV_BAD_INDEX);
      } else if (atomicSub(prm.refs + id, 1) <= 0) {
        atomicAdd(prm.refs + id, 1);
        report(prm, SVA_DEV_BAD_INDEX);
      }
    }
    if (threadIdx.x == 0) atomicMin(prm.lengths + row, keep);
  }
}

// workspace of a compaction: [0] moves, [1] live pages | [4 ..] src | dst (one entry per two pages each) | map [pages]
struct CompactSpace {
  int32_t *count, *src, *dst, *map;
  __host__ __device__ CompactSpace(void* ws, int pages) {
    count = static_cast<int32_t*>(ws);
    src = count + 4;
    dst = src + (pages + 1) / 2;
    map = dst + (pages + 1) / 2;
  }
};

__global__ void __launch_bounds__(PLAN_THREADS) pages_compact_plan_kernel(const PoolParams prm, void* ws, int32_t* live_out) {
  __shared__ int sums[32];
  const int zero = grid_dep_wait();
  const CompactSpace space(ws, prm.pages);
  int mine = 0, live;
  for (long long p = (int)threadIdx.x + zero; p < prm.pages; p += PLAN_THREADS) mine += prm.refs[p] > 0;
  (void)block_scan(mine, sums, live);
  int holes = 0, movers = 0;
  for (long long p0 = 0; p0 < prm.pages; p0 += PLAN_THREADS * PLAN_EACH) {
    const long long first = p0 + (long long)threadIdx.x * PLAN_EACH;
    int flag[PLAN_EACH], both = 0;                            // free ids below the border in the low half, pages in use above it in the high one
#pragma unroll
    for (int e = 0; e < PLAN_EACH; ++e) {
      const long long p = first + e;
      flag[e] = 0;
      if (p < prm.pages) {
        const bool used = prm.refs[p] > 0;
        if (p < live) flag[e] = used ? 0 : 1;
        else {
          flag[e] = used ? 1 << 16 : 0;
          if (!used) space.map[p] = -1;
        }
      }
      both += flag[e];
    }
    int sum;
    int before = block_scan(both, sums, sum);
#pragma unroll
    for (int e = 0; e < PLAN_EACH; ++e) {
      if (flag[e] == 1) space.dst[holes + (before & 0xffff)] = (int)(first + e);
      if (flag[e] == 1 << 16) space.src[movers + (before >> 16)] = (int)(first + e);
      before += flag[e];
    }
    holes += sum & 0xffff;
    movers += sum >> 16;
  }
  __syncthreads();                                            // (src and dst are written; there are as many of one as of the other)
  for (int k = (int)threadIdx.x; k < movers; k += PLAN_THREADS) {
    const int src = space.src[k], dst = space.dst[k];
    space.map[src] = dst;
    prm.refs[dst] = prm.refs[src];
    prm.refs[src] = 0;
  }
  if (threadIdx.x == 0) {
    space.count[0] = movers;
    space.count[1] = live;
    if (live_out) *live_out = live;
  }
}

__global__ void __launch_bounds__(MOVE_THREADS) pages_compact_kernel(const PoolParams prm, void* ws, int parts) {
  const int zero = grid_dep_wait();
  const CompactSpace space(ws, prm.pages);
  const int moves = space.count[0 + zero], live = space.count[1 + zero];
  const long long entries = (long long)prm.rows * prm.max_pages;
  for (long long i = (long long)blockIdx.x * MOVE_THREADS + threadIdx.x; i < entries; i += (long long)gridDim.x * MOVE_THREADS) {
    int32_t* entry = prm.table + i / prm.max_pages * prm.table_stride + i % prm.max_pages;
    const int id = *entry;
    if (id < live) continue;
    const int to = id < prm.pages ? space.map[id] : -1;
    if (to < 0) report(prm, SVA_DEV_BAD_INDEX);
    *entry = to;
  }
  for (long long task = blockIdx.x; task < (long long)moves * parts; task += gridDim.x) {
    const int k = (int)(task / parts);
    copy_page(prm, space.src[k], space.dst[k], (int)(task % parts), parts);
  }
}

static PoolParams pool_params(const sva_kv_cache_t* c) {
  PoolParams prm = {};
  prm.arrays[0] = (uint8_t*)c->k_codes; prm.arrays[1] = (uint8_t*)c->k_scale; prm.arrays[2] = (uint8_t*)c->k_sf;
  prm.arrays[3] = (uint8_t*)c->v_codes; prm.arrays[4] = (uint8_t*)c->v_scale; prm.arrays[5] = (uint8_t*)c->v_sf;
  const long long rows = (long long)c->H * c->page;
  const bool fp4 = c->format == SVA_CACHE_FP4;
  prm.bytes[0] = rows * (fp4 ? c->d / 2 : c->d);
  prm.bytes[1] = 4LL * (c->format == SVA_CACHE_E4M3_PAGE ? c->H : rows);
  prm.bytes[2] = fp4 ? rows * (c->d / 16) : 0;
  prm.pages = c->pages;
  prm.page = c->page;
  return prm;
}
// slices of a page, half of them K's: as many as make few calls fill the device, down to 4 KB, and none larger than a step
static int page_parts(const PoolParams& prm, long long pages) {
  long long least = (prm.bytes[0] + COPY_EACH * MOVE_THREADS * 16 - 1) / (COPY_EACH * MOVE_THREADS * 16), most = (prm.bytes[0] + 4095) / 4096;
  long long of = pages > 0 ? 148 * 4 / pages : 1;
  of = of < least ? least : of > most ? most : of;
  return 2 * (int)(of < 1 ? 1 : of > 1024 ? 1024 : of);
}
static unsigned grid_rows(int n) { return (unsigned)(n < 65535 ? n : 65535); }

int launch_pages_copy(const sva_kv_cache_t* c, const int32_t* src, const int32_t* dst, int n, int32_t* status, cudaStream_t st) {
  PoolParams prm = pool_params(c);
  prm.from = src; prm.to = dst; prm.n = n; prm.status = status;
  return launch_dep(pages_copy_kernel, dim3((unsigned)page_parts(prm, n), grid_rows(n)), MOVE_THREADS, 0, st, prm);
}

static PoolParams table_params(const sva_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t stride, int rows, int max_pages, int32_t* status) {
  PoolParams prm = pool_params(c);
  prm.refs = refs; prm.table = table; prm.table_stride = stride; prm.rows = rows; prm.max_pages = max_pages; prm.status = status;
  return prm;
}

int launch_pages_take(const sva_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t stride, int rows, int max_pages, const int32_t* lengths,
                      const int32_t* counts, int32_t* status, cudaStream_t st) {
  PoolParams prm = table_params(c, refs, table, stride, rows, max_pages, status);
  prm.lengths = const_cast<int32_t*>(lengths); prm.keep = counts;
  return launch_dep(pages_take_kernel, 1, PLAN_THREADS, 0, st, prm);
}

int launch_pages_fork(const sva_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t stride, int rows, int max_pages, int32_t* lengths,
                      const int32_t* parents, const int32_t* children, int n, int32_t* status, cudaStream_t st) {
  PoolParams prm = table_params(c, refs, table, stride, rows, max_pages, status);
  prm.lengths = lengths; prm.from = parents; prm.to = children; prm.n = n;
  const int rc = launch_dep(pages_fork_plan_kernel, 1, PLAN_THREADS, 0, st, prm);
  return rc ? rc : launch_dep(pages_fork_kernel, dim3((unsigned)page_parts(prm, n) + 1, grid_rows(n)), MOVE_THREADS, 0, st, prm);
}

int launch_pages_free(const sva_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t stride, int rows, int max_pages, int32_t* lengths,
                      const int32_t* which, const int32_t* keep, int n, int32_t* status, cudaStream_t st) {
  PoolParams prm = table_params(c, refs, table, stride, rows, max_pages, status);
  prm.lengths = lengths; prm.to = which; prm.keep = keep; prm.n = n;
  return launch_dep(pages_free_kernel, dim3(1, grid_rows(n)), MOVE_THREADS, 0, st, prm);
}

size_t pages_compact_workspace_bytes(const sva_kv_cache_t* c) { return 16 + 8 * (size_t)((c->pages + 1) / 2) + 4 * (size_t)c->pages; }

int launch_pages_compact(const sva_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t stride, int rows, int max_pages, int32_t* live,
                         int32_t* status, void* ws, cudaStream_t st) {
  PoolParams prm = table_params(c, refs, table, stride, rows, max_pages, status);
  const int rc = launch_dep(pages_compact_plan_kernel, 1, PLAN_THREADS, 0, st, prm, ws, live);
  return rc ? rc : launch_dep(pages_compact_kernel, 148 * 4, MOVE_THREADS, 0, st, prm, ws, page_parts(prm, c->pages));
}

}  // namespace sva
