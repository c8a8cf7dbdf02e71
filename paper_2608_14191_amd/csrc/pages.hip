// Page tables on the device: fork, free, reserve, compact and copy.
//
// Whole numbers and moved bytes only.  Counts change by atomic additions, whose order does not
// matter; which free page goes where follows from prefix sums in the order of the pages and the
// rows, taken by one workgroup (a table's bookkeeping is a few thousand numbers, and its time
// that of a few dependent memory accesses).  Copies are bound by memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace aatc {
namespace {

constexpr int kListThreads = 256;
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
// Pages per thread and step of a scan: four where one step has the whole pool then (all waves share
// it), else sixteen (fewer steps).
constexpr int kFewPages = 4, kManyPages = 16;

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Exclusive prefix sum of v over a workgroup of kPlanThreads; total in `sum`.  (Two barriers:
// the scratch is free again at the return.)
__device__ inline int block_scan(int v, int& sum, int* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    incl += lane >= o ? up : 0;
  }
  if (lane == 63) scratch[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? scratch[w] : 0;
    all += scratch[w];
  }
  __syncthreads();
  sum = all;
  return before + incl - v;
}

// The pages of a step, in order: wave, then k, then lane (64 consecutive ones an access).
template <int PP>
__device__ inline int64_t plan_page(int64_t base, int k) {
  return base + (int64_t)(threadIdx.x >> 6) * (64 * PP) + k * 64 + (threadIdx.x & 63);
}

// Marked pages of a step (flag(k)): calls take(rank, k) for each of this thread's, ranks counted
// from `first` in the pages' order, and returns how many the workgroup has.  Two barriers.
template <int PP, class Flag, class Take>
__device__ inline int rank_pages(int first, int* scratch, Flag flag, Take take) {
  const int wave = threadIdx.x >> 6;
  uint64_t marks[PP];
  int mine = 0;
#pragma unroll
  for (int k = 0; k < PP; ++k) {
    marks[k] = __builtin_amdgcn_ballot_w64(flag(k));
    mine += __popcll(marks[k]);
  }
  if ((threadIdx.x & 63) == 0) scratch[wave] = mine;
  __syncthreads();
  int before = first, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? scratch[w] : 0;
    all += scratch[w];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PP; ++k) {
    const uint64_t bit = (uint64_t)1 << (threadIdx.x & 63);
    if (marks[k] & bit) take(before + __popcll(marks[k] & (bit - 1)), k);
    before += __popcll(marks[k]);
  }
  return all;
}

// ---------------------------------------------------------------------------------------
// Fork: a workgroup per pair.
__global__ __launch_bounds__(kListThreads) void fork_kernel(
    const int32_t* __restrict__ src, int64_t src_stride, int src_rows, int32_t* __restrict__ dst,
    int64_t dst_stride, int dst_rows, int entries, int32_t* __restrict__ ref, int n_pages,
    const int32_t* __restrict__ pairs, int64_t n) {
  const int64_t i = blockIdx.x;
  const int from = pairs[2 * i], to = pairs[2 * i + 1];
  if (from < 0 || from >= src_rows || to < 0 || to >= dst_rows) return;      // (uniform)
  // A later pair with the same destination (and a source that exists) takes it.
  int later = 0;
  for (int64_t j = i + 1 + threadIdx.x; j < n; j += kListThreads)
    later |= pairs[2 * j + 1] == to && pairs[2 * j] >= 0 && pairs[2 * j] < src_rows;
  if (__syncthreads_or(later)) return;
  for (int e = threadIdx.x; e < entries; e += kListThreads) {
    const int page = src[from * src_stride + e];
    dst[to * dst_stride + e] = page;
    if (page >= 0 && page < n_pages) atomicAdd(&ref[page], 1);
  }
}

// Free: a workgroup per listed row; the exchange gives each entry to one of the workgroups that
// a row listed twice has.
__global__ __launch_bounds__(kListThreads) void free_kernel(int32_t* table, int64_t stride,
                                                            int rows, int entries, int32_t* ref,
                                                            int n_pages,
                                                            const int32_t* __restrict__ list) {
  const int row = list[blockIdx.x];
  if (row < 0 || row >= rows) return;
  for (int e = threadIdx.x; e < entries; e += kListThreads) {
    const int page = atomicExch(&table[row * stride + e], -1);
    if (page >= 0 && page < n_pages) atomicAdd(&ref[page], -1);
  }
}

// ---------------------------------------------------------------------------------------
// Reserve: one workgroup.  A row's claims are the entries that its new tokens fall into, the begun
// page first where there is one; claims are numbered row after row, entry after entry.  A claim wants
// a free page where its entry names none (a begun one then gets none), or one that other entries
// name too, unless all of those are earlier claims that leave it.  Wants get their places in the list
// of free pages in the order of the claims.
//
// The rows' first claims, the wants and the free pages are in LDS as far as they fit (the round trips
// to memory are the time), else in the workspace, which also counts the earlier claims of a page over
// several steps.  Where no row has two claims (a decode step) claim i is row i's; else they are
// numbered by a scan and found by a search, four a thread and step where they are many.  64 rows of a
// new page each in a pool of 4096 5.6 us (6.3 with the scan and the search), 8192 pages of one row
// 19.0 (24.5 with one claim a thread and step).
struct ReserveSpace {
  int32_t *first, *row, *entry, *free;
};
__host__ __device__ inline ReserveSpace reserve_space(void* ws, int64_t rows, int64_t n_pages) {
  auto* p = static_cast<int32_t*>(ws);
  return {p, p + rows, p + rows + n_pages, p + rows + 2 * n_pages};
}
constexpr int kListLds = 2048;
constexpr int kManyClaims = 4;                  // a thread and step
constexpr int kBegun = 1 << 30;                 // of a want's entry (below 2^30): the row's begun page,
constexpr int kShared = (int)(1u << 31);        // a page that others keep

template <int PP>
__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(
    int32_t* table, int64_t stride, int rows, int32_t* ref, int n_pages, int shift, int len_max,
    const int32_t* __restrict__ held, const int32_t* __restrict__ wanted, int32_t* pairs,
    int32_t* lacking, void* ws) {
  __shared__ int scratch[kPlanWaves];
  __shared__ int chunk[kPlanThreads * kManyClaims], first_s[kPlanThreads], from_s[kPlanThreads];
  __shared__ int row_s[kListLds], entry_s[kListLds], free_s[kListLds];
  const int tid = threadIdx.x;
  const ReserveSpace sp = reserve_space(ws, rows, n_pages);
  const bool small = rows <= kPlanThreads;
  const int mask = (1 << shift) - 1;
  // Row r: tokens from .. to - 1 to come, and its claims.
  auto length = [&](const int32_t* list, int r) { return min(max(list[r], 0), len_max); };
  struct Row {
    int from, claims;
  };
  auto row_of = [&](int r) {
    if (r >= rows) return Row{0, 0};
    const int from = length(held, r), to = length(wanted, r);
    return Row{from, to > from ? ((to + mask) >> shift) - (from >> shift) : 0};
  };
  // The free ones of this thread's pages of a step, a bit each (the first step's are read now).
  auto open_pages = [&](int64_t base) {
    unsigned open = 0;
#pragma unroll
    for (int k = 0; k < PP; ++k) {
      const int64_t p = plan_page<PP>(base, k);
      if (p < n_pages && ref[p] <= 0) open |= 1u << k;
    }
    return open;
  };
  const unsigned open0 = open_pages(0);
  // (1) The rows' claims.
  const Row row0 = row_of(tid);
  int more = row0.claims > 1;
  for (int r = tid; r < rows; r += kPlanThreads) {
    if (r != tid) more |= row_of(r).claims > 1;
    pairs[2 * r] = -1;
    pairs[2 * r + 1] = -1;
  }
  const bool one = !__syncthreads_or(more);     // claim i is row i's (some have none)
  int claims = one ? rows : 0;
  if (!one)
    for (int base = 0; base < rows; base += kPlanThreads) {
      const int r = base + tid;
      const Row w = base == 0 ? row0 : row_of(r);
      int sum = 0;
      const int first = claims + block_scan(w.claims, sum, scratch);
      if (r < rows) {
        if (small) {
          first_s[r] = first;
          from_s[r] = w.from;
        } else {
          sp.first[r] = first;
        }
      }
      claims += sum;
    }
  // (2) What they want.  `earlier`, in the place of the free pages' list: claims of each shared page
  // in the steps before.
  int32_t* earlier = sp.free;
  const bool many = !one && claims > kPlanThreads;
  const int step = kPlanThreads * (many ? kManyClaims : 1);
  const bool steps = claims > step;
  if (steps)
    for (int64_t p = tid; p < n_pages; p += kPlanThreads)
      __hip_atomic_store(&earlier[p], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __builtin_amdgcn_s_waitcnt(0);                // (a barrier does not wait for stores)
  __syncthreads();
  auto wants_of = [&](auto per, int base, int demand) {
    constexpr int K = decltype(per)::value;
    int row[K], entry[K], page[K], count[K];    // (entry: with kBegun, and kShared later)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = (int)plan_page<K>(base, k);
      bool on = i < claims;
      int r, from, at;                          // its `at`th claim
      if (one) {
        const Row w = base == 0 ? row0 : row_of(i);
        r = min(i, rows - 1), from = w.from, at = 0;
        on = w.claims > 0;
      } else {
        const int x = min(i, claims - 1);
        r = 0;
        int hi = rows - 1, first = small ? first_s[0] : sp.first[0];
        while (r < hi) {                        // the last row whose claims begin at or before x
          const int mid = (r + hi + 1) / 2, f = small ? first_s[mid] : sp.first[mid];
          if (f <= x) r = mid, first = f;
          else hi = mid - 1;
        }
        from = small ? from_s[r] : length(held, r);
        at = x - first;
      }
      row[k] = r;
      entry[k] = on ? (from >> shift) + at : 0;
      page[k] = table[r * stride + entry[k]];
      page[k] = on && page[k] >= 0 && page[k] < n_pages ? page[k] : -1;
      entry[k] |= at == 0 && (from & mask) != 0 ? kBegun : 0;
      row[k] = on ? r : -1;
    }
    int shared = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = ref[max(page[k], 0)];
      count[k] = page[k] >= 0 ? c : 0;
      shared |= count[k] > 1;
    }
    if (__syncthreads_or(shared)) {             // pages that others name too: who leaves them?
#pragma unroll
      for (int k = 0; k < K; ++k) chunk[(int)plan_page<K>(0, k)] = count[k] > 1 ? page[k] : -1;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (count[k] <= 1) continue;
        int before = steps ? __hip_atomic_load(&earlier[page[k]], __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT)
                           : 0;
        const int upto = (int)plan_page<K>(0, k);
#pragma unroll 8
        for (int j = 0; j < upto; ++j) before += chunk[j] == page[k];
        if (count[k] - before > 1) entry[k] |= kShared;
      }
      __syncthreads();                          // (the counts are read)
      if (steps) {
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (count[k] > 1)
            __hip_atomic_fetch_add(&earlier[page[k]], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_s_waitcnt(0);          // (the barriers below come before the next step)
      }
    }
    return rank_pages<K>(demand, scratch, [&](int k) {
      return row[k] >= 0 && ((entry[k] & kShared) != 0 || ((entry[k] & kBegun) == 0 && count[k] <= 0));
    }, [&](int rank, int k) {
      if (rank >= n_pages) return;              // (more than there can be)
      if (rank < kListLds) {
        row_s[rank] = row[k];
        entry_s[rank] = entry[k];
      } else {
        sp.row[rank] = row[k];
        sp.entry[rank] = entry[k];
      }
    });
  };
  int demand = 0;
  for (int base = 0; base < claims; base += step)
    demand += many ? wants_of(std::integral_constant<int, kManyClaims>{}, base, demand)
                   : wants_of(std::integral_constant<int, 1>{}, base, demand);
  __syncthreads();                              // (`earlier` is read: the free pages go there)
  // (3) The lowest free pages, as many.
  int found = 0;
  for (int64_t base = 0; base < n_pages && found < demand; base += kPlanThreads * PP) {
    const unsigned open = base == 0 ? open0 : open_pages(base);
    found += rank_pages<PP>(found, scratch, [&](int k) { return (open >> k & 1u) != 0u; },
                        [&](int rank, int k) {
                          if (rank >= demand) return;
                          const int page = (int)plan_page<PP>(base, k);
                          if (rank < kListLds) free_s[rank] = page;
                          else sp.free[rank] = page;
                        });
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();                              // (the lists are this workgroup's own)
  const bool enough = found >= demand;
  if (tid == 0) *lacking = enough ? 0 : demand - found;
  if (!enough) return;
  // (4) Hand out.
  for (int i = tid; i < demand; i += kPlanThreads) {
    const bool lds = i < kListLds;
    const int row = lds ? row_s[i] : sp.row[i], e = lds ? entry_s[i] : sp.entry[i];
    const int now = lds ? free_s[i] : sp.free[i];
    int32_t* at = table + row * stride + (e & (kBegun - 1));
    const int old = e & kShared ? *at : -1;
    *at = now;
    ref[now] = 1;
    if (old >= 0) atomicAdd(&ref[old], -1);
    if (e & kBegun) {
      pairs[2 * row] = old;
      pairs[2 * row + 1] = now;
    }
  }
}

// ---------------------------------------------------------------------------------------
// Compact: where each page goes (one workgroup), then the table (all of them).  Workspace: the
// new place of every page.
template <int PP>
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(const int32_t* ref,
                                                                    int n_pages, int32_t* ref_out,
                                                                    int32_t* pairs,
                                                                    int32_t* moves, int32_t* to) {
  __shared__ int scratch[kPlanWaves];
  const int tid = threadIdx.x;
  constexpr int kStep = kPlanThreads * PP;
  int live = 0;
  for (int64_t base = 0; base < n_pages; base += kStep)
    live += rank_pages<PP>(0, scratch, [&](int k) {
      const int64_t p = plan_page<PP>(base, k);
      return p < n_pages && ref[p] > 0;
    }, [](int, int) {});
  // Pages in use from `live` on, and free ones below it: as many of one as of the other.  (ref_out
  // may be ref: no count is written before all of its own step are read.)
  int movers = 0, holes = 0;
  for (int64_t base = 0; base < n_pages; base += kStep) {
    int count[PP];
#pragma unroll
    for (int k = 0; k < PP; ++k) {
      const int64_t p = plan_page<PP>(base, k);
      count[k] = p < n_pages ? ref[p] : 0;
    }
#pragma unroll
    for (int k = 0; k < PP; ++k) {
      const int64_t p = plan_page<PP>(base, k);
      if (p >= n_pages) continue;
      to[p] = (int)p;
      if (ref_out != ref) ref_out[p] = p < live ? count[k] : 0;
    }
    movers += rank_pages<PP>(movers, scratch, [&](int k) {
      return count[k] > 0 && plan_page<PP>(base, k) >= live;
    }, [&](int rank, int k) { pairs[2 * rank] = (int)plan_page<PP>(base, k); });
    holes += rank_pages<PP>(holes, scratch, [&](int k) {
      return count[k] <= 0 && plan_page<PP>(base, k) < live;
    }, [&](int rank, int k) { pairs[2 * rank + 1] = (int)plan_page<PP>(base, k); });
  }
  __syncthreads();
  if (tid == 0) *moves = movers;
  for (int64_t i = tid; i < n_pages / 2; i += kPlanThreads) {
    if (i < movers) {
      const int from = pairs[2 * i], dst = pairs[2 * i + 1];
      to[from] = dst;
      ref_out[dst] = ref[from];
      if (ref_out == ref) ref_out[from] = 0;
    } else {
      pairs[2 * i] = -1;
      pairs[2 * i + 1] = -1;
    }
  }
}

__global__ __launch_bounds__(kListThreads) void compact_table_kernel(
    const int32_t* table, int64_t stride, int rows, int entries, int32_t* out, int64_t out_stride,
    int n_pages, const int32_t* __restrict__ to) {
  const int64_t all = (int64_t)rows * entries;
  for (int64_t i = (int64_t)blockIdx.x * kListThreads + threadIdx.x; i < all;
       i += (int64_t)gridDim.x * kListThreads) {
    const int64_t r = i / entries, e = i - r * entries;
    const int page = table[r * stride + e];
    out[r * out_stride + e] = page >= 0 && page < n_pages ? to[page] : page;
  }
}

// ---------------------------------------------------------------------------------------
// Copy: 16 bytes a thread and step, workgroups over (pair, pool, piece of the page).
constexpr int kCopyUnroll = 4;
constexpr int64_t kCopyPiece = 16 * kListThreads * kCopyUnroll;

// FAR: past the caches (copies that would not stay in them: 2048 pages of 32 KiB in eight pools
// 212.5 us, 218.4 through the caches; 128 copies of pages of 64 KiB that children share, in sixteen
// pools, with the three launches before them 58.2, 51.9 through them).  All listed pairs count,
// whether they copy or not: how many do, only the device knows.
constexpr int64_t kFarBytes = (int64_t)512 << 20;
template <bool FAR>
__global__ __launch_bounds__(kListThreads) void copy_kernel(char* base, int64_t n_pools,
                                                            int64_t pool_stride, int n_pages,
                                                            int64_t page_bytes,
                                                            const int32_t* __restrict__ pairs,
                                                            int64_t n, const int32_t* n_dev) {
  const int64_t pieces = (page_bytes + kCopyPiece - 1) / kCopyPiece;
  const int64_t count = n_dev ? min((int64_t)max(*n_dev, 0), n) : n;
  const int64_t all = count * n_pools * pieces;
  for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
    const int64_t piece = w % pieces, rest = w / pieces;
    const int64_t pool = rest % n_pools, i = rest / n_pools;
    const int from = pairs[2 * i], to = pairs[2 * i + 1];
    if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) continue;
    const char* s = base + pool * pool_stride + from * page_bytes;
    char* d = base + pool * pool_stride + to * page_bytes;
    v4u x[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
      const int64_t o = piece * kCopyPiece + 16 * (u * kListThreads + threadIdx.x);
      const v4u* p = reinterpret_cast<const v4u*>(s + o);
      if (o < page_bytes) x[u] = FAR ? __builtin_nontemporal_load(p) : *p;
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
      const int64_t o = piece * kCopyPiece + 16 * (u * kListThreads + threadIdx.x);
      if (o >= page_bytes) continue;
      if constexpr (FAR) __builtin_nontemporal_store(x[u], reinterpret_cast<v4u*>(d + o));
      else *reinterpret_cast<v4u*>(d + o) = x[u];
    }
  }
}

aatc_status done() { return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE; }

int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

}  // namespace

aatc_status launch_pages_copy(void* base, int64_t n_pools, int64_t pool_stride, int64_t n_pages,
                              int64_t page_bytes, const int32_t* pairs, int64_t n,
                              const int32_t* n_dev, void* stream) {
  const int64_t pieces = (page_bytes + kCopyPiece - 1) / kCopyPiece;
  // At most 2^14 workgroups, which then take several pieces each.
  const int64_t cap = (int64_t)1 << 14;
  const int64_t grid = n > cap || pieces > cap ? cap : std::min(cap, n * n_pools * pieces);
  const bool far = 2.0 * (double)n * (double)n_pools * (double)page_bytes > (double)kFarBytes;
  hipLaunchKernelGGL(far ? copy_kernel<true> : copy_kernel<false>, dim3((unsigned)grid),
                     dim3(kListThreads), 0, (hipStream_t)stream, static_cast<char*>(base), n_pools,
                     pool_stride, (int)n_pages, page_bytes, pairs, n, n_dev);
  return done();
}

aatc_status launch_pages_fork(const aatc_page_table& src, const aatc_page_table& dst,
                              int32_t* ref, int64_t n_pages, const int32_t* pairs, int64_t n,
                              void* stream) {
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)n), dim3(kListThreads), 0, (hipStream_t)stream,
                     src.table, src.stride, src.rows, dst.table, dst.stride, dst.rows,
                     src.max_pages, ref, (int)n_pages, pairs, n);
  return done();
}

aatc_status launch_pages_free(const aatc_page_table& t, int32_t* ref, int64_t n_pages,
                              const int32_t* rows, int64_t n, void* stream) {
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)n), dim3(kListThreads), 0, (hipStream_t)stream,
                     t.table, t.stride, t.rows, t.max_pages, ref, (int)n_pages, rows);
  return done();
}

size_t pages_workspace_bytes(int64_t rows, int64_t n_pages) {
  return (size_t)(rows + 3 * n_pages) * sizeof(int32_t);       // (ReserveSpace; a compaction: n_pages)
}

aatc_status launch_pages_reserve(const aatc_page_table& t, int32_t* ref, int64_t n_pages,
                                 int page_tokens, const int32_t* held, const int32_t* wanted,
                                 int32_t* pairs, int32_t* lacking, void* workspace, void* stream) {
  const int64_t most = (int64_t)t.max_pages * page_tokens;
  const int len_max = (int)std::min<int64_t>(most, INT32_MAX - kMaxPage);
  const bool few = n_pages <= kPlanThreads * kFewPages;
  hipLaunchKernelGGL(few ? reserve_kernel<kFewPages> : reserve_kernel<kManyPages>, dim3(1),
                     dim3(kPlanThreads), 0, (hipStream_t)stream, t.table, t.stride, t.rows, ref,
                     (int)n_pages, log2_of(page_tokens), len_max, held, wanted, pairs, lacking,
                     workspace);
  return done();
}

aatc_status launch_pages_compact(const aatc_page_table& t, const int32_t* ref, int64_t n_pages,
                                 const aatc_page_table& t_out, int32_t* ref_out, int32_t* pairs,
                                 int32_t* moves, void* workspace, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  auto* to = static_cast<int32_t*>(workspace);
  const bool few = n_pages <= kPlanThreads * kFewPages;
  hipLaunchKernelGGL(few ? compact_plan_kernel<kFewPages> : compact_plan_kernel<kManyPages>, dim3(1),
                     dim3(kPlanThreads), 0, st, ref, (int)n_pages, ref_out, pairs, moves, to);
  if (hipGetLastError() != hipSuccess) return AATC_E_DEVICE;
  const int64_t all = (int64_t)t.rows * t.max_pages;
  const int64_t grid = std::min<int64_t>((all + kListThreads - 1) / kListThreads, 2048);
  hipLaunchKernelGGL(compact_table_kernel, dim3((unsigned)grid), dim3(kListThreads), 0, st,
                     t.table, t.stride, t.rows, t.max_pages, t_out.table, t_out.stride,
                     (int)n_pages, to);
  return done();
}

}  // namespace aatc
