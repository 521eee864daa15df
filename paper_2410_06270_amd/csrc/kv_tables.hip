// kv_tables.hip -- row starts, lengths and page tables of a batch, made on the GPU from the
// requests' lengths; pages come from a stack of free ones and go back to it.
//
// reserve:  need_s = ceil((past_s + want_s) / page) - ceil(past_s / page);  P, R: inclusive sums of
// need and want over the requests that fit their table rows;  granted where R_s <= T and (need_s = 0
// or P_s <= n_free).  P is ascending, so the requests that are granted pages are the first of those
// that need any, and request s takes pages P_s - need_s on from the top of the stack.
// release:  the same sums over the pages that ended requests hold, pushed in order.
//
// A few kilobytes move: all latency.  One workgroup sums (a thread takes S / 1024 neighbouring
// requests) and, where the batch is small, does the rest as well; a second launch with many
// workgroups writes pages, positions and slots of larger ones.
#include "attn.hpp"

namespace mc {

constexpr int kTabThreads = 1024;
constexpr int kTabFused = 1024;          // requests of a call that one workgroup does alone
constexpr int kTabRows = 8192, kTabPages = 65536;        // its rows; its table entries (release)
constexpr int kTabHead = 4;              // workspace: the stack's height, pages moved, 2 unused; then S offsets

size_t kv_tables_bytes(int S) { return ((size_t)S + kTabHead) * sizeof(int32_t); }

// The inclusive sum over the workgroup's threads before and with this one, and of all; tmp: 17 places.
__device__ __forceinline__ long long block_scan(long long x, long long* tmp, long long& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                               // the last call's places have been read
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  long long before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kTabThreads / 64; ++w) {
    const long long t = tmp[w];
    if (w < wave) before += t;
    sum += t;
  }
  all = sum;
  return x + before;
}

__device__ __forceinline__ int pages_of(int n, int page_log) {
  return (int)(((long long)n + (1 << page_log) - 1) >> page_log);
}

// The largest s in [0, S) with start[s] <= key (0 if there is none).
__device__ __forceinline__ int last_at_most(const int32_t* start, int S, int key) {
  int lo = 0, hi = S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= key)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

struct TabArgs {
  const int32_t *want, *past;            // reserve; both
  const uint8_t* done;                   // release
  int32_t* free_list;
  const int32_t* n_free;
  int32_t* n_free_out;
  int n_pages, page_log;
  int32_t *q_start, *kv_len, *table;
  int S, T, max_pages;
  int32_t* positions;
  int64_t* slots;
};

// Pages and rows number i, i + step, ... of a reservation.
__device__ __forceinline__ void reserve_fill(const TabArgs& a, const int32_t* off, int height, int total, int i,
                                             int step) {
  const int mask = (1 << a.page_log) - 1;
  for (int p = i; p < total; p += step) {
    const int s = last_at_most(off, a.S, p);
    const int past = a.kv_len[s] - (a.q_start[s + 1] - a.q_start[s]);
    a.table[(size_t)s * a.max_pages + pages_of(past, a.page_log) + (p - off[s])] = a.free_list[height - 1 - p];
  }
  if (!a.positions && !a.slots) return;
  const int rows = a.q_start[a.S];
  for (int t = i; t < a.T; t += step) {
    int pos = -1;
    int64_t slot = -1;
    if (t < rows) {
      const int s = last_at_most(a.q_start, a.S, t);
      const int end = a.kv_len[s], next = a.q_start[s + 1], past = end - (next - a.q_start[s]);
      pos = end - (next - t);
      // a page that another thread is about to write is read where that one reads it
      const int e = pos >> a.page_log, old = pages_of(past, a.page_log);
      const int page = e < old ? a.table[(size_t)s * a.max_pages + e] : a.free_list[height - 1 - (off[s] + e - old)];
      slot = ((int64_t)page << a.page_log) | (pos & mask);
    }
    if (a.positions) a.positions[t] = pos;
    if (a.slots) a.slots[t] = slot;
  }
}

__device__ __forceinline__ void release_fill(const TabArgs& a, const int32_t* off, int height, int total, int i,
                                             int step) {
  for (int p = i; p < total; p += step) {
    const int s = last_at_most(off, a.S, p);
    if (height + p < a.n_pages) a.free_list[height + p] = a.table[(size_t)s * a.max_pages + (p - off[s])];
  }
}

__device__ __forceinline__ int stack_height(const TabArgs& a) {
  const int n = *a.n_free;
  return n < 0 ? 0 : n > a.n_pages ? a.n_pages : n;
}

// FUSED: the whole call (S <= kTabFused); else the sums, left in the workspace for tab_fill_kernel.
template <bool RESERVE, bool FUSED>
__global__ void __launch_bounds__(kTabThreads) tab_scan_kernel(TabArgs a, int32_t* ws) {
  __shared__ long long tmp[kTabThreads / 64];
  __shared__ int32_t s_off[FUSED ? kTabFused : 1];
  int32_t* off = FUSED ? s_off : ws + kTabHead;
  const int height = stack_height(a);
  const int per = FUSED ? 1 : (a.S + kTabThreads - 1) / kTabThreads;
  const int s0 = threadIdx.x * per < a.S ? threadIdx.x * per : a.S, s1 = s0 + per < a.S ? s0 + per : a.S;
  const long long most = (long long)a.max_pages << a.page_log;
  // a request that fits its row of the table (and, of a release, has ended)
  auto fits = [&](int s, int& past, int& want, int& need) {
    past = a.past[s];
    want = need = 0;
    if (RESERVE) {
      const int w = a.want[s];
      if (w < 0 || past < 0 || (long long)past + w > most) return;
      want = w;
      need = pages_of(past + w, a.page_log) - pages_of(past, a.page_log);
    } else if (a.done[s] && past > 0) {
      need = past > most ? a.max_pages : pages_of(past, a.page_log);
    }
  };
  int past, want, need;
  long long np = 0, nr = 0, all;
  for (int s = s0; s < s1; ++s) {
    fits(s, past, want, need);
    np += need;
    nr += want;
  }
  long long P = block_scan(np, tmp, all) - np;
  int total;
  if (RESERVE) {
    long long R = block_scan(nr, tmp, all) - nr;
    // which are granted, and how many rows and pages that makes
    auto granted = [&](long long p, long long r) { return r <= a.T && (need == 0 || p <= height); };
    long long p = P, r = R, rows = 0, taken = 0;
    for (int s = s0; s < s1; ++s) {
      fits(s, past, want, need);
      p += need;
      r += want;
      if (granted(p, r)) {
        rows += want;
        taken += need;
      }
    }
    long long start = block_scan(rows, tmp, all) - rows;
    if (threadIdx.x == 0) a.q_start[a.S] = (int)all;
    block_scan(taken, tmp, all);
    total = (int)all;
    p = P;
    r = R;
    for (int s = s0; s < s1; ++s) {
      fits(s, past, want, need);
      off[s] = (int)(p < total ? p : total);     // (those that are not granted any lie behind the last)
      p += need;
      r += want;
      const int n = granted(p, r) ? want : 0;
      a.q_start[s] = (int)start;
      a.kv_len[s] = past + n;
      start += n;
    }
    if (threadIdx.x == 0) *a.n_free_out = height - total;
  } else {
    const long long room = a.n_pages;            // (what is beyond it is not written)
    total = (int)(all < room ? all : room);
    for (int s = s0; s < s1; ++s) {
      fits(s, past, want, need);
      off[s] = (int)(P < total ? P : total);
      P += need;
      a.kv_len[s] = a.done[s] ? 0 : past;
    }
    if (threadIdx.x == 0) {
      const long long n = height + all;
      *a.n_free_out = (int)(n < room ? n : room);
    }
  }
  if (FUSED) {
    __syncthreads();
    if (RESERVE)
      reserve_fill(a, off, height, total, threadIdx.x, kTabThreads);
    else
      release_fill(a, off, height, total, threadIdx.x, kTabThreads);
  } else if (threadIdx.x == 0) {
    ws[0] = height;
    ws[1] = total;
  }
}

constexpr int kTabFillThreads = 256;

template <bool RESERVE>
__global__ void __launch_bounds__(kTabFillThreads) tab_fill_kernel(TabArgs a, const int32_t* __restrict__ ws) {
  const int i = blockIdx.x * kTabFillThreads + threadIdx.x, step = gridDim.x * kTabFillThreads;
  if (RESERVE)
    reserve_fill(a, ws + kTabHead, ws[0], ws[1], i, step);
  else
    release_fill(a, ws + kTabHead, ws[0], ws[1], i, step);
}

template <bool RESERVE>
static hipError_t tab_launch(const TabArgs& a, bool fused, void* ws, hipStream_t stream) {
  int32_t* w = static_cast<int32_t*>(ws);
  timing_begin(stream, kSiteKvTables);
  if (fused) {
    hipLaunchKernelGGL((tab_scan_kernel<RESERVE, true>), dim3(1), dim3(kTabThreads), 0, stream, a, w);
  } else {
    hipLaunchKernelGGL((tab_scan_kernel<RESERVE, false>), dim3(1), dim3(kTabThreads), 0, stream, a, w);
    hipLaunchKernelGGL(tab_fill_kernel<RESERVE>, dim3(256), dim3(kTabFillThreads), 0, stream, a, w);
  }
  timing_end(stream, kSiteKvTables);
  return hipGetLastError();
}

hipError_t launch_kv_reserve(const int32_t* want, const int32_t* past, const PoolArgs& p, const BatchOut& b,
                             int32_t* positions, int64_t* slots, void* ws, hipStream_t stream) {
  const TabArgs a = {want, past, nullptr, p.free_list, p.n_free, p.n_free_out, p.n_pages, p.page_log, b.q_start,
                     b.kv_len, b.page_table, b.S, b.T, b.max_pages, positions, slots};
  return tab_launch<true>(a, b.S <= kTabFused && b.T <= kTabRows, ws, stream);
}

hipError_t launch_kv_release(const uint8_t* done, const int32_t* past, const PoolArgs& p, const BatchOut& b, void* ws,
                             hipStream_t stream) {
  const TabArgs a = {nullptr, past, done, p.free_list, p.n_free, p.n_free_out, p.n_pages, p.page_log, nullptr,
                     b.kv_len, b.page_table, b.S, 0, b.max_pages, nullptr, nullptr};
  return tab_launch<false>(a, b.S <= kTabFused && (long long)b.S * b.max_pages <= kTabPages, ws, stream);
}

}  // namespace mc
