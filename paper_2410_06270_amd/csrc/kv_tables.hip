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
// What one workgroup does alone: requests, rows (reserve), table entries (release).  A release and a
// reservation: 64 requests, a token each 11.3 us and by two launches each 16.8; 256, 7700 rows 15.6 and 16.9;
// 1024, 8700 rows 19.9 and 17.8; 64, 48000 rows 42 and 17.
constexpr int kTabFused = 1024, kTabRows = 8192, kTabPages = 32768;
// A reservation of few rows by 256 threads, whose barriers meet sooner (by 256 and by 1024, us: 64 requests of a row
// 3.8, 5.6; 256 of a row 4.3, 6.1; 64 of some 15 rows 5.9, 5.6; 256 of some 30 28.5, 11.8; a release 4.7, 3.7).
constexpr int kTabFew = 256, kTabFewRows = 512;
constexpr int kTabHead = 4;              // workspace: the stack's height, pages moved, 2 unused; then S offsets

size_t kv_tables_bytes(int S) { return ((size_t)S + kTabHead) * sizeof(int32_t); }

// x plus the x of the lanes that the DPP control and row mask name (0 where there is none).
template <int CTRL, int ROWS>
__device__ __forceinline__ long long dpp_add(long long x) {
  const unsigned long long b = (unsigned long long)x;
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)b, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(b >> 32), CTRL, ROWS, 0xf, false);
  return x + (long long)(((unsigned long long)hi << 32) | lo);
}

// The inclusive sum over the wave's lanes: within rows of 16, then the rows before.
__device__ __forceinline__ long long wave_scan(long long x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
}

struct Two {
  long long a, b;
};

// The inclusive sums over the workgroup's threads before and with this one, and of all; tmp: a place a wave.
__device__ __forceinline__ Two block_scan(Two x, Two* tmp, Two& all) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  x.a = wave_scan(x.a);
  x.b = wave_scan(x.b);
  __syncthreads();                               // the last call's places have been read
  if ((threadIdx.x & 63) == 63) tmp[wave] = x;
  __syncthreads();
  all = Two{0, 0};
  for (int w = 0; w < waves; ++w) {
    const Two t = tmp[w];
    if (w < wave) {
      x.a += t.a;
      x.b += t.b;
    }
    all.a += t.a;
    all.b += t.b;
  }
  return x;
}

__device__ __forceinline__ int pages_of(int n, int page_log) {
  return (int)(((long long)n + (1 << page_log) - 1) >> page_log);
}

// The largest s in [0, S) with start[s] <= key (0 if there is none), start being in LDS.
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

// The same in memory for keys first + lane, first being wave-uniform: the whole wave finds the first key's,
// and the next 64 starts, which the lanes hold, give the others' (2048 requests: 3 loads one after the
// other for 11).  Every lane of the wave has to take part.
__device__ __forceinline__ int last_of_wave(const int32_t* __restrict__ start, int S, int first) {
  const int lane = threadIdx.x & 63, key = first + lane;
  int base = find_sequence(start, S, first, 1, 0, 1), s = base;
  while (base + 1 < S) {
    const int v = base + 1 + lane < S ? start[base + 1 + lane] : 0x7fffffff;
    // how many of the 64 are at most key (they ascend)
    int n = 0;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
      if (__shfl(v, n + d - 1) <= key) n += d;
    const int end = __builtin_amdgcn_readlane(v, 63);
    s += n == 63 && end <= key ? 64 : n;         // (0 for lanes that have theirs)
    if (end > first + 63) break;
    base += 64;
  }
  return s;
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

// The sums as the second half of a call reads them: offsets of the requests' pages among those that
// move, row starts and lengths.
struct TabSums {
  const int32_t *off, *start, *len;
};

// Pages and rows number i, i + step, ... of a reservation (FUSED: the sums are in LDS; else i - lane is a
// multiple of 64 and wave-uniform, and so is step).
template <bool FUSED>
__device__ __forceinline__ void reserve_fill(const TabArgs& a, const TabSums& t, int height, int total, int i,
                                             int step) {
  const int mask = (1 << a.page_log) - 1;
  const int lane = threadIdx.x & 63;
  for (int p = i; FUSED ? p < total : p - lane < total; p += step) {
    const int s = FUSED ? last_at_most(t.off, a.S, p) : last_of_wave(t.off, a.S, p - lane);
    if (p >= total) continue;
    const int past = t.len[s] - (t.start[s + 1] - t.start[s]);
    a.table[(size_t)s * a.max_pages + pages_of(past, a.page_log) + (p - t.off[s])] = a.free_list[height - 1 - p];
  }
  if (!a.positions && !a.slots) return;
  const int rows = t.start[a.S];
  for (int r = i; FUSED ? r < a.T : r - lane < a.T; r += step) {
    int pos = -1;
    int64_t slot = -1;
    const int s = FUSED ? last_at_most(t.start, a.S, r) : last_of_wave(t.start, a.S, r - lane);
    if (r >= a.T) continue;
    if (r < rows) {
      const int end = t.len[s], next = t.start[s + 1], past = end - (next - t.start[s]);
      pos = end - (next - r);
      // a page that another thread is about to write is read where that one reads it
      const int e = pos >> a.page_log, old = pages_of(past, a.page_log);
      const int32_t* from =
          e < old ? a.table + (size_t)s * a.max_pages + e : a.free_list + (height - 1 - (t.off[s] + e - old));
      slot = ((int64_t)*from << a.page_log) | (pos & mask);
    }
    if (a.positions) a.positions[r] = pos;
    if (a.slots) a.slots[r] = slot;
  }
}

template <bool FUSED>
__device__ __forceinline__ void release_fill(const TabArgs& a, const int32_t* off, int height, int total, int i,
                                             int step) {
  const int lane = threadIdx.x & 63;
  for (int p = i; FUSED ? p < total : p - lane < total; p += step) {
    const int s = FUSED ? last_at_most(off, a.S, p) : last_of_wave(off, a.S, p - lane);
    if (p < total && height + p < a.n_pages) a.free_list[height + p] = a.table[(size_t)s * a.max_pages + (p - off[s])];
  }
}

__device__ __forceinline__ int stack_height(const TabArgs& a) {
  const int n = *a.n_free;
  return n < 0 ? 0 : n > a.n_pages ? a.n_pages : n;
}

// FUSED: the whole call (S <= kTabFused), the sums in LDS; else they are left in the workspace for
// tab_fill_kernel.
template <bool RESERVE, bool FUSED>
__global__ void __launch_bounds__(kTabThreads) tab_scan_kernel(TabArgs a, int32_t* ws) {
  constexpr int N = FUSED ? kTabFused : 1;
  __shared__ Two tmp[kTabThreads / 64];
  __shared__ int32_t s_off[N], s_start[N + 1], s_len[N];
  int32_t* off = FUSED ? s_off : ws + kTabHead;
  const int height = stack_height(a), threads = blockDim.x;
  const int per = FUSED && threads == kTabThreads ? 1 : (a.S + threads - 1) / threads;
  const int s0 = threadIdx.x * per < a.S ? threadIdx.x * per : a.S, s1 = s0 + per < a.S ? s0 + per : a.S;
  const long long most = (long long)a.max_pages << a.page_log;
  // a request that fits its row of the table (and, of a release, has ended)
  auto read = [&](int s, int& past, int& want, int& need) {
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
  // a thread's requests stay in registers, where they are few (2048 requests in 1024 threads)
  constexpr int kHeld = FUSED ? 1 : 4;
  int held[kHeld][3];
  if (per <= kHeld) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (s0 + i < s1) read(s0 + i, held[i][0], held[i][1], held[i][2]);
  }
  int past, want, need;
  auto each = [&](auto f) {
    if (per <= kHeld) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (s0 + i < s1) {
          past = held[i][0];
          want = held[i][1];
          need = held[i][2];
          f(s0 + i);
        }
    } else {
      for (int s = s0; s < s1; ++s) {
        read(s, past, want, need);
        f(s);
      }
    }
  };
  Two mine = {0, 0}, all;
  each([&](int) {
    mine.a += need;
    mine.b += want;
  });
  const Two upto = block_scan(mine, tmp, all);
  const long long P = upto.a - mine.a, R = upto.b - mine.b;
  int total;
  if (RESERVE) {
    // which are granted, and how many rows and pages that makes
    auto granted = [&](long long p, long long r) { return r <= a.T && (need == 0 || p <= height); };
    long long p = P, r = R;
    Two got = {0, 0};
    each([&](int) {
      p += need;
      r += want;
      if (granted(p, r)) {
        got.a += want;
        got.b += need;
      }
    });
    long long start = block_scan(got, tmp, all).a - got.a;
    total = (int)all.b;
    if (threadIdx.x == 0) {
      a.q_start[a.S] = (int)all.a;
      if (FUSED) s_start[a.S] = (int)all.a;
      *a.n_free_out = height - total;
    }
    p = P;
    r = R;
    each([&](int s) {
      off[s] = (int)(p < total ? p : total);     // (those that are not granted any lie behind the last)
      p += need;
      r += want;
      const int n = granted(p, r) ? want : 0;
      a.q_start[s] = (int)start;
      a.kv_len[s] = past + n;
      if (FUSED) {
        s_start[s] = (int)start;
        s_len[s] = past + n;
      }
      start += n;
    });
  } else {
    const long long room = a.n_pages;            // (what is beyond it is not written)
    long long p = P;
    total = (int)(all.a < room ? all.a : room);
    each([&](int s) {
      off[s] = (int)(p < total ? p : total);
      p += need;
      a.kv_len[s] = a.done[s] ? 0 : past;
    });
    if (threadIdx.x == 0) {
      const long long n = height + all.a;
      *a.n_free_out = (int)(n < room ? n : room);
    }
  }
  if (FUSED) {
    __syncthreads();
    if (RESERVE)
      reserve_fill<true>(a, TabSums{s_off, s_start, s_len}, height, total, threadIdx.x, threads);
    else
      release_fill<true>(a, s_off, height, total, threadIdx.x, threads);
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
    reserve_fill<false>(a, TabSums{ws + kTabHead, a.q_start, a.kv_len}, ws[0], ws[1], i, step);
  else
    release_fill<false>(a, ws + kTabHead, ws[0], ws[1], i, step);
}

template <bool RESERVE>
static hipError_t tab_launch(const TabArgs& a, bool fused, void* ws, hipStream_t stream) {
  int32_t* w = static_cast<int32_t*>(ws);
  timing_begin(stream, kSiteKvTables);
  if (fused) {
    const bool few = RESERVE && a.S <= kTabFew && a.T <= kTabFewRows;
    hipLaunchKernelGGL((tab_scan_kernel<RESERVE, true>), dim3(1), dim3(few ? kTabFew : kTabThreads), 0, stream, a, w);
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
