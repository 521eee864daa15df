// attn_select.hip -- bounds on the keys of a page, and the pages that each query attends to.
//
//   bounds of a page and key-value head:  s = max |k| / 127 (times the fp32 number nearest to 1/127),
//   hi = ceil(max_t k / s),  lo = floor(min_t k / s)
//   score of a page for a row:  max over the group's heads of (sq s) sum_i (q8_i > 0 ? q8_i hi_i : q8_i lo_i)
// with q8 = rint(q / sq), sq = max |q| / 127: no key of the page has a larger product with the
// rounded query.  All sums are of whole numbers below 2^24 and so exact in any order; what is rounded
// is one product, the same in any implementation, and so is the selection.
//
// kv_summary_kernel: one workgroup a touched page and head.  page_score_kernel: the products of 16
// pages with 16 (row, head) columns are 2 D / 64 matrix instructions on bytes; negative parts of the
// query go with lo, positive ones with hi.  page_select_kernel: one workgroup a row and head finds the
// n-th largest score digit by digit and lists what is above it, and of its equals the first.
#include "attn.hpp"

namespace mc {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;

constexpr float k127th = 1.0f / 127.0f;

// ----------------------------------------------------------------- summary --
constexpr int kSumThreads = 256;

// Pages that n new tokens from q_start on touch: (n + page - 2) / page + 1 at most; sequence s owns
// the slots from floor(q_start[s] / page) + 2 s on, at least floor(n / page) + 2 of them.
template <int D, int KV>
__global__ void __launch_bounds__(kSumThreads) kv_summary_kernel(BatchArgs b, KvArgs c, SummaryArgs sm) {
  constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  constexpr int U = E2 ? 32 : E4 ? 16 : 8, kUnits = D / U, kLanes = 16 * kUnits, kTeams = kSumThreads / kLanes;
  constexpr int kBlockBytes = KvFormat<D, KV>::kBlockBytes;
  __shared__ float s_lo[kTeams][D], s_hi[kTeams][D];
  __shared__ float s_most[kSumThreads / 64];
  const int hk = blockIdx.x % c.Hkv, slot = blockIdx.x / c.Hkv;
  const int page_log = c.lb + 4;
  int s, page;
  if (b.q_start) {
    s = find_sequence(b.q_start, b.S, slot, 1 << page_log, 2, 1);
    const long long first = b.q_start[s], n = (long long)b.q_start[s + 1] - first;
    const long long group = slot - ((first >> page_log) + 2ll * s), p0 = (long long)b.kv_len[s] - n;
    if (n <= 0 || group < 0) return;
    const long long at = ((p0 > 0 ? p0 : 0) >> page_log) + group;
    if (at << page_log >= kv_length(c, b, s)) return;
    page = (int)at;
  } else {
    s = slot;
    const int len = kv_length(c, b, s);
    if (len == 0) return;
    page = (len - 1) >> page_log;
  }
  const int held = min(kv_length(c, b, s) - (page << page_log), 1 << page_log);
  const int number = b.page_table[(size_t)s * b.max_pages + page];
  if (number < 0 || number >= c.n_pages) return;

  // thread (team, unit, token): a unit of its token in every kTeams-th block
  const int team = threadIdx.x / kLanes, in = threadIdx.x % kLanes, unit = in >> 4, t = in & 15;
  float lo[U], hi[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    lo[i] = -kNegInf;
    hi[i] = kNegInf;
  }
  for (int blk = team; 16 * blk < held; blk += kTeams) {
    if (16 * blk + t >= held) continue;
    const char* kp = c.k + kv_block_offset<kBlockBytes>(c, number, hk, blk) + unit * 256 + t * 16;
    const u32x4 w = *reinterpret_cast<const u32x4*>(kp);
    float scale = 1.0f;
    if (E2)
      scale = __uint_as_float((uint32_t)(uint8_t)c.k[kv_scale_offset<D>(c, number, hk, blk) + 16 * unit + 4 * (t & 3) +
                                                     (t >> 2)]
                              << 23);
#pragma unroll
    for (int g = 0; g < U / 8; ++g) {
      const u32x4 x = E2 ? e2m1_to_bf16(w[g], scale) : E4 ? e4m3_to_bf16(w[2 * (g & 1)], w[2 * (g & 1) + 1]) : w;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = half_of(x[i / 2], i & 1);
        const bool number_ok = fabsf(v) < -kNegInf;      // (neither NaN nor infinite)
        lo[8 * g + i] = fminf(lo[8 * g + i], number_ok ? v : -kNegInf);
        hi[8 * g + i] = fmaxf(hi[8 * g + i], number_ok ? v : kNegInf);
      }
    }
  }
  // over the 16 tokens
#pragma unroll
  for (int i = 0; i < U; ++i) {
    float x = lo[i], y = hi[i];
    x = fminf(x, dpp<0xb1>(x));
    x = fminf(x, dpp<0x4e>(x));
    x = fminf(x, dpp<0x141>(x));
    x = fminf(x, dpp<0x140>(x));
    y = fmaxf(y, dpp<0xb1>(y));
    y = fmaxf(y, dpp<0x4e>(y));
    y = fmaxf(y, dpp<0x141>(y));
    y = fmaxf(y, dpp<0x140>(y));
    if (t == (i & 15)) {
      s_lo[team][unit * U + i] = x;
      s_hi[team][unit * U + i] = y;
    }
  }
  __syncthreads();
  const int d = threadIdx.x;
  float x = 0.0f, y = 0.0f, most = 0.0f;
  if (d < D) {
    x = s_lo[0][d];
    y = s_hi[0][d];
#pragma unroll
    for (int i = 1; i < kTeams; ++i) {
      x = fminf(x, s_lo[i][d]);
      y = fmaxf(y, s_hi[i][d]);
    }
    if (x > y) x = y = 0.0f;                     // no number among the keys
    most = fmaxf(fabsf(x), fabsf(y));
  }
  most = wave_max(most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  __syncthreads();
  if (d >= D) return;
  most = s_most[0];
#pragma unroll
  for (int i = 1; i < D / 64; ++i) most = fmaxf(most, s_most[i]);
  const float scale = most * k127th, by = scale > 0.0f ? scale : 1.0f;
  auto bounded = [](float v) { return (int8_t)(v > 127.0f ? 127.0f : v < -127.0f ? -127.0f : v); };
  const size_t at = (size_t)number * c.Hkv + hk;
  sm.bounds[at * 2 * D + d] = bounded(floorf(x / by));      // IEEE divisions
  sm.bounds[at * 2 * D + D + d] = bounded(ceilf(y / by));
  if (d == 0) sm.scale[at] = scale;
}

hipError_t launch_kv_summarize(int D, const BatchArgs& b, const KvArgs& c, const SummaryArgs& sm, hipStream_t stream) {
  const int slots = b.q_start ? (b.T >> (c.lb + 4)) + 2 * b.S : b.S;
  const dim3 grid((unsigned)((size_t)slots * c.Hkv));
  timing_begin(stream, kSiteKvSummary);
  with_kv_kind(c, [&](auto kind) {
    constexpr int KV = decltype(kind)::value;
    if (D == 64)
      hipLaunchKernelGGL((kv_summary_kernel<64, KV>), grid, dim3(kSumThreads), 0, stream, b, c, sm);
    else
      hipLaunchKernelGGL((kv_summary_kernel<128, KV>), grid, dim3(kSumThreads), 0, stream, b, c, sm);
  });
  timing_end(stream, kSiteKvSummary);
  return hipGetLastError();
}

// ------------------------------------------------------------------ scores --
constexpr int kScoreThreads = 256;
constexpr int kScoreCols = 16;           // (row, head) columns of a product
constexpr int kScorePages = 256;         // pages of a workgroup, a quarter of them a wave's

// Rows of a workgroup: those whose heads fill the columns.
__host__ __device__ static inline int score_rows(int g) { return g >= kScoreCols ? 1 : kScoreCols / g; }

// Pages [lo, hi] that a row at position pos may take.
__device__ __forceinline__ void page_range(const SelectArgs& a, int pos, int page_log, int& lo, int& hi) {
  hi = pos >> page_log;
  lo = a.window > 0 && pos >= a.window ? (pos - a.window + 1) >> page_log : 0;
}

// The sequence and position of row t (-1: padding, or a row that sees nothing).
__device__ __forceinline__ int row_position(const BatchArgs& b, const KvArgs& c, int t, int& s) {
  if (!b.q_start) {
    s = t;
    return kv_length(c, b, s) - 1;
  }
  s = find_sequence(b.q_start, b.S, t, 1, 0, 1);
  if (t < b.q_start[s] || t >= b.q_start[s + 1]) return -1;
  const long long pos = (long long)b.kv_len[s] - ((long long)b.q_start[s + 1] - t);
  const int len = kv_length(c, b, s);
  return pos < 0 || len == 0 ? -1 : pos < len ? (int)pos : len - 1;
}

// Workspace: scores [row - row0][Hkv][pages], pages the row length of the tables.
template <int D>
__global__ void __launch_bounds__(kScoreThreads)
    page_score_kernel(RowsIn q, BatchArgs b, KvArgs c, SummaryArgs sm, SelectArgs a, int row0, int row1, int chunks,
                      float* __restrict__ scores) {
  constexpr int NV = D / 64;
  __shared__ float s_part[kScoreThreads / 64][16][kScoreCols + 1];
  const int lane = threadIdx.x & 63, wave = wave_id(), n = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int chunk = id % chunks;
  id /= chunks;
  const int hk = id % c.Hkv, slot = id / c.Hkv, R = score_rows(a.g), page_log = c.lb + 4;
  // rows first, ..., first + rows - 1, of one sequence
  int s, first, rows;
  if (b.q_start) {
    s = find_sequence(b.q_start, b.S, slot, R, 1, 1);
    int start, count;
    sequence_rows(b, s, start, count);
    const long long at = ((long long)slot - ((long long)b.q_start[s] / R + s)) * R;
    if (at < 0 || at >= count) return;
    first = start + (int)at;
    rows = min(R, count - (int)at);
  } else {
    s = first = slot;
    rows = 1;
  }
  if (first + rows <= row0 || first >= row1) return;
  int lo, hi, lo1, hi1, s1;
  const int pos = row_position(b, c, first + rows - 1, s1), pos0 = row_position(b, c, first, s1);
  if (pos < 0) return;
  page_range(a, pos, page_log, lo1, hi);
  page_range(a, pos0 < 0 ? 0 : pos0, page_log, lo, hi1);
  const int p0 = lo / 16 * 16 + chunk * kScorePages + 16 * wave;
  if (lo / 16 * 16 + chunk * kScorePages > hi) return;

  // the columns' queries as bytes: lane (column n, quarter) holds dimensions 64 v + 16 quarter ..
  const int row = first + n / a.g;
  const bool live = n / a.g < rows && a.g <= kScoreCols;
  const int32_t* pages = b.page_table + (size_t)s * b.max_pages;
  const int tiles = (a.g + kScoreCols - 1) / kScoreCols;        // of heads, where they pass the columns
  for (int ht = 0; ht < tiles; ++ht) {
    const int h = a.g > kScoreCols ? kScoreCols * ht + n : n % a.g;
    const bool mine = a.g > kScoreCols ? h < a.g : live;
    const uint16_t* qr = q.p + (size_t)(mine ? (a.g > kScoreCols ? first : row) : first) * q.stride +
                         (size_t)(hk * a.g + (mine ? h : 0)) * D + 16 * quarter;
    float x[NV][16], most = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(qr + 64 * v + 8 * w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float f = half_of(r[e / 2], e & 1);
          if (a.negative) f = -f;
          f = fabsf(f) < -kNegInf ? f : 0.0f;
          x[v][8 * w + e] = f;
          most = fmaxf(most, fabsf(f));
        }
      }
    most = halves_max(rows_max(most));
    const float sq = most * k127th, by = sq > 0.0f ? sq : 1.0f;
    i32x4 neg[NV], plus[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t lo4 = 0, hi4 = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float f = rintf(x[v][4 * w + e] / by);
          f = f > 127.0f ? 127.0f : f < -127.0f ? -127.0f : f;
          const int i = (int)f;
          lo4 |= (uint32_t)((i < 0 ? i : 0) & 0xff) << (8 * e);
          hi4 |= (uint32_t)((i > 0 ? i : 0) & 0xff) << (8 * e);
        }
        neg[v][w] = (int)lo4;
        plus[v][w] = (int)hi4;
      }
    for (int p = p0; p <= hi && p < p0 + kScorePages; p += kScoreThreads / 64 * 16) {
      const int mine_p = min(p + n, b.max_pages - 1);
      const size_t at = ((size_t)kv_page(c, pages[mine_p]) * c.Hkv + hk) * 2 * D + 16 * quarter;
      i32x4 sum = {0, 0, 0, 0};
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const i32x4 bl = *reinterpret_cast<const i32x4*>(sm.bounds + at + 64 * v);
        const i32x4 bh = *reinterpret_cast<const i32x4*>(sm.bounds + at + D + 64 * v);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bl, neg[v], sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bh, plus[v], sum, 0, 0, 0);
      }
      // lane (column n, quarter): pages p + 4 quarter + r
      asm volatile("" ::: "memory");             // the wave's own places: LDS is in order
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int pr = min(p + 4 * quarter + r, b.max_pages - 1);
        const float ps = sm.scale[(size_t)kv_page(c, pages[pr]) * c.Hkv + hk];
        s_part[wave][4 * quarter + r][n] = mine ? (float)sum[r] * (sq * ps) : kNegInf;
      }
      asm volatile("" ::: "memory");
      const int page = p + n;
      for (int i = quarter; i < rows; i += 4) {
        const int cols = min(a.g, kScoreCols);
        float m = s_part[wave][n][i * cols];
        for (int j = 1; j < cols; ++j) m = fmaxf(m, s_part[wave][n][i * cols + j]);
        const int t = first + i;
        if (page <= hi && t >= row0 && t < row1) {
          float* out = scores + ((size_t)(t - row0) * c.Hkv + hk) * b.max_pages + page;
          if (ht > 0) m = fmaxf(m, *out);
          *out = m;
        }
      }
      asm volatile("" ::: "memory");
    }
  }
}

// --------------------------------------------------------------- selection --
constexpr int kSelThreads = 256;
constexpr int kSelCached = 8192;         // scores that fit LDS

// A float's bits, ordered as unsigned numbers (zeros of both signs alike; NaN last).
__device__ __forceinline__ uint32_t score_key(float f) {
  if (!(f == f)) return 0u;
  const uint32_t u = __float_as_uint(f == 0.0f ? 0.0f : f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Threads before this one whose flag is set, and all of them; tmp: one place a wave.
__device__ __forceinline__ int flags_before(bool flag, int* tmp, int& all) {
  const uint64_t set = __ballot(flag);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();                               // the last call's places have been read
  if (lane == 0) tmp[wave] = __popcll(set);
  __syncthreads();
  int before = __popcll(set & ((1ull << lane) - 1)), sum = 0;
#pragma unroll
  for (int w = 0; w < kSelThreads / 64; ++w) {
    if (w < wave) before += tmp[w];
    sum += tmp[w];
  }
  all = sum;
  return before;
}

__global__ void __launch_bounds__(kSelThreads)
    page_select_kernel(BatchArgs b, KvArgs c, SelectArgs a, int row0, const float* __restrict__ scores) {
  __shared__ uint32_t s_key[kSelCached];
  __shared__ int s_hist[256], s_tmp[kSelThreads / 64], s_found[2];
  const int t = row0 + blockIdx.x / c.Hkv, hk = blockIdx.x % c.Hkv, page_log = c.lb + 4;
  if (b.q_start && (t < b.q_start[0] || t >= b.q_start[b.S])) return;       // padding
  int s;
  const int pos = row_position(b, c, t, s);
  int32_t* out = a.sel + ((size_t)t * c.Hkv + hk) * a.n_sel;
  int lo = 0, hi = -1;
  if (pos >= 0) page_range(a, pos, page_log, lo, hi);
  const int pages = hi - lo + 1, count = min(pages, a.n_sel);
  if (threadIdx.x == 0) a.count[(size_t)t * c.Hkv + hk] = count;
  if (pages <= a.n_sel) {
    for (int i = threadIdx.x; i < a.n_sel; i += kSelThreads) out[i] = i < pages ? lo + i : -1;
    return;
  }
  const float* row = scores + ((size_t)(t - row0) * c.Hkv + hk) * b.max_pages + lo;
  auto key_of = [&](int i) {                     // pages that are always taken come first
    const int p = lo + i;
    return p < a.first || p > hi - a.last ? 0xffffffffu : score_key(row[i]);
  };
  const bool cached = pages <= kSelCached;
  if (cached)
    for (int i = threadIdx.x; i < pages; i += kSelThreads) s_key[i] = key_of(i);
  auto key = [&](int i) { return cached ? s_key[i] : key_of(i); };
  // the n_sel-th largest key, a byte at a time; `left`: how many of its equals are taken
  uint32_t prefix = 0;
  int left = a.n_sel;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    s_hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < pages; i += kSelThreads) {
      const uint32_t k = key(i);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (threadIdx.x < 64) {
      // lane l: digits 255 - 4 l downwards; the first whose running count reaches `left`
      const int l = threadIdx.x;
      int h[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = s_hist[255 - 4 * l - i];
        sum += h[i];
      }
      int before = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(before, d);
        if (l >= d) before += y;
      }
      before -= sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < left && before + h[i] >= left) {
          s_found[0] = 255 - 4 * l - i;
          s_found[1] = left - before;
        }
        before += h[i];
      }
    }
    __syncthreads();
    prefix = prefix << 8 | (uint32_t)s_found[0];
    left = s_found[1];
  }
  int done = 0, equal = 0;
  for (int i0 = 0; i0 < pages; i0 += kSelThreads) {
    const int i = i0 + threadIdx.x;
    const uint32_t k = i < pages ? key(i) : 0u;
    int all_eq, all;
    const bool eq = i < pages && k == prefix;
    const int rank = equal + flags_before(eq, s_tmp, all_eq);
    const bool take = i < pages && (k > prefix || (eq && rank < left));
    const int at = done + flags_before(take, s_tmp, all);
    if (take && at < a.n_sel) out[at] = lo + i;
    equal += all_eq;
    done += all;
  }
}

static int score_slots(const BatchArgs& b, int g) {
  const int R = score_rows(g);
  return b.q_start ? (b.T + R - 1) / R + b.S - 1 : b.S;
}

// Rows whose scores are held at once: 256 MB of them.
static size_t select_rows(int rows, int Hkv, int max_pages) {
  const size_t most = ((size_t)256 << 20) / ((size_t)Hkv * max_pages * sizeof(float));
  return most < 1 ? 1 : most < (size_t)rows ? most : (size_t)rows;
}

size_t attn_select_bytes(int rows, int Hkv, int max_pages) {
  return select_rows(rows, Hkv, max_pages) * Hkv * max_pages * sizeof(float);
}

long long select_workgroups(const BatchArgs& b, const KvArgs& c, int g) {
  return (long long)score_slots(b, g) * c.Hkv * ((b.max_pages + kScorePages - 1) / kScorePages + 1);
}

hipError_t launch_attn_select(RowsIn q, int D, const BatchArgs& b, const KvArgs& c, const SummaryArgs& sm,
                              const SelectArgs& a, void* ws, hipStream_t stream) {
  const int rows = b.q_start ? b.T : b.S, each = (int)select_rows(rows, c.Hkv, b.max_pages);
  // (the first chunk begins at a multiple of 16 pages, below the first page of the row)
  const int chunks = (b.max_pages + kScorePages - 1) / kScorePages + 1;
  float* scores = static_cast<float*>(ws);
  hipError_t err = hipSuccess;
  for (int row0 = 0; row0 < rows && err == hipSuccess; row0 += each) {
    const int row1 = row0 + each < rows ? row0 + each : rows;
    const dim3 grid((unsigned)((size_t)score_slots(b, a.g) * c.Hkv * chunks));
    timing_begin(stream, kSiteAttnSelect);
    if (D == 64)
      hipLaunchKernelGGL(page_score_kernel<64>, grid, dim3(kScoreThreads), 0, stream, q, b, c, sm, a, row0, row1,
                         chunks, scores);
    else
      hipLaunchKernelGGL(page_score_kernel<128>, grid, dim3(kScoreThreads), 0, stream, q, b, c, sm, a, row0, row1,
                         chunks, scores);
    hipLaunchKernelGGL(page_select_kernel, dim3((unsigned)((size_t)(row1 - row0) * c.Hkv)), dim3(kSelThreads), 0,
                       stream, b, c, a, row0, scores);
    timing_end(stream, kSiteAttnSelect);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace mc
