// attn_select.hip -- bounds on the keys of a page, and the pages that each query attends to.
//
//   bounds of a page and key-value head:  s = max |k| / 127 (times the fp32 number nearest to 1/127),
//   hi = ceil(max_t k / s),  lo = floor(min_t k / s)
//   score of a page for a row:  max over the group's heads of (sq s) sum_i (q8_i > 0 ? q8_i hi_i : q8_i lo_i)
// with q8 = rint(q / sq), sq = max |q| / 127.  It bounds the products of the page's finite keys with the rounded
// query from above, up to 2^-22 of sum |q_i| max |k|: s is rounded, and where 127 s lies below max |k| the quotient's
// ceiling, 128, is cut to 127.  All sums are of whole numbers below 2^24 and so exact in any order; what is
// rounded is one product, the same in any implementation, and so is the selection.
//
// kv_summary_kernel: one workgroup a touched page and head.  page_score_kernel: the products of 16
// pages with 16 (row, head) columns are 2 D / 64 matrix instructions on bytes; negative parts of the
// query go with lo, positive ones with hi.  page_select_kernel: one workgroup a row and head finds the
// n-th largest score digit by digit and lists what is above it, and of its equals the first.
//
// Bounds are 2 D + 4 bytes a page and head (pages of 64 bf16 tokens: 1/126 of their keys and values), read
// in pieces of 2 D bytes wherever the pages lie.  16 rows of some 1180 pages, 8 heads: scores 18 us (39 MB at
// the least, 47 measured), selection 8.4, bounds of the last pages 5.8; one row of 521: 5.3, 5.9 and 4.9, each a chain
// of memory latencies.  (Both in one launch of 1024 threads, the scores in LDS: 35 us for 25, and 21 for 13.)
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
constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
constexpr int kScoreCols = 16;           // (row, head) columns of a product

// Rows of a workgroup: those whose heads fill the columns.
__host__ __device__ static inline int score_rows(int g) { return g >= kScoreCols ? 1 : kScoreCols / g; }

// Pages [lo, hi] that a row at position pos may take.
__device__ __forceinline__ void page_range(const SelectArgs& a, int pos, int page_log, int& lo, int& hi) {
  hi = pos >> page_log;
  lo = a.window > 0 && pos >= a.window ? (pos - a.window + 1) >> page_log : 0;
}

// The position of row t of sequence s, whose rows end before `end` (-1: a row that sees nothing).
__device__ __forceinline__ int row_position(const BatchArgs& b, const KvArgs& c, int s, long long end, int t) {
  const int len = kv_length(c, b, s);
  const long long pos = (long long)b.kv_len[s] - (end - t);
  return pos < 0 || len == 0 ? -1 : pos < len ? (int)pos : len - 1;
}

// rint(x / by), r being some 1 / by: from the product, unless that is so near to a half that the
// quotient might lie on the other side of it.
__device__ __forceinline__ float rint_quotient(float x, float by, float r) {
  const float y = x * r;
  float n = rintf(y);
  if (__any(!(fabsf(y - n) <= 0.4999f))) n = rintf(x / by);     // (and where the product is no number)
  return n;
}

// Workspace: scores [row - row0][Hkv][pages], pages the row length of the tables.  A workgroup takes 64 pages
// of a head, 16 a wave.  (256, four tiles a wave at once: one row of 521 pages 3 us more, 16 rows of some 1180
// pages 1 us less of 79, 228 rows of some 200 1 us more.)
template <int D>
__global__ void __launch_bounds__(kScoreThreads)
    page_score_kernel(RowsIn q, BatchArgs b, KvArgs c, SummaryArgs sm, SelectArgs a, int row0, int row1, int chunks,
                      float* __restrict__ scores) {
  constexpr int NV = D / 64, kPages = 64, kQ = D + 16;       // (a row of queries, off the banks of the last)
  __shared__ float s_part[kScoreWaves][16][kScoreCols + 1];
  __shared__ float s_most[kScoreWaves][kScoreCols], s_sq[kScoreCols];
  __shared__ __attribute__((aligned(16))) int8_t s_q[2][kScoreCols][kQ];
  const int lane = threadIdx.x & 63, wave = wave_id(), n = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int chunk = id % chunks;
  id /= chunks;
  const int hk = id % c.Hkv, slot = id / c.Hkv, R = score_rows(a.g), page_log = c.lb + 4;
  // rows first, ..., first + rows - 1, of one sequence
  int s, first, rows;
  long long end;
  if (b.q_start) {
    s = find_sequence(b.q_start, b.S, slot, R, 1, 1);
    end = b.q_start[s + 1];
    int start, count;
    sequence_rows(b, s, start, count);
    const long long at = ((long long)slot - ((long long)b.q_start[s] / R + s)) * R;
    if (at < 0 || at >= count) return;
    first = start + (int)at;
    rows = min(R, count - (int)at);
  } else {
    s = first = slot;
    end = first + 1;
    rows = 1;
  }
  if (first + rows <= row0 || first >= row1) return;
  int lo, hi, lo1, hi1;
  const int pos = row_position(b, c, s, end, first + rows - 1), pos0 = row_position(b, c, s, end, first);
  if (pos < 0) return;
  page_range(a, pos, page_log, lo1, hi);
  page_range(a, pos0 < 0 ? 0 : pos0, page_log, lo, hi1);
  const int p0 = lo / 16 * 16 + chunk * kPages + 16 * wave;       // the wave's: p0 .. p0 + 15
  if (lo / 16 * 16 + chunk * kPages > hi) return;

  // A head tile's queries: thread (wave, column n, quarter) takes dimensions 32 wave + 8 quarter ..
  const int tiles = (a.g + kScoreCols - 1) / kScoreCols;        // of heads, where they pass the columns
  const int cols = min(a.g, kScoreCols);
  const int d0 = 32 * wave + 8 * quarter;
  auto load_q = [&](int ht, bool& mine) {
    const int r = n / cols, h = a.g > kScoreCols ? kScoreCols * ht + n : n % cols;
    mine = r < rows && h < a.g && d0 < D;
    const uint16_t* qr = q.p + (size_t)(first + (mine ? r : 0)) * q.stride + (size_t)(hk * a.g + (mine ? h : 0)) * D;
    return *reinterpret_cast<const u32x4*>(qr + (mine ? d0 : 0));
  };
  bool mine;
  u32x4 u = load_q(0, mine);

  // the bounds of the wave's pages: lane (page n, quarter) holds dimensions 64 v + 16 quarter ..
  const int32_t* pages = b.page_table + (size_t)s * b.max_pages;
  const size_t at = (size_t)kv_page(c, pages[min(p0 + n, hi)]) * c.Hkv + hk;
  const int8_t* from = sm.bounds + at * 2 * D + 16 * quarter;
  i32x4 bl[NV], bh[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    bl[v] = *reinterpret_cast<const i32x4*>(from + 64 * v);
    bh[v] = *reinterpret_cast<const i32x4*>(from + D + 64 * v);
  }
  const float ps = sm.scale[at];

  // The columns' queries as bytes, by way of LDS (each wave for itself: four times the instructions, which a
  // workgroup runs once and waits for), while the bounds are on their way: the barriers do not wait for them
  for (int ht = 0; ht < tiles; ++ht) {
    if (ht > 0) u = load_q(ht, mine);
    float x[8], most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f = half_of(u[e / 2], e & 1);
      f = mine && fabsf(f) < -kNegInf ? f : 0.0f;
      x[e] = a.negative ? -f : f;
      most = fmaxf(most, fabsf(f));
    }
    most = halves_max(rows_max(most));
    if (ht > 0) lds_barrier();                     // the last tile's have been read
    if (quarter == 0) s_most[wave][n] = most;
    lds_barrier();
    most = fmaxf(fmaxf(s_most[0][n], s_most[1][n]), fmaxf(s_most[2][n], s_most[3][n]));
    const float sq = most * k127th, by = sq > 0.0f ? sq : 1.0f, rby = 1.0f / by;
    if (threadIdx.x < kScoreCols) s_sq[n] = sq;
    if (d0 < D) {
      u32x2 lo8 = {0u, 0u}, hi8 = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f = rint_quotient(x[e], by, rby);
        f = f > 127.0f ? 127.0f : f < -127.0f ? -127.0f : f;
        const int i = (int)f;
        lo8[e / 4] |= (uint32_t)((i < 0 ? i : 0) & 0xff) << (8 * (e & 3));
        hi8[e / 4] |= (uint32_t)((i > 0 ? i : 0) & 0xff) << (8 * (e & 3));
      }
      *reinterpret_cast<u32x2*>(&s_q[0][n][d0]) = lo8;
      *reinterpret_cast<u32x2*>(&s_q[1][n][d0]) = hi8;
    }
    lds_barrier();
    i32x4 neg[NV], plus[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      neg[v] = *reinterpret_cast<const i32x4*>(&s_q[0][n][64 * v + 16 * quarter]);
      plus[v] = *reinterpret_cast<const i32x4*>(&s_q[1][n][64 * v + 16 * quarter]);
    }
    if (p0 > hi) continue;                           // the same for the whole wave
    i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bl[v], neg[v], sum, 0, 0, 0);
      sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bh[v], plus[v], sum, 0, 0, 0);
    }
    // lane (column n, quarter): pages 4 quarter + r of the tile.  Heads are joined by way of LDS, whose
    // accesses are in order (the places are the wave's own); there lane (n, quarter) has page n
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < 4; ++r) s_part[wave][4 * quarter + r][n] = (float)sum[r];
    asm volatile("" ::: "memory");
    const int page = p0 + n;
    for (int k = quarter; k < rows; k += 4) {
      float m = kNegInf;
      for (int j = 0; j < cols && cols * ht + j < a.g; ++j)
        m = fmaxf(m, s_part[wave][n][k * cols + j] * (s_sq[k * cols + j] * ps));
      const int t = first + k;
      if (page <= hi && t >= row0 && t < row1) {
        float* out = scores + ((size_t)(t - row0) * c.Hkv + hk) * b.max_pages + page;
        if (ht > 0) m = fmaxf(m, *out);
        *out = m;
      }
    }
    asm volatile("" ::: "memory");
  }
}

// --------------------------------------------------------------- selection --
constexpr int kSelThreads = 256;

// A float's bits, ordered as unsigned numbers (zeros of both signs alike; NaN last).
__device__ __forceinline__ uint32_t score_key(float f) {
  if (!(f == f)) return 0u;
  const uint32_t u = __float_as_uint(f == 0.0f ? 0.0f : f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sum over the threads before this one, and over all; tmp: one place a wave.
__device__ __forceinline__ int counts_before(int x, int* tmp, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int y = wave_scan(x);
  lds_barrier();                                 // the last call's places have been read
  if (lane == 63) tmp[wave] = y;
  lds_barrier();
  int before = y - x, sum = 0;
#pragma unroll
  for (int w = 0; w < kSelThreads / 64; ++w) {
    if (w < wave) before += tmp[w];
    sum += tmp[w];
  }
  all = sum;
  return before;
}

// A thread takes K neighbouring pages a round, in registers; more than one round of them (HELD
// false) are read again in each pass.
template <int K, bool HELD>
__device__ void select_pages(const SelectArgs& a, const float* __restrict__ row, int lo, int hi,
                             int32_t* __restrict__ out, int (*s_hist)[256], int* s_tmp, int* s_found) {
  const int pages = hi - lo + 1, rounds = HELD ? 1 : (pages + K * kSelThreads - 1) / (K * kSelThreads);
  uint32_t key[K];
  auto load = [&](int round) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = (round * kSelThreads + (int)threadIdx.x) * K + k, p = lo + i;
      key[k] = i >= pages ? 0u : p < a.first || p > hi - a.last ? 0xffffffffu : score_key(row[i]);
    }
  };
  // the n_sel-th largest key, a byte at a time; `left`: how many of those at the prefix are taken.  (Places
  // behind the last page hold 0 and lose to every page.)
  uint32_t prefix = 0;
  int left = a.n_sel, shift = 24;
  for (int i = threadIdx.x; i < 512; i += kSelThreads) s_hist[i >> 8][i & 255] = 0;
  if (HELD) load(0);
  for (;; shift -= 8) {
    int* hist = s_hist[(shift >> 3) & 1];
    lds_barrier();
    for (int r = 0; r < rounds; ++r) {
      if (!HELD) load(r);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const bool in = shift == 24 || (key[k] >> (shift + 8)) == prefix;
        const uint32_t digit = (key[k] >> shift) & 255u;
        // most scores share their first digits: those of the first lane's are counted at once
        const uint32_t lead = __builtin_amdgcn_readfirstlane(digit);
        const uint64_t same = __ballot(in && digit == lead);
        if (in && digit != lead)
          atomicAdd(&hist[digit], 1);
        else if ((threadIdx.x & 63) == 0 && same)
          atomicAdd(&hist[lead], __popcll(same));
      }
    }
    lds_barrier();
    if (threadIdx.x < 64) {
      // lane l: digits 255 - 4 l downwards; the first whose running count reaches `left`
      const int l = threadIdx.x;
      int h[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = hist[255 - 4 * l - i];
        sum += h[i];
      }
      int before = wave_scan(sum) - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < left && before + h[i] >= left) {
          s_found[0] = 255 - 4 * l - i;
          s_found[1] = left - before;
          s_found[2] = h[i];
        }
        before += h[i];
      }
    } else {
      int* next = s_hist[((shift >> 3) & 1) ^ 1];
      for (int i = threadIdx.x - 64; i < 256; i += kSelThreads - 64) next[i] = 0;
    }
    lds_barrier();
    prefix = prefix << 8 | (uint32_t)s_found[0];
    left = s_found[1];
    if (shift == 0 || left == s_found[2]) break;           // all at the prefix are taken
  }
  // those above the prefix and the first `left` at it, in order
  int done = 0, equal = 0;
  for (int r = 0; r < rounds; ++r) {
    if (!HELD) load(r);
    int above = 0, at = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t top = key[k] >> shift;
      above += top > prefix;
      at += top == prefix;
    }
    // (both sums in one: up to 2^14 a round)
    int all;
    const int before = counts_before(above << 16 | at, s_tmp, all);
    int rank = equal + (before & 0xffff);                  // of the first at the prefix
    int place = done + (before >> 16) + min(rank, left);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t top = key[k] >> shift;
      const bool take = top > prefix || (top == prefix && rank < left);
      rank += top == prefix;
      if (take && place < a.n_sel) out[place] = lo + (r * kSelThreads + (int)threadIdx.x) * K + k;
      place += take;
    }
    done += all >> 16;
    equal += all & 0xffff;
  }
}

__global__ void __launch_bounds__(kSelThreads)
    page_select_kernel(BatchArgs b, KvArgs c, SelectArgs a, int row0, const float* __restrict__ scores) {
  __shared__ int s_hist[2][256], s_tmp[kSelThreads / 64], s_found[3];
  const int t = row0 + blockIdx.x / c.Hkv, hk = blockIdx.x % c.Hkv, page_log = c.lb + 4;
  int s = t;
  long long end = t + 1;
  if (b.q_start) {
    s = find_sequence(b.q_start, b.S, t, 1, 0, 1);
    end = b.q_start[s + 1];
    if (t < b.q_start[s] || t >= end) return;      // padding
  }
  const int pos = row_position(b, c, s, end, t);
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
  if (pages <= 2 * kSelThreads)
    select_pages<2, true>(a, row, lo, hi, out, s_hist, s_tmp, s_found);      // (200 pages: 8 keys a thread 3 us more)
  else if (pages <= 4 * kSelThreads)
    select_pages<4, true>(a, row, lo, hi, out, s_hist, s_tmp, s_found);
  else if (pages <= 8 * kSelThreads)
    select_pages<8, true>(a, row, lo, hi, out, s_hist, s_tmp, s_found);
  else
    select_pages<8, false>(a, row, lo, hi, out, s_hist, s_tmp, s_found);
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

// Chunks of 64 pages that cover any row's (the first begins at a multiple of 16 pages, below the first page of
// the row).
static int score_chunks(int max_pages) { return (max_pages + 63) / 64 + 1; }

long long select_workgroups(const BatchArgs& b, const KvArgs& c, int g) {
  return (long long)score_slots(b, g) * c.Hkv * score_chunks(b.max_pages);
}

hipError_t launch_attn_select(RowsIn q, int D, const BatchArgs& b, const KvArgs& c, const SummaryArgs& sm,
                              const SelectArgs& a, void* ws, hipStream_t stream) {
  const int rows = b.q_start ? b.T : b.S, each = (int)select_rows(rows, c.Hkv, b.max_pages);
  const int chunks = score_chunks(b.max_pages);
  const dim3 grid((unsigned)((size_t)score_slots(b, a.g) * c.Hkv * chunks));
  float* scores = static_cast<float*>(ws);
  hipError_t err = hipSuccess;
  for (int row0 = 0; row0 < rows && err == hipSuccess; row0 += each) {
    const int row1 = row0 + each < rows ? row0 + each : rows;
    timing_begin(stream, kSiteAttnSelect);
    if (D == 64)
      hipLaunchKernelGGL(page_score_kernel<64>, grid, dim3(kScoreThreads), 0, stream, q, b, c, sm, a, row0, row1, chunks,
                         scores);
    else
      hipLaunchKernelGGL(page_score_kernel<128>, grid, dim3(kScoreThreads), 0, stream, q, b, c, sm, a, row0, row1, chunks,
                         scores);
    hipLaunchKernelGGL(page_select_kernel, dim3((unsigned)((size_t)(row1 - row0) * c.Hkv)), dim3(kSelThreads), 0,
                       stream, b, c, a, row0, scores);
    timing_end(stream, kSiteAttnSelect);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace mc
