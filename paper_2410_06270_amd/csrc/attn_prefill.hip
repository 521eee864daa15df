// attn_prefill.hip -- causal attention of prompts and prompt chunks over the
// paged cache.
//
//   o_i = sum_j p_ij v_j / l_i,  p_ij = exp2(s_ij - m_i),  l_i = sum_j p_ij
// in one pass over the keys with a running maximum m_i for each row.
//
// Bound by the matrix units and the exponentials together: a 32 x 32 tile of
// scores costs 16 matrix instructions of 32x32x16 for D = 128 (512 cycles of a
// SIMD) and 16 exponentials a lane (256) beside some 12 plain instructions a score.
//
// A workgroup of four waves takes 128 rows of one sequence and key-value head;
// the g query heads that share it are packed into the rows (row = token * g +
// head), so a short chunk fills a tile with heads and a tile's rows span few
// positions.  Keys and values come through LDS in tiles of 64, two buffers;
// the cache's 16-byte units are already the order in which the matrix
// instructions read them, so a bf16 tile is copied straight to LDS by direct
// loads and read without bank conflicts; e4m3 is widened on the way (exactly).
// Scores are keys x rows (S^T = K Q^T): a lane holds 16 keys of ONE row, so the
// row's maximum and sum are in-lane but for one exchange between the half waves,
// and the score rows are dealt so that the lane's keys are the ones that it
// supplies to O^T = V^T P^T: the weights never leave their registers.
#include <type_traits>

#include "attn.hpp"

namespace mc {

constexpr int kPreWaves = 4;
constexpr int kPreThreads = 64 * kPreWaves;
constexpr int kPreRows = 32 * kPreWaves;      // rows of a workgroup
constexpr int kPreKeys = 64;                  // keys of a tile

// Row tiles: sequence s owns slots floor(q_start[s] g / 128) + s and on, at
// least ceil(rows / 128) of them.
static int prefill_slots(int T, int S, int g) { return (int)((long long)T * g / kPreRows) + S; }

// Few row tiles are split over the keys, up to kPreTarget workgroups (two a
// CU), each with 512 keys at least.
constexpr int kPreTarget = 512, kPreMaxSplit = 32;

static int prefill_splits(int slots, int Hkv, int max_len) {
  long long n = kPreTarget / ((long long)slots * Hkv);
  const int most = (max_len + 511) / 512;
  n = n > most ? most : n;
  return (int)(n < 1 ? 1 : n > kPreMaxSplit ? kPreMaxSplit : n);
}

// T g / 128 <= slots and nsplit slots Hkv <= kPreTarget, so a split call has at
// most 128 kPreTarget partial rows.
size_t attn_prefill_split_rows(int T, int Hq) {
  const size_t all = (size_t)T * Hq * kPreMaxSplit, most = (size_t)kPreRows * kPreTarget;
  return all < most ? all : most;
}

// The larger of x in lanes l and l ^ 32, and the sum of both.
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The running maximum follows a larger score only when it is left behind by more
// than this (log2): weights up to 2^8 lose nothing in fp32 sums or in bf16, and most
// tiles need no scaling and no exchange between the half waves.
constexpr float kMaxSlack = 8.0f;

// Largest magnitude bits of the eight bf16 of w, by pairs (for the search for
// infinities and NaN: those have all exponent bits set).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 magnitude_max(u16x2 acc, const u32x4& w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = w[i] & 0x7fff7fffu;
    u16x2 h;
    __builtin_memcpy(&h, &t, 4);
    acc = __builtin_elementwise_max(acc, h);
  }
  return acc;
}

template <int D, bool E4, bool EXTRA>
__global__ void __launch_bounds__(kPreThreads, 2)
    attn_prefill_kernel(RowsIn q, BatchArgs b, KvArgs c, ScoreArgs a, RowsOut o, float* __restrict__ lse, SplitArgs sp,
                        int slots) {
  constexpr int DT = D / 32, DK = D / 16;      // value tiles; score steps
  constexpr int kTileBytes = kPreKeys * D * 2, kBlk = kKvBlock * D * 2;      // in LDS: bf16
  constexpr int kBlockBytes = kKvBlock * D * (E4 ? 1 : 2);                   // in the cache
  __shared__ __attribute__((aligned(16))) char s_kv[2][2 * kTileBytes];      // [buffer], keys then values
  const int lane = threadIdx.x & 63, wave = wave_id(), n = lane & 31, half = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % c.Hkv;
  id /= c.Hkv;
  const int split = id % sp.nsplit;
  const int slot = slots - 1 - id / sp.nsplit;       // later rows see more keys: they go first
  const int s = find_sequence(b.q_start, b.S, slot, kPreRows, 1, a.g);
  int first, count;
  sequence_rows(b, s, first, count);
  const long long base64 = (long long)b.q_start[s] * a.g / kPreRows + s;
  const long long row0l = (slot - base64) * kPreRows;
  if (row0l < 0 || row0l >= (long long)count * a.g) return;
  const int row0 = (int)row0l;

  const int len = kv_length(c, b, s);
  const int pos0 = len - count;
  const int pre = kv_prefix(a, s, len);
  const int rows_in = min(kPreRows, count * a.g - row0);
  const int pos_first = pos0 + row0 / a.g, pos_last = pos0 + (row0 + rows_in - 1) / a.g;

  // this lane's row
  const int row = row0 + 32 * wave + n;
  const bool live = row < count * a.g;
  const int tok = live ? row / a.g : 0, head = hk * a.g + (live ? row - tok * a.g : 0);
  const int pos = live ? pos0 + tok : -1;            // a negative position sees nothing
  // of the wave's live rows
  const int wrow = row0 + 32 * wave;
  const bool wave_live = wrow < count * a.g;
  const int wpos_first = pos0 + wrow / a.g, wpos_last = pos0 + min(wrow + 31, count * a.g - 1) / a.g;

  // queries: lane (row n, half) holds units half, half + 2, ... of its row (a row
  // that is not live takes another's).  A negative scale turns their signs, so that
  // the largest product is the largest score.
  bf16x8 qf[DK];
  {
    const uint16_t* qr = q.p + (size_t)(first + tok) * q.stride + (size_t)head * D + 8 * half;
    const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int i = 0; i < DK; ++i) {
      u32x4 r = *reinterpret_cast<const u32x4*>(qr + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] ^= sign;
      qf[i] = as_bf16x8(r);
    }
  }

  // key tiles that some row sees: [0, ia) and [ib, end)
  int hi = pos_last + 1 > pre ? pos_last + 1 : pre;
  if (hi > len) hi = len;
  const int end = hi > 0 ? (hi + kPreKeys - 1) / kPreKeys : 0;
  const int wstart = a.window > 0 && pos_first >= a.window ? pos_first - a.window + 1 : 0;
  int ia = (pre + kPreKeys - 1) / kPreKeys, ib = wstart / kPreKeys;
  if (ib <= ia) ia = ib = 0;
  const int tiles = max(0, ia + end - ib), per = (tiles + sp.nsplit - 1) / sp.nsplit;
  const int t_end = min(tiles, (split + 1) * per), t_begin = min(split * per, t_end);
  const int32_t* pages = b.page_table + (size_t)s * b.max_pages;
  const int last_blk = len > 0 ? (len - 1) >> 4 : 0;
  auto tile_key = [&](int t) { return (t < ia ? t : t - ia + ib) * kPreKeys; };

  // A tile's 4 blocks of keys and 4 of values: wave w takes block w of each.
  constexpr int kPieces = kBlockBytes / 1024;
  u32x4 stage[E4 ? 2 * kPieces : 1];
  // The page number comes a tile earlier: its load would otherwise hold up the
  // tile's own.
  auto tile_blk = [&](int t) { return min((tile_key(t) >> 4) + wave, last_blk); };
  auto page_of = [&](int t) { return uniform_entry(pages, tile_blk(min(t, t_end - 1)) >> c.lb); };
  auto fetch = [&](int t, char* to, int page) {
    const size_t off = kv_block_offset<kBlockBytes>(c, kv_page(c, page), hk,
                                                    tile_blk(t)) + 16 * lane;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if constexpr (E4) {
        stage[i] = *reinterpret_cast<const u32x4*>(c.k + off + 1024 * i);
        stage[kPieces + i] = *reinterpret_cast<const u32x4*>(c.v + off + 1024 * i);
      } else {
        lds_dma16(c.k + off + 1024 * i, to + wave * kBlk + 1024 * i);
        lds_dma16(c.v + off + 1024 * i, to + kTileBytes + wave * kBlk + 1024 * i);
      }
    }
  };
  // e4m3: the fetched units, widened to the bf16 units of the block.  Unit x of the
  // keys is (16 dimensions, token): two bf16 units, 256 bytes apart; of the values
  // (dimension, 16 tokens): D * 16 apart.
  auto put = [&](char* to) {
    if constexpr (E4) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int x = 64 * i + lane;
        char* kd = to + wave * kBlk + (x >> 4) * 512 + (x & 15) * 16;
        *reinterpret_cast<u32x4*>(kd) = e4m3_to_bf16(stage[i][0], stage[i][1]);
        *reinterpret_cast<u32x4*>(kd + 256) = e4m3_to_bf16(stage[i][2], stage[i][3]);
        char* vd = to + kTileBytes + wave * kBlk + x * 16;
        *reinterpret_cast<u32x4*>(vd) = e4m3_to_bf16(stage[kPieces + i][0], stage[kPieces + i][1]);
        *reinterpret_cast<u32x4*>(vd + D * 16) = e4m3_to_bf16(stage[kPieces + i][2], stage[kPieces + i][3]);
      }
    }
  };

  f32x16 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
  float m = kNegInf, l = 0.0f;       // l: of the lane's own keys
  const float kscale = E4 ? c.k_scale[hk] : 1.0f;
  const ScoreConsts sc = {fabsf(a.scale) * kscale, fabsf(a.scale) * kscale * kLog2e, a.softcap,
                          a.softcap > 0.0f ? 1.0f / a.softcap : 0.0f};
  const float slope2 = EXTRA && a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  // keys of a score tile: row m of the tile is key (m with bits 2 and 3 swapped)
  const int krow = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);
  const int koff = (krow >> 4) * kBlk + (krow & 15) * 16 + half * 256;
  const int voff = half * D * 16 + n * 16;

  // the row sees the keys below rpre and in (rlow, pos]
  const int rlow = a.window > 0 && pos >= a.window ? pos - a.window : -1, rpre = pos >= 0 ? pre : 0;
  // (j counted from the first of the tile's keys that the half wave takes)
  struct Mask {
    int pos, low, pre;
  };
  auto visible = [&](const Mask& k, int j) { return ((j <= k.pos) & (j > k.low)) | (j < k.pre); };
  // The product with a tile of values some of which are not finite: those are left
  // out of it and added, key by key, to the rows that see them (a weight is
  // positive, so it changes neither an infinity nor a NaN).
  auto add_odd = [&](const char* vs, const u32x4 (&p)[4], int key0) {
    int h = half, vo = voff;
    asm volatile("" : "+v"(h), "+v"(vo));              // nothing of this is computed ahead of the loop
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        u32x4 v = *reinterpret_cast<const u32x4*>(vs + vo + i * kBlk + 512 * d);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = (v[e] & 0x7f80u) == 0x7f80u ? v[e] & 0xffff0000u : v[e];
          v[e] = (v[e] & 0x7f800000u) == 0x7f800000u ? v[e] & 0xffffu : v[e];
        }
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(p[i]), acc[d], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll 1
    for (int e = 0; e < kPreKeys; ++e) {
      const bool in = visible(Mask{pos - key0, rlow - key0, rpre - key0}, e);
      // dimension 32 d + 8 (r / 4) + 4 half + r % 4 of key e
      const char* vk = vs + (e >> 4) * kBlk + ((e >> 3) & 1) * D * 16 + 64 * h + 2 * (e & 7);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t w = *reinterpret_cast<const uint16_t*>(vk + 16 * (32 * d + 8 * (r >> 2) + (r & 3)));
          acc[d][r] += in && (w & 0x7f80u) == 0x7f80u ? bf16_bits_to_float(w) : 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // One tile.  MASKED: some key is hidden from some row of the wave.
  auto tile = [&](auto masked, const char* kv, int key0) {
    constexpr bool MASKED = decltype(masked)::value;
    const char* ks = kv + koff;
    const char* vs = kv + kTileBytes;
    f32x16 sv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) sv[h][r] = 0.0f;
#pragma unroll
    for (int i = 0; i < DK; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        sv[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const u32x4*>(ks + 2 * h * kBlk + 512 * i)), qf[i], sv[h], 0, 0, 0);
    // score (h, 8 w + e) of the lane is of key key0 + 32 h + 16 w + 8 half + e
    const int hkey = key0 + 8 * half;
    const Mask mask = {pos - hkey, rlow - hkey, rpre - hkey};
    float x[32];
    float mx = kNegInf;
    if (MASKED || EXTRA) {
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int j = 32 * (e >> 4) + 16 * ((e >> 3) & 1) + (e & 7);
        x[e] = score2<EXTRA>(sv[e >> 4][e & 15], sc, slope2, j - mask.pos);
        if (MASKED) x[e] = visible(mask, j) ? x[e] : kNegInf;
        mx = fmaxf(mx, x[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 32; ++e) mx = fmaxf(mx, sv[e >> 4][e & 15]);
      mx *= sc.scale2;
    }
    if (__any(mx > m + kMaxSlack)) {
      const float m_new = fmaxf(m, halves_max(mx));
      const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
      m = m_new;
    }
    const float m0 = m == kNegInf ? 0.0f : m;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      x[e] = exp2_fast(MASKED || EXTRA ? x[e] - m0 : __builtin_fmaf(sv[e >> 4][e & 15], sc.scale2, -m0));
      l += x[e];
    }
    if (MASKED) asm volatile("" : "+v"(l));     // summed here: the weights' registers are needed below
    u32x4 p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[i][e] = bf16_pair(x[8 * i + 2 * e], x[8 * i + 2 * e + 1]);
    if (MASKED) {
      // a value that is not finite must not reach the rows that do not see it
      u16x2 most = {0, 0};
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i)
        most = magnitude_max(most, *reinterpret_cast<const u32x4*>(vs + voff + (i / DT) * kBlk + (i % DT) * 512));
      asm volatile("" : : : "memory");     // the tile is read again: its registers are needed elsewhere
      if (__any(most[0] >= 0x7f80 || most[1] >= 0x7f80)) {
        add_odd(vs, p, key0);
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const u32x4*>(vs + voff + i * kBlk + 512 * d)), as_bf16x8(p[i]), acc[d], 0, 0, 0);
  };

  // Round t: the loads of tile t + 1, then tile t.  The buffers are distinct and
  // passed as such: reads of one do not wait for the loads into the other.
  int page = t_begin < t_end ? page_of(t_begin) : 0;     // of tile t + 1
  auto round = [&](char* __restrict__ cur, char* __restrict__ nxt, int t) {
    const int key0 = tile_key(t);
    if (t >= t_begin && key0 + kPreKeys > len) {
      // what lies behind the sequence may be anything: no value of it counts
      int i = threadIdx.x;
      asm volatile("" : "+v"(i));
#pragma unroll 1
      for (; i < kTileBytes / 16; i += kPreThreads) {
        // unit i of the value tile: block i / (2D), token group (i / D) % 2
        const int over = key0 + 16 * (i / (2 * D)) + 8 * ((i / D) & 1) + 8 - len;   // hidden tokens of the unit
        if (over > 0) {
          u32x4 w = *reinterpret_cast<u32x4*>(cur + kTileBytes + 16 * i);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = over >= 8 - 2 * e ? 0u : over == 7 - 2 * e ? w[e] & 0xffffu : w[e];
          *reinterpret_cast<u32x4*>(cur + kTileBytes + 16 * i) = w;
        }
      }
      lds_barrier();
    }
    if (t + 1 < t_end) {
      const int next = page_of(t + 2);
      fetch(t + 1, nxt, page);
      page = next;
    }
    if (t >= t_begin && wave_live && (key0 <= wpos_last || key0 < pre)) {
      const bool whole = (wpos_first >= 0 && key0 + kPreKeys <= pre) ||
                         (key0 + kPreKeys - 1 <= wpos_first && (a.window == 0 || key0 > wpos_last - a.window));
      if (whole)
        tile(std::false_type{}, cur, key0);
      else
        tile(std::true_type{}, cur, key0);
    }
    if (E4 && t + 1 < t_end) put(nxt);
  };
  for (int t = t_begin - 1; t < t_end; ++t) {
    // tile t is in LDS once every wave's loads are; the barrier also ends every
    // wave's reads of the other buffer
    if constexpr (!E4) wait_vmcnt<0>();
    lds_barrier();
    round(s_kv[t & 1], s_kv[(t + 1) & 1], t);
  }

  l = halves_sum(l);
  if (!live) return;
  const float m0 = m == kNegInf ? 0.0f : m;
  const size_t out_row = (size_t)(first + tok);
  if (sp.nsplit > 1) {
    const size_t part = (out_row * a.Hq + head) * sp.nsplit + split;
    if (half == 0) {
      sp.ml[2 * part] = m0;
      sp.ml[2 * part + 1] = l;
    }
    if (l == 0.0f) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 w = {acc[d][4 * r], acc[d][4 * r + 1], acc[d][4 * r + 2], acc[d][4 * r + 3]};
        *reinterpret_cast<f32x4*>(sp.o + part * D + 32 * d + 8 * r + 4 * half) = w;
      }
    return;
  }
  const float f = l == 0.0f ? 0.0f : (E4 ? c.v_scale[hk] : 1.0f) / l;
  uint16_t* out = o.p + out_row * o.stride + (size_t)head * D + 4 * half;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      u32x2 w = {0u, 0u};
      if (l != 0.0f) {
        w[0] = bf16_pair(acc[d][4 * r] * f, acc[d][4 * r + 1] * f);
        w[1] = bf16_pair(acc[d][4 * r + 2] * f, acc[d][4 * r + 3] * f);
      }
      *reinterpret_cast<u32x2*>(out + 32 * d + 8 * r) = w;
    }
  if (lse && half == 0) lse[out_row * a.Hq + head] = l == 0.0f ? kNegInf : (m0 + __log2f(l)) * kLn2;
}

template <int D, bool E4>
static void prefill_launch(RowsIn q, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a, RowsOut o, float* lse,
                           const SplitArgs& sp, int slots, hipStream_t stream) {
  const dim3 grid((unsigned)((size_t)slots * c.Hkv * sp.nsplit));
  if (a.softcap > 0.0f || a.slopes)
    hipLaunchKernelGGL((attn_prefill_kernel<D, E4, true>), grid, dim3(kPreThreads), 0, stream, q, b, c, a, o, lse, sp,
                       slots);
  else
    hipLaunchKernelGGL((attn_prefill_kernel<D, E4, false>), grid, dim3(kPreThreads), 0, stream, q, b, c, a, o, lse,
                       sp, slots);
}

hipError_t launch_attn_prefill(RowsIn q, int D, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a, RowsOut o,
                               float* lse, int max_len, void* ws, hipStream_t stream) {
  const bool e4 = c.k_scale != nullptr;
  const int slots = prefill_slots(b.T, b.S, a.g);
  if (a.window > 0 && !a.prefix && a.window + kPreRows < max_len) max_len = a.window + kPreRows;
  SplitArgs sp;
  sp.nsplit = prefill_splits(slots, c.Hkv, max_len);
  sp.o = static_cast<float*>(ws);
  sp.ml = sp.o + (size_t)b.T * a.Hq * sp.nsplit * D;
  timing_begin(stream, kSiteAttnPrefill);
  if (D == 64)
    e4 ? prefill_launch<64, true>(q, b, c, a, o, lse, sp, slots, stream)
       : prefill_launch<64, false>(q, b, c, a, o, lse, sp, slots, stream);
  else
    e4 ? prefill_launch<128, true>(q, b, c, a, o, lse, sp, slots, stream)
       : prefill_launch<128, false>(q, b, c, a, o, lse, sp, slots, stream);
  timing_end(stream, kSiteAttnPrefill);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit == 1) return err;
  return launch_attn_join(sp, b.T, a.Hq, a.g, D, c.v_scale, o, lse, &b, stream);
}

}  // namespace mc
