// attn_prefill.hip -- causal attention of prompts and prompt chunks over the
// paged cache.
//
//   o_i = sum_j p_ij v_j / l_i,  p_ij = exp2(s_ij - m_i),  l_i = sum_j p_ij
// in one pass over the keys with a running maximum m_i for each row.
//
// Bound by the matrix units, and by the vector units beside them: a wave's 32 rows x 64
// keys cost 32 matrix instructions of 32x32x16 for D = 128 (1024 cycles of a SIMD), and 32
// exponentials and some 105 other vector instructions (800 cycles).  Each wave has both in
// every round, the vector work of one tile beside the products of the next.  8192 tokens
// of 32 query heads over 8: 528 us, 1.04 PFLOP/s (the library's product of two 8192 x
// 8192 matrices reaches 1.19, and this loop with nothing but its products 1.33: the
// clock falls under matrix load); 4096 of 16 heads: 83 us, 0.83, matrix units busy half of
// the time, as late row tiles end alone: with a prefix of all 4096 every row tile has 64 tiles of
// keys, and 33/64 of that call's 129 us would be 67.
//
// A workgroup of four waves (or two teams of four, each half of the keys) takes 128
// rows of one sequence and key-value head; the g query heads that share it are packed into
// the rows (row = token * g + head), so a short chunk fills a tile with heads and a tile's rows span few
// positions.  Keys and values come through LDS in tiles of 64, two buffers;
// the cache's 16-byte units are already the order in which the matrix
// instructions read them, so a bf16 tile is copied straight to LDS by direct
// loads and read without bank conflicts; e4m3 is widened on the way (exactly).
// Scores are keys x rows (S^T = K Q^T): a lane holds 16 keys of ONE row, so the
// row's maximum and sum are in-lane but for one exchange between the half waves,
// and the score rows are dealt so that the lane's keys are the ones that it
// supplies to O^T = V^T P^T: the weights never leave their registers.
#include "attn.hpp"

namespace mc {

constexpr int kPreWaves = 4;
constexpr int kPreThreads = 64 * kPreWaves;
constexpr int kPreRows = 32 * kPreWaves;      // rows of a workgroup
constexpr int kPreKeys = 64;                  // keys of a tile

// Row tiles: sequence s owns slots floor(q_start[s] g / 128) + s and on, at
// least ceil(rows / 128) of them.
static int prefill_slots(int T, int S, int g) {
  return (int)(((long long)T * g + kPreRows - 1) / kPreRows) + S - 1;
}

// Few row tiles are split over the keys, below kPreTarget workgroups (two a
// CU), each with 512 keys at least.  (Not at one a CU: a wave alone on its SIMD gets 90 %
// of what two get for heads of 128, and the join would cost more.)
constexpr int kPreTarget = 512, kPreMaxSplit = 32;

static int prefill_splits(int slots, int Hkv, int max_len) {
  long long n = (kPreTarget - 1) / ((long long)slots * Hkv);
  const int most = (max_len + 511) / 512;
  n = n > most ? most : n;
  return (int)(n < 1 ? 1 : n > kPreMaxSplit ? kPreMaxSplit : n);
}

// Heads of 64, whose products are half as long, leave a lone wave waiting for 30 % of its
// time, and a row tile is as long as its keys are many.  Up to two workgroups a CU that
// are not split take two teams of waves, each half of the keys, joined in LDS (32 query
// heads over 8 key-value heads, one prompt of 1024 tokens: 23.0 -> 19.4 us, of 2048: 41.8
// -> 38.8; chunks of 2048 over 14000 tokens, 16 heads: 253 -> 179); more keep one (4096
// tokens of 32 heads: 101, with two 120), and so do short ones (256 tokens: 10.2, with two
// 10.4).  Heads of 128: no difference (4096 tokens of 16 heads 85.3, with two 85.8).
static bool prefill_two_teams(int slots, int Hkv, int nsplit, int max_len) {
  return nsplit == 1 && (long long)slots * Hkv <= kPreTarget && max_len >= 512;
}

// T g / 128 <= slots and nsplit slots Hkv < kPreTarget where nsplit > 1, so a split call has at
// most 128 kPreTarget partial rows.
size_t attn_prefill_split_rows(int T, int Hq) {
  const size_t all = (size_t)T * Hq * kPreMaxSplit, most = (size_t)kPreRows * kPreTarget;
  return all < most ? all : most;
}

// The running maximum follows a larger score only when it is left behind by more
// than this (log2): weights up to 2^8 lose nothing in fp32 sums or in bf16, and most
// tiles need no scaling and no exchange between the half waves.
constexpr float kMaxSlack = 8.0f;

// Plain scores are multiplied out with the maximum's subtraction, unrounded, while the
// maximum is a rounded product: the largest weight is then 2^(2^-24 |m|) either way.  From this
// maximum on (log2), where that passes 2^-11 and nears a weight's rounding, a wave takes every
// tile the way of masked ones, whose scores are rounded first, as decode's are.  (It is looked at
// where the maximum moves.  2048 tokens over 14000, two teams: 172 us, tested at every tile 175,
// without 170.)
constexpr float kFarScore = 8192.0f;

// A tile of values that some row does not see whole.  Those behind its first n
// keys may be anything and become 0; so do infinities and NaN, which a weight of 0
// would not keep from the rows that do not see them.  Returns whether the thread met
// any of those (they are added to the rows that see them at the end).
template <int D>
__device__ __forceinline__ bool clean_values(char* vt, int n) {
  uint32_t odd = 0;
#pragma unroll 1
  for (int i = threadIdx.x % kPreThreads; i < kPreKeys * D / 8; i += kPreThreads) {
    // unit i of the tile: block i / (2D), token group (i / D) % 2
    const int over = 16 * (i / (2 * D)) + 8 * ((i / D) & 1) + 8 - n;      // hidden tokens of the unit
    u32x4 w = *reinterpret_cast<u32x4*>(vt + 16 * i);
    bool change = over > 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = over >= 8 - 2 * e ? 0u : over == 7 - 2 * e ? w[e] & 0xffffu : w[e];
      const uint32_t lo = (w[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u;
      const uint32_t hi = (w[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
      odd |= lo | hi;
      change = change || (lo | hi);
      w[e] &= ~(lo | hi);
    }
    if (change) *reinterpret_cast<u32x4*>(vt + 16 * i) = w;
  }
  return odd != 0;
}

// The order of a round's instructions: LDS reads some matrix instructions before their
// use, and the vector work (some 135 instructions) spread over the spaces between all of
// them: the first products with the values need only the first weights.  Heads of 128, 32
// products: 3 instructions a space (8192 tokens of 32 heads over 8: 528 us, with 4 532 and
// with 5 543); of 64, 16 products: 10 and reads 3 ahead (2048 tokens over 14000 175 us,
// with 8 and 5 ahead 178).
template <int DK, int DT>
__device__ __forceinline__ void interleave() {
  constexpr int kMfmas = 2 * DK + 4 * DT, kReadAhead = DT == 2 ? 3 : 5, kVector = DT == 2 ? 10 : 3;
  __builtin_amdgcn_sched_group_barrier(0x100, kReadAhead, 0);      // LDS reads
#pragma unroll
  for (int i = 0; i < kMfmas; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);             // matrix
    if (i + kReadAhead < kMfmas) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, kVector, 0);  // vector
  }
}

// MODE: as score2 (attn.hpp).
template <int D, bool E4, int MODE, int G>
__global__ void __launch_bounds__(G * kPreThreads, 2)
    attn_prefill_kernel(RowsIn q, BatchArgs b, KvArgs c, ScoreArgs a, RowsOut o, float* __restrict__ lse, SplitArgs sp,
                        int slots) {
  constexpr int DT = D / 32, DK = D / 16;      // value tiles; score steps
  constexpr int kTileBytes = kPreKeys * D * 2, kBlk = kKvBlock * D * 2;      // in LDS: bf16
  constexpr int kBlockBytes = kKvBlock * D * (E4 ? 1 : 2);                   // in the cache
  constexpr int kPieces = kBlockBytes / 1024, kUnit = E4 ? 16 : 8;
  // one array: for several the compiler keeps marks of its own that replace those
  // of the parameters of round() below, and then waits for every load before a read
  constexpr int kTeamBytes = 4 * kTileBytes + (E4 ? kPreWaves * 2 * kBlockBytes : 0);
  __shared__ __attribute__((aligned(16))) char s_all[G * kTeamBytes];
  const int team = G == 1 ? 0 : wave_id() / kPreWaves, wave = wave_id() % kPreWaves;
  char* const s_lds = s_all + team * kTeamBytes;
  char* const s_k[2] = {s_lds, s_lds + kTileBytes};
  char* const s_v[2] = {s_lds + 2 * kTileBytes, s_lds + 3 * kTileBytes};
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % c.Hkv;
  id /= c.Hkv;
  const int split = id % sp.nsplit;
  // Later rows see more keys: the later half of the row tiles goes first, from the
  // last on, then the other from the first on, so that where all workgroups are on the chip
  // at once a CU has a long and a short one (4096 tokens of 16 heads, 512 workgroups: 92.1
  // us from the last to the first, 86.6 so).  Of two teams a CU holds one workgroup, and the
  // first to end takes the next: from the last to the first (4096 tokens, 16 heads over 4: 68.5
  // us by halves, 57.0 so).
  const int turn = id / sp.nsplit, later = (slots + 1) / 2;
  const int slot = G > 1 || turn < later ? slots - 1 - turn : turn - later;
  const int s = find_sequence(b.q_start, b.S, slot, kPreRows, 1, a.g);
  int first, count;
  sequence_rows(b, s, first, count);
  const long long slot0 = (long long)b.q_start[s] * a.g / kPreRows + s;
  const long long row0l = (slot - slot0) * kPreRows;
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
  int wpos_first = pos0 + wrow / a.g;
  const int wpos_last = pos0 + min(wrow + 31, count * a.g - 1) / a.g;

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
  const int tiles = max(0, ia + end - ib), per = (tiles + G * sp.nsplit - 1) / (G * sp.nsplit);
  auto end_of = [&](int tm) { return min(tiles, (split * G + tm + 1) * per); };
  const int t_end = end_of(team), t_begin = min((split * G + team) * per, t_end);
  const int rounds = end_of(0) - min(split * G * per, tiles);          // the first team's, no fewer than another's
  const int32_t* pages = b.page_table + (size_t)s * b.max_pages;
  const int last_blk = len > 0 ? (len - 1) >> 4 : 0;
  auto tile_key = [&](int t) { return (t < ia ? t : t - ia + ib) * kPreKeys; };
  // tiles of which every row sees every key (those within a prefix may be others)
  const int in_first =
      max(ia, (a.window > 0 && pos_last >= a.window ? (pos_last - a.window) / kPreKeys + 1 : 0) + ia - ib);
  const int in_count = max(0, (pos_first >= 0 ? (pos_first + 1) / kPreKeys : 0) + ia - ib - in_first);
  auto inside = [&](int t) { return (unsigned)(t - in_first) < (unsigned)in_count; };
  int wave_inside = in_count;                          // the wave's: 0 from far scores on

  // A tile's 4 blocks of keys and 4 of values: wave w takes block w of each, both
  // at the same offset.  The lanes find the offsets of 64 tiles together, from `known` on.
  int known = t_begin;
  uint32_t off_lo = 0, off_hi = 0;
  auto find_offsets = [&]() {
    const int blk = min((tile_key(min(known + lane, max(t_end - 1, 0))) >> 4) + wave, last_blk);
    const size_t off = kv_block_offset<kBlockBytes>(c, kv_page(c, pages[blk >> c.lb]), hk, blk);
    off_lo = (uint32_t)off;
    off_hi = (uint32_t)(off >> 32);
  };
  auto fetch = [&](const char* from, size_t off, char* to) {
    const Buffer src = buffer_of(from + off, kBlockBytes);
    lds_dma16<0>(src, 16 * lane, 0, to);
    if constexpr (kPieces > 1) lds_dma16<1024>(src, 16 * lane, 0, to);
    if constexpr (kPieces > 2) {
      lds_dma16<2 * 1024>(src, 16 * lane, 0, to);
      lds_dma16<3 * 1024>(src, 16 * lane, 0, to);
    }
  };
  // e4m3: a fetched block's units, widened to bf16 units.  Unit x of the keys is
  // (16 dimensions, token): two bf16 units, 256 bytes apart; of the values (dimension,
  // 16 tokens): D * 16 apart.
  auto widen = [&](const char* raw, bool keys, char* to) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(raw + 1024 * i + 16 * lane);
      const int x = 64 * i + lane;
      char* d = to + (keys ? (x >> 4) * 512 + (x & 15) * 16 : x * 16);
      *reinterpret_cast<u32x4*>(d) = e4m3_to_bf16(w[0], w[1]);
      *reinterpret_cast<u32x4*>(d + (keys ? 256 : D * 16)) = e4m3_to_bf16(w[2], w[3]);
    }
  };

  f32x16 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
  float m = kNegInf, l = 0.0f;       // l: of the lane's own keys
  const float kscale = E4 ? c.k_scale[hk] : 1.0f, scale = fabsf(a.scale) * kscale;
  const ScoreConsts sc = score_consts(scale, a.softcap);
  const float slope2 = MODE & 2 ? a.slopes[head] * kLog2e : 0.0f;
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

  // Scores of a tile: (h, 8 w + e) of the lane is of key 32 h + 16 w + 8 half + e.
  auto qk = [&](const char* kt, f32x16 (&sv)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) sv[h][r] = 0.0f;
#pragma unroll
    for (int i = 0; i < DK; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        sv[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const u32x4*>(kt + koff + 2 * h * kBlk + 512 * i)), qf[i], sv[h], 0, 0, 0);
  };
  // Weights of a tile, from plain products (mul: the scale) or scores (mul: 1).  For
  // the matrix units they are rounded to bf16, by up to 2^-8 of each; their sum takes them as they
  // are, so that lse keeps fp32's precision and the roundings of o do not add up one way.
  auto weigh = [&](const f32x16 (&sv)[2], float mul, u32x4 (&p)[4]) {
    const float m0 = m == kNegInf ? 0.0f : m;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x[e] = exp2_fast(__builtin_fmaf(sv[i >> 3][(2 * i + e) & 15], mul, -m0));
        sum[e] += x[e];
      }
      p[i >> 2][i & 3] = bf16_pair(x[0], x[1]);
    }
    l += sum[0] + sum[1];
  };
  auto pv = [&](const char* vt, const u32x4 (&p)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const u32x4*>(vt + voff + i * kBlk + 512 * d)), as_bf16x8(p[i]), acc[d], 0, 0,
            0);
  };
  auto largest = [&](const f32x16 (&sv)[2]) {
    float mx[2] = {kNegInf, kNegInf};
#pragma unroll
    for (int e = 0; e < 32; ++e) mx[e >> 4] = fmaxf(mx[e >> 4], sv[e >> 4][e & 15]);
    return fmaxf(mx[0], mx[1]);
  };
  // A tile's scores in place of its products, where it is masked or the score is not
  // a multiple of the product, and the running maximum.  Returns what weigh multiplies by.
  auto settle = [&](f32x16 (&sv)[2], float mx, int t) {
    const int key0 = tile_key(t);
    // (those inside first: two teams, 2048 tokens over 14000, 175 -> 173 us; one team, 8192
    // tokens of heads of 64, no difference)
    const bool masked =
        (G == 1 || (unsigned)(t - in_first) >= (unsigned)wave_inside) &&
        !(((wpos_first >= 0) & (key0 + kPreKeys <= pre)) |
          ((key0 + kPreKeys - 1 <= wpos_first) & ((a.window == 0) | (key0 > wpos_last - a.window))));
    if (masked || MODE) {
      const int hkey = key0 + 8 * half;
      const Mask k = {pos - hkey, rlow - hkey, rpre - hkey};
      const float dist = (float)-k.pos;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int j = 32 * (e >> 4) + 16 * ((e >> 3) & 1) + (e & 7);
        sv[e >> 4][e & 15] = score2<MODE>(sv[e >> 4][e & 15], sc, slope2, dist + (float)j);
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const int j = 32 * (e >> 4) + 16 * ((e >> 3) & 1) + (e & 7);
          sv[e >> 4][e & 15] = visible(k, j) ? sv[e >> 4][e & 15] : kNegInf;
        }
      }
      mx = (MODE & 1) && !(MODE & 2) && !masked ? score2<MODE>(mx, sc, 0.0f, 0.0f) : largest(sv);
    } else {
      mx *= sc.scale2;
    }
    float mul = masked || MODE ? 1.0f : sc.scale2;
    if (__any(mx > m + kMaxSlack)) {
      const float m_new = fmaxf(m, halves_max(mx));
      const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
      m = m_new;
      if constexpr (!MODE) {
        if (__any(fabsf(m) > kFarScore && m != kNegInf)) {
          if (!masked) {
#pragma unroll
            for (int e = 0; e < 32; ++e) sv[e >> 4][e & 15] *= mul;
            mul = 1.0f;
          }
          wave_inside = 0;                             // every tile is masked
          wpos_first = -1;
        }
      }
    }
    return mul;
  };
  // a tile with a key that some row of the workgroup does not see
  auto edge = [&](int t) {
    const int key0 = tile_key(t);
    return !inside(t) && !(((pos_first >= 0) & (key0 + kPreKeys <= pre)) |
                           ((key0 + kPreKeys - 1 <= pos_first) & ((a.window == 0) | (key0 > pos_last - a.window))));
  };

  // Round t: the scores of tile t + 1 beside the weights of tile t, whose values
  // then are added up: the matrix units work on one tile while the vector units
  // work on the other.  Loads: keys of tile t + 2 and values of t + 1 (e4m3: of one
  // more, the ones before being widened).  The buffers are distinct and passed as
  // such: reads of one do not wait for the loads into another.
  size_t off_v = 0;                                    // of the next tile of values
  float mul = 1.0f;
  bool odd = false;
  char* raw_k = s_lds + 4 * kTileBytes + wave * 2 * kBlockBytes;      // e4m3 only
  char* raw_v = raw_k + (E4 ? kBlockBytes : 0);
  // the values of tile t - 1 and the keys of tile t
  auto load = [&](int t, char* kt, char* vt) {
    if (t > t_begin && t <= t_end) fetch(c.v, off_v, E4 ? raw_v : vt + wave * kBlk);
    if (t >= t_end) return;
    if (t == known + 64) {
      known = t;
      find_offsets();
    }
    off_v = (size_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, t - known) << 32 |
            (uint32_t)__builtin_amdgcn_readlane(off_lo, t - known);
    fetch(c.k, off_v, E4 ? raw_k : kt + wave * kBlk);
  };
  auto lds_done = [&]() {                              // what was read may be overwritten
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
    asm volatile("" ::: "memory");
  };
  auto round = [&](const char* __restrict__ kt, const char* __restrict__ vt, char* __restrict__ knext,
                   char* __restrict__ vnext, f32x16 (&cur)[2], f32x16 (&nxt)[2], int t) {
    if constexpr (E4) {
      if (t + 2 < t_end) widen(raw_k, true, knext + wave * kBlk);
      if (t + 1 < t_end) widen(raw_v, false, vnext + wave * kBlk);
      lds_done();
      load(t + 3, knext, vnext);
    } else {
      load(t + 2, knext, vnext);
    }
    if (wave_live && (G == 1 || t < t_end)) {
      // (the last round's next tile is whatever its buffer holds, and not used)
      // The wave with matrix work goes first: chunks of capped scores 366 -> 349 us, 8192
      // tokens of e4m3 570 -> 555; plain scores of heads of 64 lose (343 -> 347).
      constexpr bool kFirst = MODE || D == 128;
      if (kFirst) __builtin_amdgcn_s_setprio(1);
      u32x4 p[4];
      qk(kt, nxt);
      weigh(cur, mul, p);
      pv(vt, p);
      float mx = largest(nxt);
      asm volatile("" : "+v"(mx));                     // here, beside the products, not where it is used
      interleave<DK, DT>();
      if (kFirst) __builtin_amdgcn_s_setprio(0);
      if (t + 1 < t_end) mul = settle(nxt, mx, t + 1);
    }
  };
  // what the last round loaded is in LDS once every wave's loads are; the barrier
  // also ends every wave's reads of the buffers that are filled next
  auto begin_round = [&](char* vt, int t) {
    if constexpr (!E4) wait_vmcnt<0>();
    lds_barrier();
    if constexpr (E4) loads_landed();
    bool any = false;                                  // a tile of some team
#pragma unroll
    for (int tm = 0; tm < G; ++tm) {
      const int tt = (split * G + tm) * per + t - t_begin;
      any |= (G == 1 || tt < end_of(tm)) && edge(tt);
    }
    if (any) {
      if (G == 1 || (t < t_end && edge(t))) odd = clean_values<D>(vt, len - tile_key(t)) || odd;
      lds_barrier();
    }
  };
  if (rounds > 0) {
    f32x16 sa[2], sb[2];
    find_offsets();
    load(t_begin, s_k[0], s_v[1]);
    if constexpr (E4) {
      loads_landed();
      widen(raw_k, true, s_k[0] + wave * kBlk);
      lds_done();
    }
    load(t_begin + 1, s_k[1], s_v[0]);
    if constexpr (E4) {
      loads_landed();
      if (t_begin + 1 < t_end) widen(raw_k, true, s_k[1] + wave * kBlk);
      widen(raw_v, false, s_v[0] + wave * kBlk);
      lds_done();
      load(t_begin + 2, s_k[0], s_v[1]);
    } else {
      wait_vmcnt<0>();
    }
    lds_barrier();
    if (wave_live && (G == 1 || t_begin < t_end)) {
      qk(s_k[0], sa);
      mul = settle(sa, largest(sa), t_begin);
    }
    for (int t = t_begin; t < t_begin + rounds; t += 2) {
      begin_round(s_v[0], t);
      round(s_k[1], s_v[0], s_k[0], s_v[1], sa, sb, t);
      if (t + 1 == t_begin + rounds) break;
      begin_round(s_v[1], t + 1);
      round(s_k[0], s_v[1], s_k[1], s_v[0], sb, sa, t + 1);
    }
    // whether any wave met values that clean_values left out
    lds_barrier();
    const int any_odd = __any(odd) ? 1 : 0;
    int* flags = reinterpret_cast<int*>(s_k[0]);       // of the team
    if (lane == 0) flags[wave] = any_odd;
    lds_barrier();
    if (flags[0] | flags[1] | flags[2] | flags[3]) {
      // they go to the rows that see them: a weight is positive and changes neither an
      // infinity nor a NaN.  The lane sums dimensions 32 d + 8 (r / 4) + 4 half + r % 4.
#pragma unroll 1
      for (int i = 0; i < (t_end - t_begin) * kPreKeys; ++i) {
        const int t = t_begin + i / kPreKeys, j = tile_key(t) + i % kPreKeys;
        if (j >= len || !edge(t)) continue;
        const int blk = j >> 4, page = kv_page(c, pages[blk >> c.lb]), u = (j & 15) / kUnit;
        const char* vj = c.v + kv_block_offset<kBlockBytes>(c, page, hk, blk) + u * D * 16 + 64 * half +
                         (j % kUnit) * (E4 ? 1 : 2);
        const bool in = visible(Mask{pos, rlow, rpre}, j);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const char* at = vj + 16 * (32 * d + 8 * (r >> 2) + (r & 3));
            const uint32_t w = E4 ? *reinterpret_cast<const uint8_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
            const bool is_odd = E4 ? (w & 0x7fu) == 0x7fu : (w & 0x7f80u) == 0x7f80u;
            acc[d][r] += in && is_odd ? (E4 ? __builtin_nanf("") : bf16_bits_to_float(w)) : 0.0f;
          }
      }
    }
  }

  if constexpr (G > 1) {
    // join the teams: a lane of one holds the same row and dimensions as the lane of
    // the other, whose part comes by way of LDS
    f32x4* part = reinterpret_cast<f32x4*>(s_all) + wave * (16 * DT / 4 + 1) * 64 + lane;
    lds_barrier();
    if (team == 1) {
      part[0] = f32x4{m, l, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i)
        part[64 * (i + 1)] = f32x4{acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2],
                                   acc[i / 4][4 * (i % 4) + 3]};
    }
    lds_barrier();
    if (team == 1) return;
    const f32x4 ml = part[0];
    const float M = fmaxf(m, ml[0]);
    // (a part without a maximum joins one with it at factor 0, and its equal at 1)
    const float f0 = m == M ? 1.0f : exp2_fast(m - M), f1 = ml[0] == M ? 1.0f : exp2_fast(ml[0] - M);
    m = M;
    l = l * f0 + ml[1] * f1;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
      const f32x4 w = part[64 * (i + 1)];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i / 4][4 * (i % 4) + e] = acc[i / 4][4 * (i % 4) + e] * f0 + w[e] * f1;
    }
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
                           const SplitArgs& sp, int slots, int max_len, hipStream_t stream) {
  const dim3 grid((unsigned)((size_t)slots * c.Hkv * sp.nsplit));
  with_score_mode(a, [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    if constexpr (D == 64) {
      if (prefill_two_teams(slots, c.Hkv, sp.nsplit, max_len)) {
        hipLaunchKernelGGL((attn_prefill_kernel<D, E4, MODE, 2>), grid, dim3(2 * kPreThreads), 0, stream, q, b, c, a,
                           o, lse, sp, slots);
        return;
      }
    }
    hipLaunchKernelGGL((attn_prefill_kernel<D, E4, MODE, 1>), grid, dim3(kPreThreads), 0, stream, q, b, c, a, o, lse,
                       sp, slots);
  });
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
    e4 ? prefill_launch<64, true>(q, b, c, a, o, lse, sp, slots, max_len, stream)
       : prefill_launch<64, false>(q, b, c, a, o, lse, sp, slots, max_len, stream);
  else
    e4 ? prefill_launch<128, true>(q, b, c, a, o, lse, sp, slots, max_len, stream)
       : prefill_launch<128, false>(q, b, c, a, o, lse, sp, slots, max_len, stream);
  timing_end(stream, kSiteAttnPrefill);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit == 1) return err;
  return launch_attn_join(sp, b.T, a.Hq, a.g, D, c.v_scale, o, lse, &b, stream);
}

}  // namespace mc
