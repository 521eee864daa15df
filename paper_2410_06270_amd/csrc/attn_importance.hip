// attn_importance.hip -- token importance (Sec. 3.3.2, Eq. 6) from a prompt's
// queries, its cached keys and the softmax statistics of its attention, without
// an attention map.
//
//   I_j = ||x_j||_1 * (1/Hq) * sum_h sum_{i >= j} exp(s_hij - lse_hi) / (L - j)
//
// A map would be Hq L^2 bf16 values, written and read; here each probability is
// formed again where it is summed, one matrix product (half of the attention's)
// and one exponential a pair.  Bound by the vector units: 16 pairs a lane of a 32 x 32
// tile cost 8 matrix instructions (256 cycles of a SIMD for D = 128) and 16 x (an
// exponential, a multiply-add and an add: 24 cycles).  4096 tokens of 32 query heads over
// 8: 96 us in all, what reading the lower half of a map takes alone (0.54 GB); 0.82
// PFLOP/s in the sums' kernel; 16384 tokens: 1.12 ms, 0.98 PFLOP/s.
//
// attn_colsum_kernel: a workgroup keeps 256 keys of one key-value head in
// registers (64 a wave) and walks the rows below the diagonal, 32 at a time, of each of
// the head's query heads; the queries come through LDS, a ring of 4 tiles.  Scores are keys x
// rows, so a lane adds its own row's probabilities to 32 sums, one a key, and the 32
// lanes' sums are joined once at the end.  The rows are dealt out to `slices` workgroups.
// attn_finish_kernel: one wave a key: its partial sums, the norm of x_j, I_j and
// the selection key that importance_select takes.
#include "attn.hpp"

namespace mc {

constexpr int kColWaves = 4;
constexpr int kColThreads = 64 * kColWaves;
constexpr int kColKeys = 64 * kColWaves;      // keys of a workgroup

__host__ __device__ static inline int col_tiles(int L) { return (L + kColKeys - 1) / kColKeys; }

// Row slices of a (key tile, key-value head).  A workgroup costs some 5 us of
// loading its keys and joining its sums, a round of the loop under 1: about kColRounds
// rounds each, between two workgroups a CU and eight (which evens out the triangle).
constexpr int kColRounds = 32, kColLeast = 512, kColMost = 2048;

static int col_slices(int L, int Hkv, int g) {
  const long long tiles = (L + 31) / 32, wgs = (long long)col_tiles(L) * Hkv;
  long long want = wgs * tiles * g / 2 / kColRounds;
  want = want < kColLeast ? kColLeast : want > kColMost ? kColMost : want;
  const long long n = (want + wgs - 1) / wgs, most = tiles * g;
  return (int)(n > most ? most : n);
}

static size_t up256(size_t b) { return (b + 255) / 256 * 256; }

static size_t col_partial_bytes(int L, int Hkv, int g) {
  return up256((size_t)col_tiles(L) * kColKeys * Hkv * col_slices(L, Hkv, g) * sizeof(float));
}

// Workspace: partial sums [Hkv * slices][tiles * 256] | selection keys.  The
// slices depend on the number of key-value heads, which divides Hq.
size_t attn_importance_bytes(int Hq, int L) {
  size_t most = 0;
  for (int Hkv = 1; Hkv <= Hq; ++Hkv)
    if (Hq % Hkv == 0) {
      const size_t b = col_partial_bytes(L, Hkv, Hq / Hkv);
      if (b > most) most = b;
    }
  return most + up256((size_t)L * sizeof(uint64_t));
}

// Row tiles in flight: one is a few microseconds of memory latency away, its
// products a fraction of one.
constexpr int kColRing = 4;

template <int D, int KV, int MODE>
__global__ void __launch_bounds__(kColThreads, 2)
    attn_colsum_kernel(RowsIn q, const float* __restrict__ lse, BatchArgs b, KvArgs c, ScoreArgs a, int L, int slices,
                       float* __restrict__ partial) {
  constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  constexpr int DK = D / 16, kBlockBytes = KvFormat<D, KV>::kBlockBytes, kRowBytes = 32 * D * 2;
  constexpr int kLoads = D / 64 + 1;            // direct loads of a wave for a row tile
  // a tile's queries, then its rows' lse: a copy for each wave, twice over the half waves
  constexpr int kSlotBytes = kRowBytes + kColWaves * 256;
  __shared__ __attribute__((aligned(16))) char s_ring[kColRing * kSlotBytes];
  const int lane = threadIdx.x & 63, wave = wave_id(), n = lane & 31, half = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % c.Hkv;
  id /= c.Hkv;
  const int slice = id % slices, tile = id / slices;     // the first keys have the most rows: they go first
  const int key0 = tile * kColKeys + 64 * wave;

  f32x16 acc[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[h][r] = 0.0f;
  const float kscale = E4 ? c.k_scale[hk] : 1.0f;
  const ScoreConsts sc = score_consts(a.scale * kscale, a.softcap);

  // (row tile, head of the group) pairs, from the diagonal down: pair y is head
  // y % g of row tile t0 + y / g; this workgroup takes slice, slice + slices, ...
  const int t0 = tile * (kColKeys / 32), nt = (L + 31) / 32;
  const long long wend = a.window > 0 ? ((long long)(tile + 1) * kColKeys + a.window - 2) / 32 + 1 : nt;
  const int t1 = wend < nt ? (int)wend : nt;
  const int pairs = (t1 - t0) * a.g, count = pairs > slice ? (pairs - slice + slices - 1) / slices : 0;
  const int step_t = slices / a.g, step_h = slices - step_t * a.g;
  auto next = [&](int& t, int& h) {
    t += step_t;
    h += step_h;
    if (h >= a.g) {
      h -= a.g;
      ++t;
    }
  };
  // LDS: unit (u, row) of the tile at u * 512 + row * 16, so that a step's read is
  // contiguous; wave w copies a quarter of the units
  int ft = t0 + slice / a.g, fh = slice % a.g;           // the next pair to fetch
  int ct = ft, ch = fh;                                  // the next to work on
  auto fetch = [&](char* slot) {
    const int head = hk * a.g + fh, row = min(n, L - 1 - 32 * ft);      // of the tile
    const Buffer src = buffer_of(q.p + (size_t)(32 * ft) * q.stride + (size_t)head * D, 0x7fffffff);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const int u = 2 * (D / 64 * wave + i);
      lds_dma16<0>(src, row * (2 * (int)q.stride) + 16 * half, 16 * u, slot + u * 512);
    }
    lds_dma4(buffer_of(lse + (size_t)(32 * ft) * a.Hq + head, 0x7fffffff), row * (4 * a.Hq),
             slot + kRowBytes + 256 * wave);
    next(ft, fh);
  };

  // the first tiles' loads, then the keys', and a wait for all of them: the
  // compiler would otherwise wait for the keys, and with them for every tile, in each
  // round
#pragma unroll
  for (int i = 0; i < kColRing - 1; ++i)
    if (i < count) fetch(s_ring + i * kSlotBytes);
  // keys: lane (key n of 32, half) holds units half, half + 2, ... (bf16), or units of
  // 16 whose first and last 8 dimensions go to two steps (e4m3), or of 32 that go to four (e2m1).
  bf16x8 kf[2][DK];
  const int last_blk = (L - 1) >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int blk = min((key0 + 32 * h + n) >> 4, last_blk);
    const int page = kv_page(c, b.page_table[blk >> c.lb]);
    const char* kp = c.k + kv_block_offset<kBlockBytes>(c, page, hk, blk) + (n & 15) * 16 + half * 256;
    if constexpr (E4) {
#pragma unroll
      for (int i = 0; i < DK / 2; ++i) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(kp + 512 * i);
        kf[h][2 * i] = as_bf16x8(e4m3_to_bf16(r[0], r[1]));
        kf[h][2 * i + 1] = as_bf16x8(e4m3_to_bf16(r[2], r[3]));
      }
    } else if constexpr (E2) {
      const uint8_t* ks = reinterpret_cast<const uint8_t*>(c.k + kv_scale_offset<D>(c, page, hk, blk));
#pragma unroll
      for (int i = 0; i < DK / 4; ++i) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(kp + 512 * i);
        const float scale = __uint_as_float((uint32_t)ks[16 * (2 * i + half) + 4 * (n & 3) + ((n & 15) >> 2)] << 23);
#pragma unroll
        for (int u = 0; u < 4; ++u) kf[h][4 * i + u] = as_bf16x8(e2m1_to_bf16(r[u], scale));
      }
    } else {
#pragma unroll
      for (int i = 0; i < DK; ++i) kf[h][i] = as_bf16x8(*reinterpret_cast<const u32x4*>(kp + 512 * i));
    }
  }

  wait_vmcnt<0>();

  // Products of a tile: keys 32 h + 8 (r / 4) + 4 half + r % 4 of row n.
  auto qk = [&](const char* slot, f32x16 (&sv)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) sv[h][r] = 0.0f;
#pragma unroll
    for (int i = 0; i < DK; ++i) {
      // unit 2 i + half, or for e4m3 units 2 (i & ~1) + 2 half + (i & 1), for e2m1 2 (i & ~3) + 4
      // half + (i & 3): the dimensions of the key's unit
      const int u = E2 ? 2 * (i & ~3) + 4 * half + (i & 3) : E4 ? 2 * (i & ~1) + 2 * half + (i & 1) : 2 * i + half;
      const bf16x8 qv = as_bf16x8(*reinterpret_cast<const u32x4*>(slot + u * 512 + n * 16));
#pragma unroll
      for (int h = 0; h < 2; ++h) sv[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[h][i], qv, sv[h], 0, 0, 0);
    }
  };
  // Adds a tile's probabilities.
  struct Tile {
    int row0;
    float ls, slope2;    // log2(e) lse of the lane's row; of its head
    bool live, masked;   // reaches below the wave's diagonal; not wholly
  };
  auto add = [&](auto masked, const f32x16 (&sv)[2], const Tile& t) {
    constexpr bool MASKED = decltype(masked)::value;
    const int row = t.row0 + n, key = key0 + 4 * half;
    const float dist = (float)(key - row);
    const int low = (a.window > 0 && row >= a.window ? row - a.window : -1) - key, high = (row < L ? row : -1) - key;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = 32 * h + 8 * (r >> 2) + (r & 3);
        float p = exp2_fast(MODE ? score2<MODE>(sv[h][r], sc, t.slope2, dist + (float)j) - t.ls
                                 : __builtin_fmaf(sv[h][r], sc.scale2, -t.ls));
        if (MASKED) p = ((j <= high) & (j > low)) ? p : 0.0f;
        acc[h][r] += p;
      }
  };

  // Round i: the products of tile i beside the probabilities of tile i - 1.  Slots
  // of the ring are distinct and passed as such: a read of the current one then does
  // not wait for the loads into the others.
  Tile prev = {0, 0.0f, 0.0f, false, false};
  auto round = [&](const char* __restrict__ cur, char* __restrict__ nxt, f32x16 (&sv)[2], f32x16 (&sp)[2], int i) {
    if (i + kColRing - 1 < count) fetch(nxt);
    Tile t = {32 * ct, 0.0f, 0.0f, false, false};
    if (i < count) {
      t.slope2 = MODE & 2 ? a.slopes[hk * a.g + ch] * kLog2e : 0.0f;
      next(ct, ch);
      t.live = t.row0 + 31 >= key0;
      t.masked = !(t.row0 >= key0 + 63 && t.row0 + 32 <= L && (a.window == 0 || t.row0 + 31 - key0 < a.window));
      const float v = *reinterpret_cast<const float*>(cur + kRowBytes + 256 * wave + 4 * lane);
      t.ls = v == kNegInf ? -kNegInf : v * kLog2e;       // a row without keys: every probability 0
    }
    if (t.live && prev.live && !prev.masked) {
      // the wave with matrix work goes first (4096 tokens of 32 heads over 8: 101 -> 96 us)
      __builtin_amdgcn_s_setprio(1);
      qk(cur, sv);
      add(std::false_type{}, sp, prev);
      // LDS reads ahead of their products, and between the products the vector work
      __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
      for (int m = 0; m < 2 * DK; ++m) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (m & 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 96 / (2 * DK), 0);
      }
      __builtin_amdgcn_s_setprio(0);
    } else {
      if (t.live) qk(cur, sv);
      if (prev.live) {
        if (prev.masked)
          add(std::true_type{}, sp, prev);
        else
          add(std::false_type{}, sp, prev);
      }
    }
    prev = t;
  };
  f32x16 sa[2], sb[2];
  auto begin_round = [&](int i) {
    // tile i's loads are the oldest of those of up to kColRing - 1 tiles; the
    // barrier also ends every wave's reads of the slot that the next fetch overwrites
    if (i + kColRing - 2 < count)
      wait_vmcnt<(kColRing - 2) * kLoads>();
    else
      wait_vmcnt<0>();
    lds_barrier();
  };
  auto slot_of = [&](int i) { return s_ring + (i % kColRing) * kSlotBytes; };
  for (int i = 0; i <= count; i += 2) {
    begin_round(i);
    round(slot_of(i), slot_of(i + kColRing - 1), sa, sb, i);
    if (i == count) break;
    begin_round(i + 1);
    round(slot_of(i + 1), slot_of(i + kColRing), sb, sa, i + 1);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[h][r] = half_wave_sum(acc[h][r]);
  if (n == 0) {
    float* out = partial + ((size_t)hk * slices + slice) * col_tiles(L) * kColKeys + key0 + 4 * half;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 w = {acc[h][4 * r], acc[h][4 * r + 1], acc[h][4 * r + 2], acc[h][4 * r + 3]};
        *reinterpret_cast<f32x4*>(out + 32 * h + 8 * r) = w;
      }
  }
}

// One wave a key, 4 a workgroup: the parts over the lanes, then the row of x.
constexpr int kFinishThreads = 256;

__global__ void __launch_bounds__(kFinishThreads) attn_finish_kernel(const float* __restrict__ partial, int parts,
                                                                     int Hq, int L, const uint16_t* __restrict__ x,
                                                                     int d, bool xvec, float* __restrict__ importance,
                                                                     uint64_t* __restrict__ keys) {
  const int lane = threadIdx.x & 63;
  const int j = blockIdx.x * (kFinishThreads / 64) + wave_id();
  if (j >= L) return;
  float cs = 0.0f;
  const size_t stride = (size_t)col_tiles(L) * kColKeys;
#pragma unroll 4
  for (int i = lane; i < parts; i += 64) cs += partial[(size_t)i * stride + j];
  float n1 = 0.0f;
  const uint16_t* xr = x + (size_t)j * d;
  if (xvec) {
    // eight loads at a time: latency is what a row's few loads cost
    for (int i = 8 * lane; i < d; i += 8 * 512) {
      u32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (i + 512 * u < d) v[u] = *reinterpret_cast<const u32x4*>(xr + i + 512 * u);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          n1 += fabsf(bf16_bits_to_float(v[u][e] & 0xffffu)) + fabsf(bf16_bits_to_float(v[u][e] >> 16));
    }
  } else {
    for (int i = lane; i < d; i += 64) n1 += fabsf(bf16_bits_to_float(xr[i]));
  }
  cs = wave_sum(cs);
  n1 = wave_sum(n1);
  if (lane == 0) {
    const float I = n1 * (cs / (float)Hq) / (float)(L - j);
    if (importance) importance[j] = I;
    // I >= 0: its bits order like the value; ~j puts lower indices first
    keys[j] = ((uint64_t)__float_as_uint(I) << 32) | (uint64_t)(0xffffffffu - (uint32_t)j);
  }
}

template <int D, int KV>
static void colsum_launch(RowsIn q, const float* lse, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a, int L,
                          int slices, float* partial, hipStream_t stream) {
  const dim3 grid((unsigned)((size_t)col_tiles(L) * slices * c.Hkv));
  with_score_mode(a, [&](auto mode) {
    hipLaunchKernelGGL((attn_colsum_kernel<D, KV, decltype(mode)::value>), grid, dim3(kColThreads), 0, stream, q,
                       lse, b, c, a, L, slices, partial);
  });
}

hipError_t launch_attn_importance(RowsIn q, const float* lse, int D, const BatchArgs& b, const KvArgs& c,
                                  const ScoreArgs& a, const uint16_t* x, int d, float rho, float* importance,
                                  uint8_t* mask, void* ws, hipStream_t stream) {
  const int L = b.T, slices = col_slices(L, c.Hkv, a.g);
  float* partial = static_cast<float*>(ws);
  uint64_t* keys = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + col_partial_bytes(L, c.Hkv, a.g));
  timing_begin(stream, kSiteAttnColsum);
  with_kv_kind(c, [&](auto kind) {
    constexpr int KV = decltype(kind)::value;
    D == 64 ? colsum_launch<64, KV>(q, lse, b, c, a, L, slices, partial, stream)
            : colsum_launch<128, KV>(q, lse, b, c, a, L, slices, partial, stream);
  });
  timing_end(stream, kSiteAttnColsum);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const bool xvec = (d % 8) == 0 && (reinterpret_cast<uintptr_t>(x) % 16) == 0;
  timing_begin(stream, kSiteAttnFinish);
  hipLaunchKernelGGL(attn_finish_kernel, dim3((L + 3) / 4), dim3(kFinishThreads), 0, stream, partial,
                     c.Hkv * slices, a.Hq, L, x, d, xvec, importance, keys);
  timing_end(stream, kSiteAttnFinish);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  return launch_importance_select(keys, L, rho, mask, stream);
}

}  // namespace mc
