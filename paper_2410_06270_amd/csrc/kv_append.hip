// kv_append.hip -- new tokens into the paged cache: norm and rotation of
// queries and keys, keys and values to their places.
//
//   y = x * w / sqrt(mean(x^2) + eps);   (y_a, y_b) <- (y_a c - y_b s, y_a s + y_b c)
//
// One launch, two kinds of workgroup.  A value unit of the cache holds 8 or 16
// consecutive tokens of one dimension, so one lane reads 8 dimensions of all
// the tokens of a unit and writes whole units, transposed in its registers.  A key
// unit runs along the dimensions, and a norm over a row needs the whole row: one
// wave takes one token's queries and keys, 16 bytes a lane and load.  Bound by HBM, each
// byte moved once: 392 MB of chunks into e4m3 pages in 83 us, 4.7 TB/s; 199 MB of prompts
// with norms over rows, 53 us, 3.7 TB/s (a wave waits for its whole row); 64 tokens:
// 4.5 us, a chain of four memory latencies.  e2m1: 162 MB of prompts with norms over rows 57 us, 2.8 TB/s, the
// keys' arithmetic in 64 bits beside it; 64 tokens 6.1 us.
#include "attn.hpp"

namespace mc {

constexpr int kAppendThreads = 256;
// Chunks of 8 elements that a lane holds at once.
__host__ __device__ constexpr int row_chunks(int norm) { return norm == 2 ? 8 : 4; }

// The largest number of unit groups that n new tokens from q_start on touch is
// floor((n + 6) / U) + 1 (U = 8) and fewer for U = 16; sequence s owns the slots from
// floor(q_start[s] / U) + 2 s on, at least floor(n / U) + 2 of them.
__host__ __device__ static inline int append_slots(int T, int S, int U) { return T / U + 2 * S; }

// Where a token goes: false if it is skipped.
struct Place {
  int pos, page;
};
__device__ __forceinline__ bool append_place(const KvArgs& c, const BatchArgs& b, int s, long long pos, int n_pos,
                                             Place& out) {
  if (pos < 0 || pos >= kv_length(c, b, s) || pos >= n_pos) return false;
  out.pos = (int)pos;
  out.page = b.page_table[(size_t)s * b.max_pages + (size_t)((out.pos >> 4) >> c.lb)];
  return out.page >= 0 && out.page < c.n_pages;
}

// ------------------------------------------------------------------ e2m1 --
// Groups of e2m1 codes share a scale.  Of keys, 32 dimensions: 2^e, e the least with max|y| <=
// 7 2^e (7 being the border between 6, the largest level, and the next that there would be).  Of
// values, 64 dimensions: max|v| times the fp32 number nearest to 1/6, rounded to 6 significant bits so that its products with the codes
// are bf16 numbers.  Groups below 2^-100 are 0, those with a NaN, an infinity or more than 7 2^125 NaN.
constexpr float kGroupLeast = 0x1p-100f, kGroupMost = 0x1.cp127f;

// Byte of the scale 2^(byte - 127) of a group of keys whose largest magnitude is m (NaN: 255).
__device__ __forceinline__ uint32_t key_scale_byte(float m) {
  if (!(m <= kGroupMost)) return 255u;
  if (m < kGroupLeast) return 0u;
  const uint32_t b = __float_as_uint(m);
  // m = 2^k (1 + f): e = k - 2, or k - 1 where 1 + f > 7/4
  return (b >> 23) - 2u + ((b & 0x7fffffu) > 0x600000u ? 1u : 0u);
}

// The scale of a group of values (bf16) whose largest magnitude is m, as a float.
__device__ __forceinline__ float value_scale(float m) {
  if (!(m <= kGroupMost)) return __uint_as_float(0x7fc00000u);
  if (m < kGroupLeast) return 0.0f;
  uint32_t u = __float_as_uint(m * (1.0f / 6.0f));
  u += 0x1ffffu + ((u >> 18) & 1u);
  return __uint_as_float(u & ~0x3ffffu);
}

// The larger magnitude, NaN if one of them is (fmaxf would drop it).
__device__ __forceinline__ float magnitude(float a, float b) {
  a = fabsf(a);
  b = fabsf(b);
  return a >= b || a != a ? a : b;
}
// x of the lane that the DPP control names.
template <int CTRL>
__device__ __forceinline__ double dpp64(double x) {
  const unsigned long long b = __double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double(((long long)hi << 32) | lo);
}

// Two codes, each the nearest to x (ties to the even code, magnitudes above 6 to 6), the first in the
// low half; into byte `AT` of w.
template <int AT>
__device__ __forceinline__ uint32_t e2m1_pair(uint32_t w, float a, float b) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, 1.0f, AT);
}

// Eight codes in a word.
__device__ __forceinline__ uint32_t e2m1_word(const float (&x)[8]) {
  uint32_t w = 0;
  w = e2m1_pair<0>(w, x[0], x[1]);
  w = e2m1_pair<1>(w, x[2], x[3]);
  w = e2m1_pair<2>(w, x[4], x[5]);
  return e2m1_pair<3>(w, x[6], x[7]);
}

// a[i]'s nibble j to a[j]'s nibble i: single nibbles, then bytes, then halves.
__device__ __forceinline__ void transpose_nibbles(uint32_t (&a)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t x = a[i], y = a[i + 1];
    a[i] = (x & 0x0f0f0f0fu) | ((y & 0x0f0f0f0fu) << 4);
    a[i + 1] = ((x >> 4) & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = 4 * (k >> 1) + (k & 1);
    const uint32_t x = a[i], y = a[i + 2];       // bytes x0 y0 x2 y2, and x1 y1 x3 y3
    a[i] = __builtin_amdgcn_perm(y, x, 0x06020400u);
    a[i + 2] = __builtin_amdgcn_perm(y, x, 0x07030501u);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = a[i], y = a[i + 4];
    a[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    a[i + 4] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
}

// A double as a float that compares with every border of codes and scales (3 significant bits) as the
// double does: its first 24 bits, the last one set where any follow.  Numbers past a float's range,
// infinities and NaN become the largest float, those below it the smallest ones.  (With the
// groups' maxima in fp32 too, 8700 tokens with norms over rows took 58 us for 60.)
__device__ __forceinline__ float sticky_float(double v) {
  const unsigned long long b = __double_as_longlong(v);
  const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b;
  uint32_t h = hi & 0x7fffffffu;
  h = h < 0x38000000u ? 0x38000000u : h > 0x47efffffu ? 0x47efffffu : h;
  const uint32_t f = __builtin_amdgcn_alignbit(h - 0x38000000u, lo, 29), rest = lo & 0x1fffffffu;
  return __uint_as_float(f | (rest < 1u ? rest : 1u) | (hi & 0x80000000u));
}

// v / s, so exact that a quotient on a border of the codes is on it: v and s are bf16 numbers, whose
// quotient is a border (3 significant bits) or away from it by more than 2^-12 of itself, and where it
// is one the remainder of the first estimate corrects it to the last bit.
struct Divisor {
  float s, r;
  __device__ explicit Divisor(float scale) : s(scale), r(scale > 0.0f ? __builtin_amdgcn_rcpf(scale) : 0.0f) {}
  __device__ __forceinline__ float operator()(float v) const {
    const float x = v * r;
    return __builtin_fmaf(__builtin_fmaf(-s, x, v), r, x);
  }
};

// Values of one unit group: lanes hold 8 dimensions each, in pieces of 64.
template <int D, int KV>
__device__ void append_values(RowsIn v, const BatchArgs& b, const KvArgs& c, int n_pos, int slot, int piece,
                              u32x4* lds) {
  constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  constexpr int U = KV == MC_KV_BF16 ? 8 : 16, kBlockBytes = KvFormat<D, KV>::kBlockBytes;
  const int lane = threadIdx.x & 63, chunk = piece * 64 + lane;
  const int s = find_sequence(b.q_start, b.S, slot, U, 2, 1);
  const long long first = b.q_start[s], n = (long long)b.q_start[s + 1] - first;
  const long long group = slot - (first / U + 2ll * s);
  if (first < 0 || n <= 0 || group < 0) return;
  const long long p0 = (long long)b.kv_len[s] - n;
  const long long base = ((p0 > 0 ? p0 : 0) / U + group) * U;      // the group's first position
  const long long lo = base > p0 ? base : p0, hi = base + U < p0 + n ? base + U : p0 + n;
  Place at;
  // a group lies in one block: its first token's page is every token's
  if (lo >= hi || !append_place(c, b, s, lo, n_pos, at)) return;
  long long end = kv_length(c, b, s);
  if (end > n_pos) end = n_pos;
  const int chunks = c.Hkv * (D / 8);
  const bool mine = chunk < chunks;
  const int head = mine ? chunk / (D / 8) : 0, d0 = 8 * (chunk % (D / 8));
  u32x4 raw[U];
  bool all = true;                               // the same for the whole wave
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long pos = base + u, row = first + pos - p0;
    const bool in = pos >= lo && pos < hi && pos < end && row >= 0 && row < b.T;
    raw[u] = u32x4{0u, 0u, 0u, 0u};
    if (in && mine) raw[u] = *reinterpret_cast<const u32x4*>(v.p + (size_t)row * v.stride + 8 * chunk);
    all = all && in;
  }
  const int in_block = (int)(base & 15);
  auto unit_of = [&](int h) {                    // the group's first unit of head h
    return c.v + kv_block_offset<kBlockBytes>(c, at.page, h, at.pos >> 4) + (size_t)(in_block / U) * D * 16;
  };
  if constexpr (E2) {
    // lane: dimensions d0 .. d0 + 7, halves of 8 units; 64 dimensions in 8 neighbouring lanes
    uint32_t live = 0;
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const long long pos = base + u, row = first + pos - p0;
      live |= pos >= lo && pos < hi && pos < end && row >= 0 && row < b.T ? 1u << u : 0u;
    }
    live = __builtin_amdgcn_readfirstlane(live);
    const int blk = at.pos >> 4, unit = d0 / 32 * 256 + (d0 & 15) * 16 + (d0 / 16 & 1) * 8;
    char* codes = c.v + kv_block_offset<kBlockBytes>(c, at.page, head, blk);
    u32x2 w[8];                                  // the other tokens' codes of the bytes
    if (!all && mine) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const u32x2*>(codes + unit + 16 * i);
    }
    // a token's eight codes in a word; tokens that are not among the new ones are passed by (one token: 16
    // tests and one of these)
    uint32_t code[16] = {}, sw[8] = {};
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      if (!((live >> u) & 1u)) continue;
      float x[8], m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = half_of(raw[u][i / 2], i & 1);
        m = magnitude(x[i], m);
      }
      m = magnitude(m, dpp<0xb1>(m));
      m = magnitude(m, dpp<0x4e>(m));
      m = magnitude(m, dpp<0x141>(m));
      const float s = value_scale(m);
      sw[u / 2] |= (__float_as_uint(s) >> 16) << (16 * (u & 1));
      const Divisor by(s);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s > 0.0f ? by(x[i]) : 0.0f;
      code[u] = e2m1_word(x);
    }
    // words of a dimension's tokens
    u32x2 t[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint32_t a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = code[8 * q + i];
      transpose_nibbles(a);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i][q] = a[i];
    }
    if ((lane & 7) == 0 && mine) {
      uint16_t* scales = reinterpret_cast<uint16_t*>(c.v + kv_scale_offset<D>(c, at.page, head, blk)) + d0 / 64 * 16;
      if (all) {
        *reinterpret_cast<u32x4*>(scales) = u32x4{sw[0], sw[1], sw[2], sw[3]};
        *reinterpret_cast<u32x4*>(scales + 8) = u32x4{sw[4], sw[5], sw[6], sw[7]};
      } else {
#pragma unroll
        for (int u = 0; u < 16; ++u)
          if ((live >> u) & 1u) scales[u] = (uint16_t)(sw[u / 2] >> (16 * (u & 1)));
      }
    }
    if (!all) {
      if (!mine) return;
      uint32_t keep[2] = {0u, 0u};
#pragma unroll
      for (int u = 0; u < 16; ++u) keep[u / 8] |= (live >> u) & 1u ? 0u : 0xfu << (4 * (u & 7));
      // (codes of other tokens are written back as they were: nobody else writes this block's values)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<u32x2*>(codes + unit + 16 * i) =
            u32x2{(t[i][0] & ~keep[0]) | (w[i][0] & keep[0]), (t[i][1] & ~keep[1]) | (w[i][1] & keep[1])};
      return;
    }
    // whole units, 64 side by side, by way of LDS, where unit n of 16 lies at n ^ (its row) so that the halves
    // that a wave writes at once meet different banks
    char* half = reinterpret_cast<char*>(lds);
    const int row = 8 * lane / 32;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      *reinterpret_cast<u32x2*>(half + row * 256 + ((((8 * lane) & 15) + i) ^ (row & 15)) * 16 + (lane >> 1 & 1) * 8) =
          t[i];
    asm volatile("" ::: "memory");               // the wave's own: its LDS accesses are in order
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int u = 64 * k + lane, ch = piece * 64 + 4 * (u >> 4);        // the unit's first chunk
      const u32x4 v16 = *reinterpret_cast<const u32x4*>(half + (u >> 4) * 256 + ((u & 15) ^ (u >> 4 & 15)) * 16);
      if (ch >= chunks) continue;
      const int h = ch / (D / 8), j = ch % (D / 8) / 4;
      *reinterpret_cast<u32x4*>(c.v + kv_block_offset<kBlockBytes>(c, at.page, h, blk) + j * 256 + (u & 15) * 16) = v16;
    }
    return;
  }
  const float sc = E4 ? 1.0f / c.v_scale[head] : 1.0f;
  if (all) {
    // The lane's 8 units lie side by side.  They go out 64 side by side at a time, by
    // way of LDS: stores of a lane's own units touch 64 lines each for 16 bytes.  The
    // places in LDS are turned by the lane so that neither side meets a bank twice.
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u32x4 w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (E4) {
          w[q] = e4m3_quad(half_of(raw[4 * q][i / 2], i & 1) * sc, half_of(raw[4 * q + 1][i / 2], i & 1) * sc,
                           half_of(raw[4 * q + 2][i / 2], i & 1) * sc, half_of(raw[4 * q + 3][i / 2], i & 1) * sc);
        } else {
          const uint32_t a = raw[2 * q][i / 2], z = raw[2 * q + 1][i / 2];
          w[q] = (i & 1) ? (a >> 16) | (z & 0xffff0000u) : (a & 0xffffu) | (z << 16);
        }
      }
      lds[8 * lane + (i ^ (lane & 7))] = w;
    }
    asm volatile("" ::: "memory");               // the wave's own: its LDS accesses are in order
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int u = 64 * k + lane, l = u >> 3, ch = piece * 64 + l;
      const u32x4 w = lds[8 * l + ((u & 7) ^ (l & 7))];
      if (ch < chunks)
        *reinterpret_cast<u32x4*>(unit_of(ch / (D / 8)) + 16 * (8 * (ch % (D / 8)) + (u & 7))) = w;
    }
    return;
  }
  if (!mine) return;
  char* dst = unit_of(head) + 16 * d0;
  // a unit that other tokens share: element by element
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long pos = base + u, row = first + pos - p0;
    if (!(pos >= lo && pos < hi && pos < end && row >= 0 && row < b.T)) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (E4)
        dst[16 * i + u] = (char)e4m3_quad(half_of(raw[u][i / 2], i & 1) * sc, 0.0f, 0.0f, 0.0f);
      else
        reinterpret_cast<uint16_t*>(dst + 16 * i)[u] = (uint16_t)(raw[u][i / 2] >> (16 * (i & 1)));
    }
  }
}

__device__ __forceinline__ float square_sum(const u32x4& r) {
  float s = 0.0f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float a = half_of(r[q], 0), z = half_of(r[q], 1);
    s = __builtin_fmaf(a, a, s);
    s = __builtin_fmaf(z, z, s);
  }
  return s;
}

// The sum over the D/8 lanes of a head.
template <int DU>
__device__ __forceinline__ float head_sum(float x) {
  x += dpp<0xb1>(x);
  x += dpp<0x4e>(x);
  x += dpp<0x141>(x);
  if (DU == 16) x += dpp<0x140>(x);
  return x;
}

__device__ __forceinline__ double square_sum64(const u32x4& r) {
  double s = 0.0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const double a = half_of(r[q], 0), z = half_of(r[q], 1);
    s = __builtin_fma(a, a, s);
    s = __builtin_fma(z, z, s);
  }
  return s;
}

template <int DU>
__device__ __forceinline__ double head_sum64(double x) {
  x += dpp64<0xb1>(x);
  x += dpp64<0x4e>(x);
  x += dpp64<0x141>(x);
  if (DU == 16) x += dpp64<0x140>(x);
  return x;
}

__device__ __forceinline__ double wave_sum64(double x) {
  x = head_sum64<16>(x);
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Queries and keys of one token: chunk i of 8 elements in [0, nq + nk), the queries'
// first, 64 neighbouring ones at a time.  A head's chunks lie in D/8 neighbouring
// lanes, and a lane's chunks all start at the same dimension of their heads, so that
// its cosines and sines are loaded once.  A norm over the row needs one wave for the
// token; without it a wave takes one of its parts of 64 kRowChunks chunks: shorter waves
// overlap their loads, arithmetic and stores better.
template <int D, int KV, int NORM>
__device__ void append_rows(RowsIn q, RowsIn k, int Hq, const QkPrepArgs& p, const BatchArgs& b, const KvArgs& c,
                            RowsOut out, int t, int part) {
  constexpr int kRowChunks = row_chunks(NORM);
  constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  constexpr int DU = D / 8, kBlockBytes = KvFormat<D, KV>::kBlockBytes;
  const int lane = threadIdx.x & 63;
  const int nq = q.p ? Hq * DU : 0, total = nq + c.Hkv * DU;
  const uint16_t* qr = q.p + (size_t)t * q.stride;
  const uint16_t* kr = k.p + (size_t)t * k.stride;
  u32x4 raw[kRowChunks];
  auto load = [&](int i0) {
#pragma unroll
    for (int r = 0; r < kRowChunks; ++r) {
      const int i = i0 + 64 * r + lane;
      raw[r] = u32x4{0u, 0u, 0u, 0u};
      if (i < total) raw[r] = *reinterpret_cast<const u32x4*>(i < nq ? qr + 8 * i : kr + 8 * (i - nq));
    }
  };
  load(64 * kRowChunks * part);

  const int s = find_sequence(b.q_start, b.S, t, 1, 0, 1);
  const long long first = b.q_start[s], last = b.q_start[s + 1];
  Place at;
  if (!(t >= first && t < last && append_place(c, b, s, (long long)b.kv_len[s] - (last - t), p.n_pos, at))) return;

  const int d0 = 8 * (lane % DU), half = p.rot / 2;
  const bool turns = d0 < p.rot, low = d0 < half;
  f32x4 tab[4];
  if (turns) {
    // rotation i's cosine and sine: i = d0/2 .. +3, or d0 mod half .. +7
    const float* from = p.rope + (size_t)at.pos * p.rot + (p.pairs ? d0 : 2 * (low ? d0 : d0 - half));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < 2 || !p.pairs) tab[i] = *reinterpret_cast<const f32x4*>(from + 4 * i);
    if (low && !p.pairs) {                       // y_a cos - y_b sin, y_b cos + y_a sin
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        tab[i][1] = -tab[i][1];
        tab[i][3] = -tab[i][3];
      }
    }
  }
  const int partner = turns ? lane + (low ? half / 8 : -(half / 8)) : lane;

  u32x4 wq = {}, wk = {};
  if (NORM == 1) {
    wq = *reinterpret_cast<const u32x4*>(p.q_norm + d0);
    wk = *reinterpret_cast<const u32x4*>(p.k_norm + d0);
  }
  float row_scale[2] = {1.0f, 1.0f};
  double key_scale = 1.0;
  if (NORM == 2) {
    float ss[2] = {0.0f, 0.0f};
    double sk = 0.0;
    for (int i0 = 0; i0 < total; i0 += 64 * kRowChunks) {
      if (i0) load(i0);
#pragma unroll
      for (int r = 0; r < kRowChunks; ++r) {
        const float x = square_sum(raw[r]);
        const bool is_q = i0 + 64 * r + lane < nq;
        ss[0] += is_q ? x : 0.0f;
        ss[1] += is_q ? 0.0f : x;
        if (E2) sk += is_q ? 0.0 : square_sum64(raw[r]);
      }
    }
    if (E2) key_scale = 1.0 / sqrt(wave_sum64(sk) / (double)(c.Hkv * D) + (double)p.eps);
    if (total > 64 * kRowChunks) load(0);
#pragma unroll
    for (int w = 0; w < 2; ++w)
      row_scale[w] = __builtin_amdgcn_rsqf(halves_sum(half_wave_sum(ss[w])) / (float)((w == 0 ? Hq : c.Hkv) * D) +
                                           p.eps);
  }

  const int begin = NORM == 2 ? 0 : 64 * kRowChunks * part, end = NORM == 2 ? total : begin + 64 * kRowChunks;
  for (int i0 = begin; i0 < end; i0 += 64 * kRowChunks) {
    if (i0 != begin) load(i0);
#pragma unroll
    for (int r = 0; r < kRowChunks; ++r) {
      if (i0 + 64 * r >= total) break;           // the same for the whole wave
      const int i = i0 + 64 * r + lane;
      const bool is_q = i < nq;
      if constexpr (E2) {
        // keys in 64 bits, whose rounding next to a border of the codes does not count (the lanes of
        // a head are all keys or all queries)
        if (i0 + 64 * r + 63 >= nq) {
          double y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = (double)half_of(raw[r][j / 2], j & 1);
          if (NORM) {
            const double sc =
                NORM == 2 ? key_scale : 1.0 / sqrt(head_sum64<DU>(square_sum64(raw[r])) * (1.0 / D) + (double)p.eps);
            u32x4 w = wk;
            if (NORM == 2 && i < total && !is_q) w = *reinterpret_cast<const u32x4*>(p.k_norm + 8 * (i - nq));
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = y[j] * (double)half_of(w[j / 2], j & 1) * sc;
          }
          if (p.rot && p.pairs) {
            if (turns) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const double co = tab[j / 2][2 * (j & 1)], si = tab[j / 2][2 * (j & 1) + 1];
                const double a = y[2 * j], z = y[2 * j + 1];
                y[2 * j] = __builtin_fma(-z, si, a * co);
                y[2 * j + 1] = __builtin_fma(z, co, a * si);
              }
            }
          } else if (p.rot) {
            double o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = p.rot == 128 ? dpp64<0x128>(y[j]) : __shfl(y[j], partner);
            if (turns) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                y[j] = __builtin_fma(o[j], (double)tab[j / 2][2 * (j & 1) + 1], y[j] * (double)tab[j / 2][2 * (j & 1)]);
            }
          }
          float f[8], m = 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[j] = sticky_float(y[j]);
            m = fmaxf(m, fabsf(f[j]));
          }
          m = fmaxf(m, dpp<0xb1>(m));
          m = fmaxf(m, dpp<0x4e>(m));                    // of the lanes of 32 dimensions
          const uint32_t byte = key_scale_byte(m);
          if (i < total && !is_q) {
            // 2^(127 - byte), the products are exact, or far below the first border
            const bool number = byte != 0u && byte != 255u;
            const float by = number ? __uint_as_float((254u - byte) << 23) : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = number ? f[j] * by : 0.0f;
            const int head = (i - nq) / DU, t16 = at.pos & 15;
            char* dst = c.k + kv_block_offset<kBlockBytes>(c, at.page, head, at.pos >> 4);
            *reinterpret_cast<uint32_t*>(dst + d0 / 32 * 256 + t16 * 16 + (d0 / 8 & 3) * 4) = e2m1_word(f);
            if ((lane & 3) == 0)
              c.k[kv_scale_offset<D>(c, at.page, head, at.pos >> 4) + d0 / 32 * 16 + 4 * (t16 & 3) + (t16 >> 2)] =
                  (char)byte;
          }
        }
        if (i0 + 64 * r >= nq) continue;               // no queries among them
      }
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = half_of(raw[r][j / 2], j & 1);
      if (NORM) {
        const float sc = NORM == 2 ? row_scale[is_q ? 0 : 1]
                                   : __builtin_amdgcn_rsqf(head_sum<DU>(square_sum(raw[r])) * (1.0f / D) + p.eps);
        u32x4 w = is_q ? wq : wk;
        if (NORM == 2 && i < total)
          w = *reinterpret_cast<const u32x4*>(is_q ? p.q_norm + 8 * i : p.k_norm + 8 * (i - nq));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * sc * half_of(w[j / 2], j & 1);
      }
      if (p.rot && p.pairs) {
        if (turns) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float co = tab[j / 2][2 * (j & 1)], si = tab[j / 2][2 * (j & 1) + 1];
            const float a = x[2 * j], z = x[2 * j + 1];
            x[2 * j] = __builtin_fmaf(-z, si, a * co);
            x[2 * j + 1] = __builtin_fmaf(z, co, a * si);
          }
        }
      } else if (p.rot) {
        float o[8];
        if (p.rot == 128) {                      // the partner is 8 lanes on in the row of 16
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = dpp<0x128>(x[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = __shfl(x[j], partner);
        }
        if (turns) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float co = tab[j / 2][2 * (j & 1)], si = tab[j / 2][2 * (j & 1) + 1];
            x[j] = __builtin_fmaf(o[j], si, x[j] * co);
          }
        }
      }
      if (i >= total) continue;
      if (is_q) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
        *reinterpret_cast<u32x4*>(out.p + (size_t)t * out.stride + 8 * i) = w;
      } else if constexpr (!E2) {
        const int head = (i - nq) / DU;
        char* dst = c.k + kv_block_offset<kBlockBytes>(c, at.page, head, at.pos >> 4) + (at.pos & 15) * 16;
        if constexpr (E4) {
          const float sc = 1.0f / c.k_scale[head];
          u32x2 w = {e4m3_quad(x[0] * sc, x[1] * sc, x[2] * sc, x[3] * sc),
                     e4m3_quad(x[4] * sc, x[5] * sc, x[6] * sc, x[7] * sc)};
          *reinterpret_cast<u32x2*>(dst + (d0 / 16) * 256 + (d0 & 8)) = w;
        } else {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
          *reinterpret_cast<u32x4*>(dst + (d0 / 8) * 256) = w;
        }
      }
    }
  }
}

// The first nv workgroups write values (4 waves, each a unit group's piece),
// the others queries and keys, 4 neighbouring tokens each, a part of theirs.  Eight
// neighbouring tokens share the lines of the key blocks, and workgroups go round the 8
// XCDs in turn: of 16 row workgroups of a part, number r and r + 8 take 8 neighbouring
// tokens, so that one XCD's cache sees whole lines.
template <int D, int KV, int NORM>
__global__ void __launch_bounds__(kAppendThreads)
    kv_append_kernel(RowsIn q, RowsIn k, RowsIn v, int Hq, QkPrepArgs p, BatchArgs b, KvArgs c, RowsOut out, int nv,
                     int slots, int pieces, int parts) {
  constexpr int kUnits = KV == MC_KV_E2M1 ? 4 : 8;
  __shared__ u32x4 s_units[kAppendThreads * kUnits];
  const int blk = blockIdx.x;
  if (blk < nv) {
    const int w = blk * (kAppendThreads / 64) + wave_id();
    if (w < slots * pieces)
      append_values<D, KV>(v, b, c, p.n_pos, w / pieces, w % pieces, s_units + wave_id() * 64 * kUnits);
    return;
  }
  const int r0 = blk - nv, group = r0 / (16 * parts), in = r0 - group * 16 * parts, r = in & 15;
  const int t = 4 * (16 * group + 2 * (r & 7) + (r >> 3)) + wave_id();
  if (t < b.T) append_rows<D, KV, NORM>(q, k, Hq, p, b, c, out, t, in >> 4);
}

template <int D, int KV>
static void append_launch(RowsIn q, RowsIn k, RowsIn v, int Hq, const QkPrepArgs& p, const BatchArgs& b,
                          const KvArgs& c, RowsOut out, hipStream_t stream) {
  const int pieces = (c.Hkv * (D / 8) + 63) / 64, slots = append_slots(b.T, b.S, KV == MC_KV_BF16 ? 8 : 16);
  const int per = kAppendThreads / 64, nv = (slots * pieces + per - 1) / per;
  const int chunks = ((q.p ? Hq : 0) + c.Hkv) * (D / 8);
  auto launch = [&](auto kernel, int parts) {
    hipLaunchKernelGGL(kernel, dim3(nv + (b.T + 63) / 64 * 16 * parts), dim3(kAppendThreads), 0, stream, q, k, v, Hq, p,
                       b, c, out, nv, slots, pieces, parts);
  };
  const int each = 64 * row_chunks(0);
  if (!p.q_norm)
    launch(kv_append_kernel<D, KV, 0>, (chunks + each - 1) / each);
  else if (!p.norm_row)
    launch(kv_append_kernel<D, KV, 1>, (chunks + each - 1) / each);
  else
    launch(kv_append_kernel<D, KV, 2>, 1);
}

hipError_t launch_kv_append(RowsIn q, RowsIn k, RowsIn v, int Hq, int D, const QkPrepArgs& p, const BatchArgs& b,
                            const KvArgs& c, RowsOut out, hipStream_t stream) {
  timing_begin(stream, kSiteKvAppend);
  with_kv_kind(c, [&](auto kind) {
    constexpr int KV = decltype(kind)::value;
    D == 64 ? append_launch<64, KV>(q, k, v, Hq, p, b, c, out, stream)
            : append_launch<128, KV>(q, k, v, Hq, p, b, c, out, stream);
  });
  timing_end(stream, kSiteKvAppend);
  return hipGetLastError();
}

// ------------------------------------------------------------------- read --
// What the cache holds at the new tokens' places: a wave takes one head of a block of 16 tokens.  Keys'
// units are pieces of rows; values' units, which run along the tokens, become rows in LDS.
template <int D, int KV>
__global__ void __launch_bounds__(kAppendThreads)
    kv_read_kernel(BatchArgs b, KvArgs c, RowsOut ko, RowsOut vo, int slots) {
  constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  constexpr int kBlockBytes = KvFormat<D, KV>::kBlockBytes, kUnits = kBlockBytes / 16, kRow = D + 8;
  __shared__ __attribute__((aligned(16))) uint16_t s_rows[kAppendThreads / 64][16][kRow];
  const int lane = threadIdx.x & 63, id = blockIdx.x * (kAppendThreads / 64) + wave_id();
  const int head = id % c.Hkv, slot = id / c.Hkv;
  if (slot >= slots) return;
  const int s = find_sequence(b.q_start, b.S, slot, 16, 2, 1);
  const long long first = b.q_start[s], n = (long long)b.q_start[s + 1] - first;
  const long long group = slot - (first / 16 + 2ll * s);
  if (n <= 0 || group < 0) return;
  const long long p0 = (long long)b.kv_len[s] - n, base = ((p0 > 0 ? p0 : 0) / 16 + group) * 16;
  long long hi = kv_length(c, b, s);
  if (p0 + n < hi) hi = p0 + n;
  Place at;
  if (!append_place(c, b, s, base > p0 ? base : p0, 0x7fffffff, at) || base >= hi) return;
  const size_t off = kv_block_offset<kBlockBytes>(c, at.page, head, at.pos >> 4);
  // token t of the block: its row, or -1
  auto row_of = [&](int t) {
    const long long pos = base + t, row = first + pos - p0;
    return pos >= p0 && pos < hi && row >= 0 && row < b.T ? (int)row : -1;
  };
  const char *kp = c.k + off, *vp = c.v + off;
  const size_t so = E2 ? kv_scale_offset<D>(c, at.page, head, at.pos >> 4) : 0;
  const float ks = E4 ? c.k_scale[head] : 1.0f, vs = E4 ? c.v_scale[head] : 1.0f;
  constexpr int U = (kUnits + 63) / 64;
  u32x4 kw[U], vw[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    kw[i] = vw[i] = u32x4{0u, 0u, 0u, 0u};
    if (64 * i + lane < kUnits) {
      if (ko.p) kw[i] = *reinterpret_cast<const u32x4*>(kp + 16 * (64 * i + lane));
      if (vo.p) vw[i] = *reinterpret_cast<const u32x4*>(vp + 16 * (64 * i + lane));
    }
  }
  auto scaled = [](u32x4 x, float f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = bf16_pair(half_of(x[e], 0) * f, half_of(x[e], 1) * f);
    return x;
  };
  if (ko.p) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int x = 64 * i + lane, t = x & 15, row = row_of(t);
      if (x >= kUnits || row < 0) continue;
      uint16_t* out = ko.p + (size_t)row * ko.stride + (size_t)head * D;
      if constexpr (E2) {
        const uint32_t byte = (uint8_t)c.k[so + (x >> 4) * 16 + 4 * (t & 3) + (t >> 2)];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          *reinterpret_cast<u32x4*>(out + 32 * (x >> 4) + 8 * u) = e2m1_to_bf16(kw[i][u], __uint_as_float(byte << 23));
      } else if constexpr (E4) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          *reinterpret_cast<u32x4*>(out + 16 * (x >> 4) + 8 * u) =
              scaled(e4m3_to_bf16(kw[i][2 * u], kw[i][2 * u + 1]), ks);
      } else {
        *reinterpret_cast<u32x4*>(out + 8 * (x >> 4)) = kw[i];
      }
    }
  }
  if (!vo.p) return;
  uint16_t (*rows)[kRow] = s_rows[wave_id()];
  auto put = [&](const u32x4& x, int t0, int d) {       // tokens t0 .. t0 + 7 of dimension d
#pragma unroll
    for (int e = 0; e < 8; ++e) rows[t0 + e][d] = (uint16_t)(x[e / 2] >> (16 * (e & 1)));
  };
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int x = 64 * i + lane;
    if (x >= kUnits) continue;
    if constexpr (E2) {
      const int j = x >> 4;
      const u32x4* sc = reinterpret_cast<const u32x4*>(c.v + so + 32 * (j >> 1));
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const u32x4 sg = sc[g];
#pragma unroll
        for (int h = 0; h < 2; ++h) put(e2m1_times(vw[i][2 * h + g], sg), 8 * g, 32 * j + 16 * h + (x & 15));
      }
    } else if constexpr (E4) {
#pragma unroll
      for (int g = 0; g < 2; ++g) put(scaled(e4m3_to_bf16(vw[i][2 * g], vw[i][2 * g + 1]), vs), 8 * g, x);
    } else {
      put(vw[i], 8 * (x / D), x % D);
    }
  }
  asm volatile("" ::: "memory");                 // the wave's own: its LDS accesses are in order
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int x = 64 * i + lane, t = x / (D / 8), d = 8 * (x % (D / 8)), row = row_of(t);
    if (row >= 0)
      *reinterpret_cast<u32x4*>(vo.p + (size_t)row * vo.stride + (size_t)head * D + d) =
          *reinterpret_cast<const u32x4*>(&rows[t][d]);
  }
}

hipError_t launch_kv_read(int D, const BatchArgs& b, const KvArgs& c, RowsOut k, RowsOut v, hipStream_t stream) {
  const int slots = append_slots(b.T, b.S, 16), per = kAppendThreads / 64;
  const dim3 grid((unsigned)(((size_t)slots * c.Hkv + per - 1) / per));
  timing_begin(stream, kSiteKvRead);
  with_kv_kind(c, [&](auto kind) {
    constexpr int KV = decltype(kind)::value;
    if (D == 64)
      hipLaunchKernelGGL((kv_read_kernel<64, KV>), grid, dim3(kAppendThreads), 0, stream, b, c, k, v, slots);
    else
      hipLaunchKernelGGL((kv_read_kernel<128, KV>), grid, dim3(kAppendThreads), 0, stream, b, c, k, v, slots);
  });
  timing_end(stream, kSiteKvRead);
  return hipGetLastError();
}

}  // namespace mc
