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
// 4.5 us, a chain of four memory latencies.
#include "attn.hpp"

namespace mc {

constexpr int kAppendThreads = 256;
// Chunks of 8 elements that a lane holds at once.
__host__ __device__ constexpr int row_chunks(int norm) { return norm == 2 ? 8 : 4; }

// The largest number of unit groups that n new tokens from q_start on touch is
// floor((n + 6) / U) + 1 (U = 8) and fewer for U = 16; sequence s owns the slots from
// floor(q_start[s] / U) + 2 s on, at least floor(n / U) + 2 of them.
__host__ __device__ static inline int append_slots(int T, int S, int U) { return T / U + 2 * S; }

__device__ __forceinline__ float half_of(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xffff0000u : w << 16); }

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

// Values of one unit group: lanes hold 8 dimensions each, in pieces of 64.
template <int D, bool E4>
__device__ void append_values(RowsIn v, const BatchArgs& b, const KvArgs& c, int n_pos, int slot, int piece,
                              u32x4* lds) {
  constexpr int U = E4 ? 16 : 8, kBlockBytes = kKvBlock * D * (E4 ? 1 : 2);
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

// Queries and keys of one token: chunk i of 8 elements in [0, nq + nk), the queries'
// first, 64 neighbouring ones at a time.  A head's chunks lie in D/8 neighbouring
// lanes, and a lane's chunks all start at the same dimension of their heads, so that
// its cosines and sines are loaded once.  A norm over the row needs one wave for the
// token; without it a wave takes one of its parts of 64 kRowChunks chunks: shorter waves
// overlap their loads, arithmetic and stores better.
template <int D, bool E4, int NORM>
__device__ void append_rows(RowsIn q, RowsIn k, int Hq, const QkPrepArgs& p, const BatchArgs& b, const KvArgs& c,
                            RowsOut out, int t, int part) {
  constexpr int kRowChunks = row_chunks(NORM);
  constexpr int DU = D / 8, kBlockBytes = kKvBlock * D * (E4 ? 1 : 2);
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
  if (NORM == 2) {
    float ss[2] = {0.0f, 0.0f};
    for (int i0 = 0; i0 < total; i0 += 64 * kRowChunks) {
      if (i0) load(i0);
#pragma unroll
      for (int r = 0; r < kRowChunks; ++r) {
        const float x = square_sum(raw[r]);
        const bool is_q = i0 + 64 * r + lane < nq;
        ss[0] += is_q ? x : 0.0f;
        ss[1] += is_q ? 0.0f : x;
      }
    }
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
      } else {
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
template <int D, bool E4, int NORM>
__global__ void __launch_bounds__(kAppendThreads)
    kv_append_kernel(RowsIn q, RowsIn k, RowsIn v, int Hq, QkPrepArgs p, BatchArgs b, KvArgs c, RowsOut out, int nv,
                     int slots, int pieces, int parts) {
  __shared__ u32x4 s_units[kAppendThreads * 8];
  const int blk = blockIdx.x;
  if (blk < nv) {
    const int w = blk * (kAppendThreads / 64) + wave_id();
    if (w < slots * pieces)
      append_values<D, E4>(v, b, c, p.n_pos, w / pieces, w % pieces, s_units + wave_id() * 512);
    return;
  }
  const int r0 = blk - nv, group = r0 / (16 * parts), in = r0 - group * 16 * parts, r = in & 15;
  const int t = 4 * (16 * group + 2 * (r & 7) + (r >> 3)) + wave_id();
  if (t < b.T) append_rows<D, E4, NORM>(q, k, Hq, p, b, c, out, t, in >> 4);
}

template <int D, bool E4>
static void append_launch(RowsIn q, RowsIn k, RowsIn v, int Hq, const QkPrepArgs& p, const BatchArgs& b,
                          const KvArgs& c, RowsOut out, hipStream_t stream) {
  const int pieces = (c.Hkv * (D / 8) + 63) / 64, slots = append_slots(b.T, b.S, E4 ? 16 : 8);
  const int per = kAppendThreads / 64, nv = (slots * pieces + per - 1) / per;
  const int chunks = ((q.p ? Hq : 0) + c.Hkv) * (D / 8);
  auto launch = [&](auto kernel, int parts) {
    hipLaunchKernelGGL(kernel, dim3(nv + (b.T + 63) / 64 * 16 * parts), dim3(kAppendThreads), 0, stream, q, k, v, Hq, p,
                       b, c, out, nv, slots, pieces, parts);
  };
  const int each = 64 * row_chunks(0);
  if (!p.q_norm)
    launch(kv_append_kernel<D, E4, 0>, (chunks + each - 1) / each);
  else if (!p.norm_row)
    launch(kv_append_kernel<D, E4, 1>, (chunks + each - 1) / each);
  else
    launch(kv_append_kernel<D, E4, 2>, 1);
}

hipError_t launch_kv_append(RowsIn q, RowsIn k, RowsIn v, int Hq, int D, const QkPrepArgs& p, const BatchArgs& b,
                            const KvArgs& c, RowsOut out, hipStream_t stream) {
  timing_begin(stream, kSiteKvAppend);
  const bool e4 = c.k_scale != nullptr;
  if (D == 64)
    e4 ? append_launch<64, true>(q, k, v, Hq, p, b, c, out, stream)
       : append_launch<64, false>(q, k, v, Hq, p, b, c, out, stream);
  else
    e4 ? append_launch<128, true>(q, k, v, Hq, p, b, c, out, stream)
       : append_launch<128, false>(q, k, v, Hq, p, b, c, out, stream);
  timing_end(stream, kSiteKvAppend);
  return hipGetLastError();
}

}  // namespace mc
