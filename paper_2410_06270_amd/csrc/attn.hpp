// attn.hpp -- the paged cache as the attention kernels see it: launch
// arguments, address arithmetic, visibility and number formats.
#pragma once

#include <type_traits>

#include "mc_internal.hpp"

namespace mc {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();
constexpr int kKvBlock = 16;         // tokens of a cache block

struct KvArgs {
  char *k, *v;
  size_t page_stride;                // bytes
  int n_pages, Hkv, lb;              // lb: log2 of the blocks in a page
  const float *k_scale, *v_scale;    // e4m3 only
  int kind;                          // MC_KV_*
};

// How a kind of cache holds its elements: bytes of a block's codes, tokens (of values) or
// dimensions (of keys) that 16 bytes hold.  e2m1 has scales behind a page's codes.
template <int D, int KV>
struct KvFormat {
  static constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  static constexpr int kBlockBytes = E2 ? 8 * D : kKvBlock * D * (E4 ? 1 : 2);
  static constexpr int kScaleBytes = E2 ? D / 2 : 0;       // of a block
};

// Calls f(integral constant of the cache's kind).
template <class F>
void with_kv_kind(const KvArgs& c, F&& f) {
  if (c.kind == MC_KV_E2M1)
    f(std::integral_constant<int, MC_KV_E2M1>{});
  else if (c.kind == MC_KV_E4M3)
    f(std::integral_constant<int, MC_KV_E4M3>{});
  else
    f(std::integral_constant<int, MC_KV_BF16>{});
}

struct BatchArgs {
  const int32_t *q_start, *kv_len, *page_table;
  int S, T, max_pages;
};

struct ScoreArgs {
  int Hq, g;                         // g = Hq / Hkv
  float scale, softcap;
  int window;
  const float* slopes;
  const int32_t* prefix;
};

// Partial results of a split: o [row][Hq][nsplit][D] (unnormalised, relative to
// the part's own maximum), ml [row][Hq][nsplit][2] (maximum in the log2
// domain, sum), row a row of the outputs.
struct SplitArgs {
  float *o, *ml;
  int nsplit;
};

// Bounds of the pages' keys: bounds [n_pages][Hkv][2][D] (least, largest) in units of scale
// [n_pages][Hkv].
struct SummaryArgs {
  int8_t* bounds;
  float* scale;
};

struct SelectArgs {
  int g, negative, window;           // negative: a negative scale turns the order
  int n_sel, first, last;            // pages of a row; the first and last ones that are always taken
  int32_t *sel, *count;
};

struct PoolArgs {
  int32_t* free_list;
  const int32_t* n_free;
  int32_t* n_free_out;
  int n_pages, page_log;
};

struct BatchOut {
  int32_t *q_start, *kv_len, *page_table;
  int S, T, max_pages;
};

// The longest length the tables describe, and a sequence's length within it.
__device__ __forceinline__ int kv_length(const KvArgs& c, const BatchArgs& b, int s) {
  const int most = (b.max_pages << c.lb) * kKvBlock, n = b.kv_len[s];      // most: 2^30 or less
  return n < 0 ? 0 : n > most ? most : n;
}

__device__ __forceinline__ int kv_prefix(const ScoreArgs& a, int s, int len) {
  if (!a.prefix) return 0;
  const int p = a.prefix[s];
  return p < 0 ? 0 : p > len ? len : p;
}

// A page number of the table, clamped into the cache.
__device__ __forceinline__ int kv_page(const KvArgs& c, int p) {
  return p < 0 ? 0 : p >= c.n_pages ? c.n_pages - 1 : p;
}

// Byte offset of block `blk` (a position / 16) of head h, on page p, the block
// being BYTES long.
template <int BYTES>
__device__ __forceinline__ size_t kv_block_offset(const KvArgs& c, int p, int h, int blk) {
  const int in_page = blk & ((1 << c.lb) - 1);
  return (size_t)p * c.page_stride + (size_t)((h << c.lb) + in_page) * BYTES;
}

// Byte offset of a block's scales (e2m1).
template <int D>
__device__ __forceinline__ size_t kv_scale_offset(const KvArgs& c, int p, int h, int blk) {
  const int in_page = blk & ((1 << c.lb) - 1);
  return (size_t)p * c.page_stride + (size_t)(c.Hkv << c.lb) * (8 * D) + (size_t)((h << c.lb) + in_page) * (D / 2);
}

// The largest s in [0, S) with start[s] * g / div + mul * s <= key (0 if there is
// none; g: rows of a tile that a token takes), found by the whole wave with 64 probes a
// round: one load for up to 64 sequences, two for 4096.  key must be wave-uniform; every s
// it returns is in range whatever the array holds.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ start, int S, int key, int div, int mul,
                                             int g) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = S;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    bool below = lane == 0;
    if (lane > 0 && at < n) {
      const long long first = (long long)start[lo + at] * g;
      below = first / div + (long long)mul * (lo + at) <= key;
    }
    const int last = 63 - __builtin_clzll(__ballot(below));
    lo += last * step;
    n = n - last * step < step ? n - last * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows [first, first + n) of sequence s among the T packed ones.
__device__ __forceinline__ void sequence_rows(const BatchArgs& b, int s, int& first, int& n) {
  int lo = b.q_start[s], hi = b.q_start[s + 1];
  lo = lo < 0 ? 0 : lo > b.T ? b.T : lo;
  hi = hi < lo ? lo : hi > b.T ? b.T : hi;
  first = lo;
  n = hi - lo;
}

// Waits for the wave's LDS accesses, then for the workgroup.  Unlike
// __syncthreads() it leaves direct loads to LDS in flight: their arrival is
// waited for by count (wait_vmcnt) before it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));     // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Waits for the wave's direct loads to LDS; what it reads of them afterwards stays behind the wait
// (which alone the compiler need not keep LDS accesses behind).
__device__ __forceinline__ void loads_landed() {
  asm volatile("" ::: "memory");
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
}

// ----------------------------------------------------------- direct loads --
// 16 or 4 bytes a lane to LDS from a buffer, `bytes` at a wave-uniform address: read at
// OFF (below 4096) plus the lane's own offset and a uniform one, to dst + OFF + 16 l (or dst
// + 4 l), counted by vmcnt.  Global direct loads (lds_dma16 of an address) make the
// compiler wait for every LDS read under way wherever it waits for one; these do not.
typedef __amdgpu_buffer_rsrc_t Buffer;

__device__ __forceinline__ Buffer buffer_of(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

template <int OFF>
__device__ __forceinline__ void lds_dma16(Buffer src, int offset, int uniform, void* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, offset, uniform, OFF,
                                           0);
}

__device__ __forceinline__ void lds_dma4(Buffer src, int offset, void* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 4, offset, 0, 0, 0);
}

// ----------------------------------------------------------------- formats --

__device__ __forceinline__ uint16_t bf16_bits(float f) {     // nearest even, NaN kept
  const __bf16 h = (__bf16)f;
  uint16_t b;
  __builtin_memcpy(&b, &h, 2);
  return b;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const bf16x2 h = {(__bf16)lo, (__bf16)hi};
  uint32_t b;
  __builtin_memcpy(&b, &h, 4);
  return b;
}

__device__ __forceinline__ bf16x8 as_bf16x8(const u32x4& v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}

// Eight e4m3 codes (two words) as bf16: exact, bf16 holds every e4m3 value.
__device__ __forceinline__ u32x4 e4m3_to_bf16(uint32_t a, uint32_t b) {
  bf16x2 t[4];
  t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  u32x4 r;
  __builtin_memcpy(&r, t, 16);
  return r;
}

// Eight e2m1 codes (a word, the first in the lowest bits) times 2^(byte - 127), as bf16: exact, but
// for results below 2^-126.  (The instruction takes its factor's exponent; 255 gives NaN.)
__device__ __forceinline__ u32x4 e2m1_to_bf16(uint32_t w, float scale) {
  bf16x2 t[4];
  t[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  t[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  t[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  t[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  u32x4 r;
  __builtin_memcpy(&r, t, 16);
  return r;
}

// Eight e2m1 codes of a dimension's neighbouring tokens times their scales (bf16, of 6 significant bits):
// the products are bf16 numbers, the upper halves of the floats.
__device__ __forceinline__ u32x4 e2m1_times(uint32_t w, const u32x4& scales) {
  typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
  f32x2 t[4];
  t[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
  t[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
  t[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
  t[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = t[i][0] * __uint_as_float(scales[i] << 16), hi = t[i][1] * __uint_as_float(scales[i] & 0xffff0000u);
    r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
  }
  return r;
}

// 2^(byte - 127) for byte `at` of w.
__device__ __forceinline__ float e8m0_scale(uint32_t w, int at) {
  return __uint_as_float(((w >> (8 * at)) & 0xffu) << 23);
}

// The value of an e2m1 code, and bf16 halves of a word as floats.
__device__ __forceinline__ float e2m1_value(uint32_t code) {
  const float m = (code & 6u) ? __uint_as_float(((126u + ((code >> 1) & 3u)) << 23) | ((code & 1u) << 22))
                              : 0.5f * (float)(code & 1u);
  return code & 8u ? -m : m;
}
__device__ __forceinline__ float half_of(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xffff0000u : w << 16); }

// Four e4m3 codes: nearest, ties to even, clamped to +-448 (the comparison
// leaves a NaN as it is, and NaN converts to NaN).
__device__ __forceinline__ float e4m3_clamp(float f) { return f > 448.0f ? 448.0f : f < -448.0f ? -448.0f : f; }

__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a), e4m3_clamp(b), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c), e4m3_clamp(d), r, true);
  return (uint32_t)r;
}

// ---------------------------------------------------------- between lanes --
// The larger, and the sum, of x in lanes l and l ^ 32 (half waves) or l ^ 16 (their rows).
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float rows_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// x of the lane that the DPP control names, within the row of 16.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// The sum over the lane's half wave: neighbours, pairs of a quad, quads of 8
// (mirrored), eights of a row (mirrored), the two rows.
__device__ __forceinline__ float half_wave_sum(float x) {
  x += dpp<0xb1>(x);
  x += dpp<0x4e>(x);
  x += dpp<0x141>(x);
  x += dpp<0x140>(x);
  return rows_sum(x);
}

// The inclusive sum over the wave's lanes: within rows of 16, then the rows before.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) {
  return x + (int)__builtin_amdgcn_update_dpp(0u, (uint32_t)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
}

// The largest over the wave's lanes, and the sum.
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0xb1>(x));
  x = fmaxf(x, dpp<0x4e>(x));
  x = fmaxf(x, dpp<0x141>(x));
  x = fmaxf(x, dpp<0x140>(x));
  return halves_max(rows_max(x));
}
__device__ __forceinline__ float wave_sum(float x) { return halves_sum(half_wave_sum(x)); }

// ------------------------------------------------------------------ scores --

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A score in the log2 domain from the plain product q.k.  cap tanh(x / cap) =
// cap - 2 cap u with u = 1 / (1 + exp(2 x / cap)), off by some 2^-23 cap whatever the
// score: up to kCapPlain 2^-17, a weight's rounding to bf16 is 2^-8.  Larger caps, and rows of few keys
// (edge_mode), keep the error relative, the tanh being x / cap (1 - z/3 + 2 z^2/15 - 17 z^3/315 + 62 z^4/2835), z
// = (x / cap)^2, up to x = cap / 4 (the next term, below 2^-26), and cap (1 - 2 u) from there
// (prefill of 8192 tokens, 32 heads over 8: 803 us, by the first form 651).
constexpr float kCapPlain = 64.0f;
// Larger caps and scales are refused: theirs are finite in the log2 domain.
constexpr float kScoreMost = 0x1p126f;

struct ScoreConsts {
  float scale2;               // scale * log2(e)
  float cap2, cap_in, ratio;  // softcap * log2(e); 2 log2(e) scale / softcap; scale / softcap
};

__device__ __forceinline__ ScoreConsts score_consts(float scale, float softcap) {
  // (kept finite, so that a product of 0 stays 0 however small the cap)
  const float ratio = softcap > 0.0f ? scale / softcap : 0.0f, in = 2.0f * kLog2e * ratio;
  return {scale * kLog2e, softcap * kLog2e, fminf(fmaxf(in, -3.0e38f), 3.0e38f), ratio};
}

__device__ __forceinline__ float cap_unit(float qk, const ScoreConsts& c) {
  return __builtin_amdgcn_rcpf(1.0f + exp2_fast(qk * c.cap_in));
}

// MODE: bit 0 capped, bit 1 slopes, bit 2 (with 0) a relative error (caps above kCapPlain, and edge_mode); dist =
// j - i, a whole number (callers add small ones to one conversion: exact below 2^24).
template <int MODE>
__device__ __forceinline__ float score2(float qk, const ScoreConsts& c, float slope2, float dist) {
  float s;
  if constexpr (MODE & 4) {
    const float t = qk * c.ratio, z = t * t;
    float p = __builtin_fmaf(z, 62.0f / 2835.0f, -17.0f / 315.0f);
    p = __builtin_fmaf(z, p, 2.0f / 15.0f);
    p = __builtin_fmaf(z, p, -1.0f / 3.0f);
    p = __builtin_fmaf(z, p, 1.0f);
    const float far = c.cap2 * __builtin_fmaf(-2.0f, cap_unit(qk, c), 1.0f);
    s = fabsf(t) < 0.25f ? qk * c.scale2 * p : far;      // (a NaN takes the second, NaN too)
  } else {
    s = MODE & 1 ? __builtin_fmaf(-2.0f * c.cap2, cap_unit(qk, c), c.cap2) : qk * c.scale2;
  }
  return MODE & 2 ? __builtin_fmaf(slope2, dist, s) : s;
}

// The MODE of capped scores whose error is relative: in decode those of a step of keys that the row does not see
// whole (a row of few keys has no others), in prefill those of rows of few keys.  There an error of the cap's size
// shows, in an lse as small as the scores (one key, a cap of 50: 1.1e-6).  For all steps the form takes 50 us for 47
// (48 sequences over e2m1 pages), and a quarter more of a long prompt's time.
constexpr int edge_mode(int mode) { return mode & 1 ? mode | 4 : mode; }

// x, in a way that work on it is not taken for work on x: what two forms of a score have in common would else be
// held for all scores at once, beside the scores (registers spilled).
__device__ __forceinline__ float apart(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Calls f(integral constant of the call's MODE).
template <class F>
void with_score_mode(const ScoreArgs& a, F&& f) {
  if (a.softcap > kCapPlain)
    a.slopes ? f(std::integral_constant<int, 7>{}) : f(std::integral_constant<int, 5>{});
  else if (a.softcap > 0.0f)
    a.slopes ? f(std::integral_constant<int, 3>{}) : f(std::integral_constant<int, 1>{});
  else
    a.slopes ? f(std::integral_constant<int, 2>{}) : f(std::integral_constant<int, 0>{});
}

// Joins the parts of every (row, head); ragged: rows outside its sequences are
// left as they are.
hipError_t launch_attn_join(const SplitArgs& sp, int rows, int Hq, int g, int D, const float* v_scale, RowsOut o,
                            float* lse, const BatchArgs* ragged, hipStream_t stream);
// At least rows * Hq * nsplit of any prefill call of up to T rows that splits.
size_t attn_prefill_split_rows(int T, int Hq);

}  // namespace mc
