// attn_decode.hip -- attention of one new token a sequence over the paged
// cache, split over its length and joined.
//
//   o = sum_j p_j v_j / l,  p_j = exp2(s_j - m),  l = sum_j p_j,  m = max_j s_j
// (s in the log2 domain), in one pass with a running maximum: a larger one
// scales what was summed by exp2(m_old - m_new).  Parts of the keys join the
// same way: M = max m_w, o = sum_w 2^(m_w - M) o_w / sum_w 2^(m_w - M) l_w.
//
// Bound by HBM: every key and value is read once, 4 g operations an element
// (g query heads share it).  The products are 16x16x32 matrix instructions with up
// to 16 query heads as their columns; that most columns are empty costs nothing
// that counts (5 % of the matrix rate at 8 TB/s).  48 sequences of 300 to 8191 tokens,
// 813 MB of bf16: 141 us, 5.8 TB/s; 2 of 50000 to 131071, 380 MB of e4m3: 70 us, 5.4 TB/s.
// One of 777: 8 us, two launches of three memory latencies each.  e2m1: 4 of 50000 to 131071, 441 MB, 83 us
// on data that no cache holds (72 on what was just read), the kernel's loads alone 69 of the 72; 48 of 300 to
// 8191, 216 MB: 52 and 47, loads alone 42.  Listed pages: 64 pages of 64 bf16 tokens of 16 sequences, 268 MB,
// 45 us, 6.0 TB/s; 228 rows of 32 pages of 64 e2m1 tokens 67 us, 28 thousand vector instructions a SIMD.
//
// A wave takes KS keys a step (32 of bf16, 64 of the others: 16 KB for D = 128, 8.5 of e2m1), all
// of it in registers straight from memory, the next step's loads issued before this
// one's products.  Scores are keys x heads (S^T = K Q^T): lane (head n = lane % 16,
// quarter q) holds 4 keys of each 16-key tile, and the tiles' rows are dealt so
// that these are consecutive keys, the very ones that the lane supplies
// to the product with the values (O^T = V^T P^T): nothing moves between lanes but the maximum.
// e2m1 keys take their scale in the conversion to bf16 (one instruction for two codes), since a lane's piece of
// a key has one; a lane's values have one scale a token, which goes to the token's weight.
#include "attn.hpp"

namespace mc {

constexpr int kDecWaves = 4;
constexpr int kDecThreads = 64 * kDecWaves;
constexpr int kDecHeads = 16;        // query heads of a workgroup
constexpr int kMaxSplit = 128;
constexpr int kNowhere = 0x7f000000;     // a position past all others

// The parts a cache is cut into.  Enough to fill the chip (two workgroups of 4 waves
// fit a CU's registers), as long as every wave has a step; more, up to
// kDecTarget workgroups, where a part keeps kDecPart bytes of keys and values: the
// shorter the parts, the less a long sequence of a ragged batch is waited for (48
// sequences of 300 to 8191 tokens, 0.9 GB: 204 us at one round of workgroups, 159 at four),
// and the more their starts and the join cost (64 sequences of 512: 24 us, with parts of a
// quarter 31).
constexpr int kDecFill = 512, kDecTarget = 2048, kDecPart = 192 << 10;

static int decode_splits(int S, int Hkv, int head_tiles, int max_len, int keys, int key_bytes) {
  const long long wgs = (long long)S * Hkv * head_tiles;
  const long long steps = ((long long)max_len + keys - 1) / keys;
  const long long fill = kDecFill / wgs, more = kDecTarget / wgs;
  long long n = (long long)max_len * key_bytes / kDecPart;
  n = n > more ? more : n;
  n = n < fill ? fill : n;
  n = n > steps ? steps : n;
  return (int)(n < 1 ? 1 : n > kMaxSplit ? kMaxSplit : n);
}

// The keys of a step as a lane takes them: whole 16-byte units, of e2m1 keys the part of a unit
// that holds D / 4 dimensions.  e2m1: the scale bytes of the lane's key in each tile, and the
// scales of its values, 64 dimensions after the other.
template <int D, int KV>
struct DecodeStep {
  static constexpr bool E4 = KV == MC_KV_E4M3, E2 = KV == MC_KV_E2M1;
  static constexpr int kTiles = KV == MC_KV_BF16 ? 2 : 4;                    // 16-key tiles
  static constexpr int kChunks = E2 ? 1 : D / (E4 ? 64 : 32);                // pieces of a key that a lane takes
  static constexpr int kKeys = 16 * kTiles, kValues = D / (E2 ? 32 : 16);
  using Piece = typename std::conditional<E2 && D == 64, u32x2, u32x4>::type;
  Piece k[kTiles][kChunks];
  u32x4 v[kValues];
  uint32_t ks;
  u32x4 vs[E2 ? D / 32 : 1];
};

// The pages that each row of a sparse call reads: sel [row][Hkv][n_sel] positions in the sequence's
// table row, the first count [row][Hkv] of them.
struct SparseArgs {
  const int32_t *sel, *count;
  int n_sel;
};

// How many steps a wave holds in registers.  One, and three waves a SIMD, of an e2m1 cache (48
// sequences of 300 to 8191 tokens 54 -> 46 us, 4 of 50000 to 131071 77 -> 71; four waves a SIMD spill: 70 and
// 97) and of listed pages (228 rows of 32 pages of 64 e4m3 tokens 67.6 -> 58.4 us, bf16 no difference); two, and two
// waves, of the others.
__host__ __device__ constexpr bool one_step(int kv, bool sparse) { return kv == MC_KV_E2M1 || sparse; }

// SPARSE: a row's keys are those of its listed pages, one after the other; a row is any token of
// a ragged batch (b.q_start null: the last of its sequence).
template <int D, int KV, int MODE, bool SPARSE>
__global__ void __launch_bounds__(kDecThreads, one_step(KV, SPARSE) ? 3 : 2)
    attn_decode_kernel(RowsIn q, BatchArgs b, KvArgs c, ScoreArgs a, RowsOut o, float* __restrict__ lse, SplitArgs sp,
                       int head_tiles, SparseArgs sparse) {
  using Step = DecodeStep<D, KV>;
  constexpr bool E4 = Step::E4, E2 = Step::E2;
  constexpr int KS = Step::kKeys, KT = Step::kTiles, KC = Step::kChunks, DT = D / 16, DP = D + 4, VT = Step::kValues;
  constexpr int kBlockBytes = KvFormat<D, KV>::kBlockBytes;
  // the waves' results; before them, of a sparse call, its pages: place in the table, and number
  constexpr int kResults = kDecWaves * kDecHeads * DP * 4, kLists = SPARSE ? 8 * MC_MAX_SELECT : 0;
  __shared__ __attribute__((aligned(16))) char s_all[kResults > kLists ? kResults : kLists];
  float (*s_o)[kDecHeads][DP] = reinterpret_cast<float (*)[kDecHeads][DP]>(s_all);
  __shared__ float s_ml[2][kDecWaves][kDecHeads];
  const int lane = threadIdx.x & 63, wave = wave_id(), n = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int split = id % sp.nsplit;
  id /= sp.nsplit;
  const int ht = id % head_tiles;
  id /= head_tiles;
  const int hk = id % c.Hkv, row = id / c.Hkv;
  const int head0 = hk * a.g + ht * kDecHeads, heads = min(kDecHeads, a.g - ht * kDecHeads);
  int s = row;
  if (SPARSE && b.q_start) {
    if (row < b.q_start[0] || row >= b.q_start[b.S]) return;         // padding
    s = find_sequence(b.q_start, b.S, row, 1, 0, 1);
  }

  // queries: lane (head n, quarter) holds the units that it takes of a key
  bf16x8 qf[D / 32];
  {
    const uint16_t* qr = q.p + (size_t)row * q.stride + (size_t)(head0 + n) * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      u32x4 r = {0u, 0u, 0u, 0u};
      const int at = E2 ? D / 4 * quarter + 8 * i
                        : E4 ? 16 * (4 * (i / 2) + quarter) + 8 * (i & 1) : 8 * (4 * i + quarter);
      if (n < heads) r = *reinterpret_cast<const u32x4*>(qr + at);
      qf[i] = as_bf16x8(r);
    }
  }

  // (of a sparse call: the tokens up to the row's own)
  int len = kv_length(c, b, s);
  if (SPARSE && b.q_start) {
    const long long own = (long long)b.kv_len[s] - ((long long)b.q_start[s + 1] - row) + 1;
    len = own < 0 ? 0 : own < len ? (int)own : len;
  }
  const int pos = len - 1;
  const int pre = SPARSE ? 0 : kv_prefix(a, s, len);
  const int wstart = a.window > 0 && len > a.window ? len - a.window : 0;   // first key of the window
  int listed = 0;
  const int32_t* list = nullptr;
  if (SPARSE) {
    listed = sparse.count[(size_t)row * c.Hkv + hk];
    listed = len == 0 || listed < 0 ? 0 : min(listed, sparse.n_sel);
    list = sparse.sel + ((size_t)row * c.Hkv + hk) * sparse.n_sel;
  }
  // steps that hold a visible key: [0, ia) and [ib, all)
  const int all = ((SPARSE ? (listed << c.lb) * kKvBlock : len) + KS - 1) / KS;
  int ia = (pre + KS - 1) / KS, ib = SPARSE ? 0 : wstart / KS;
  if (ib <= ia) ia = ib = 0;
  const int steps = ia + all - ib, per = (steps + sp.nsplit - 1) / sp.nsplit;
  const int i_end = min(steps, (split + 1) * per);
  int it = split * per + wave;

  const int32_t* pages = b.page_table + (size_t)s * b.max_pages;
  const int last_blk = SPARSE ? max((listed << c.lb) - 1, 0) : len > 0 ? (len - 1) >> 4 : 0;
  // the lane's blocks of a step: keys 8 n/4 .. (bf16) or 16 n/4 .. (the others) of
  // the step go through it as a score row, keys 8 or 16 quarter .. as values
  const int kblk = KT == 4 ? n >> 2 : n >> 3, vblk = KT == 4 ? quarter : quarter >> 1;
  auto step_blk = [&](int i) { return ((i < ia ? i : i - ia + ib) * KS) >> 4; };
  auto page_of = [&](int blk) { return pages[(blk < last_blk ? blk : last_blk) >> c.lb]; };
  const int koff = (E2 && D == 64) ? (n & 3) * 16 + (quarter >> 1) * 256 + 8 * (quarter & 1)
                                   : (KT == 4 ? (n & 3) : 8 * ((n >> 2) & 1) + (n & 3)) * 16 + quarter * 256;
  const int voff = (KT == 4 ? 0 : (quarter & 1) * D * 16) + n * 16;

  // Of a sparse call: the workgroup's pages, entries e0 on of the list.  A place outside the table
  // is one past every position.
  const int e0 = SPARSE ? min(((split * per * KS) >> 4) >> c.lb, max(listed - 1, 0)) : 0;
  int* s_sel = reinterpret_cast<int*>(s_all);
  int* s_page = s_sel + MC_MAX_SELECT;
  if (SPARSE) {
    const int e1 = min(((min(i_end, steps) * KS) >> 4 >> c.lb) + 1, listed);
    for (int i = e0 + (int)threadIdx.x; i < e1; i += kDecThreads) {
      const int at = list[i];
      const bool in = at >= 0 && at < b.max_pages;
      s_sel[i - e0] = in ? at : b.max_pages;
      s_page[i - e0] = in ? kv_page(c, pages[at]) : 0;
    }
    __syncthreads();
  }

  // Values are read once and by whole lines: past the caches (64 sequences of 4096
  // e4m3 tokens, 537 MB: 109 -> 86 us; of 1024 bf16 tokens and 16 heads 100 -> 83).  A
  // load of keys takes half of each line that it touches, the next the other half: those
  // stay ordinary loads (non-temporal ones: 58 us for 50 at 4 x 32768 e4m3 tokens).  Listed pages are read by
  // many rows of a chunk: ordinary loads for both (228 rows of 32 pages of 64 bf16 tokens 118 -> 77 us).
  auto load_keys = [&](Step& st, int i, int kp) {
    const int kb = min(step_blk(i) + kblk, last_blk);
    const int kpage = SPARSE ? s_page[(kb >> c.lb) - e0] : kv_page(c, kp);
    const char* kp0 = c.k + kv_block_offset<kBlockBytes>(c, kpage, hk, kb) + koff;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int u = 0; u < KC; ++u)
        st.k[t][u] = *reinterpret_cast<const typename Step::Piece*>(kp0 + 64 * t + 1024 * u);
    if constexpr (E2) {
      const char* ks = c.k + kv_scale_offset<D>(c, kpage, hk, kb);
      st.ks = *reinterpret_cast<const uint32_t*>(ks + 16 * (D == 64 ? quarter >> 1 : quarter) + 4 * (n & 3));
    }
  };
  auto load_values = [&](Step& st, int i, int vp) {
    const int vb = min(step_blk(i) + vblk, last_blk);
    const int vpage = SPARSE ? s_page[(vb >> c.lb) - e0] : kv_page(c, vp);
    const char* vp0 = c.v + kv_block_offset<kBlockBytes>(c, vpage, hk, vb) + voff;
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const u32x4* from = reinterpret_cast<const u32x4*>(vp0 + 256 * t);
      if constexpr (SPARSE)
        st.v[t] = *from;
      else
        st.v[t] = __builtin_nontemporal_load(from);
    }
    if constexpr (E2) {
      const char* vs = c.v + kv_scale_offset<D>(c, vpage, hk, vb);
#pragma unroll
      for (int t = 0; t < D / 32; ++t) st.vs[t] = *reinterpret_cast<const u32x4*>(vs + 16 * t);
    }
  };

  auto load = [&](Step& st, int i, int kp, int vp) {
    load_keys(st, i, kp);
    load_values(st, i, vp);
  };

  f32x4 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNegInf, l = 0.0f;       // l: of the lane's own keys
  const float kscale = E4 ? c.k_scale[hk] : 1.0f;
  const ScoreConsts sc = score_consts(a.scale * kscale, a.softcap);
  const float slope2 = (MODE & 2) && n < heads ? a.slopes[head0 + n] * kLog2e : 0.0f;

  // after_keys(): called once the step's keys have been used
  auto compute = [&](Step& st, int i, auto after_keys) {
    const int key0 = step_blk(i) << 4;
    f32x4 sv[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sv[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < KC; ++u) {
        if constexpr (E2) {
          const float scale = e8m0_scale(st.ks, t);
#pragma unroll
          for (int w = 0; w < D / 32; ++w)
            sv[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(e2m1_to_bf16(st.k[t][u][w], scale)), qf[w], sv[t],
                                                            0, 0, 0);
        } else if constexpr (E4) {
          sv[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(e4m3_to_bf16(st.k[t][u][0], st.k[t][u][1])),
                                                          qf[2 * u], sv[t], 0, 0, 0);
          sv[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(e4m3_to_bf16(st.k[t][u][2], st.k[t][u][3])),
                                                          qf[2 * u + 1], sv[t], 0, 0, 0);
        } else {
          sv[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(st.k[t][u]), qf[u], sv[t], 0, 0, 0);
        }
      }
    }
    after_keys();
    // lane (n, quarter): score (t, r) is of key key0 + 4 KT quarter + 4 t + r
    int lane_key = key0 + 4 * KT * quarter;
    if (SPARSE) {
      const int vb = min((key0 >> 4) + vblk, last_blk), at = s_sel[(vb >> c.lb) - e0];
      lane_key = (((at << c.lb) + (vb & ((1 << c.lb) - 1))) << 4) + (KT == 4 ? 0 : 8 * (quarter & 1));
      if (at >= b.max_pages || (key0 >> 4) + vblk > last_blk) lane_key = kNowhere;
    }
    const float dist = (float)(lane_key - pos);
    float x[4 * KT];
#pragma unroll
    for (int e = 0; e < 4 * KT; ++e) x[e] = score2<MODE>(sv[e / 4][e % 4], sc, slope2, dist + (float)e);
    const bool whole = SPARSE ? __all(lane_key >= wstart && lane_key + 4 * KT <= len)
                              : (key0 >= wstart && key0 + KS <= len) || key0 + KS <= pre;
    if (!whole) {
      if constexpr (MODE != edge_mode(MODE)) {     // (again: chosen before the loop above, registers spilled)
        const float far = apart(dist);
#pragma unroll
        for (int e = 0; e < 4 * KT; ++e)
          x[e] = score2<edge_mode(MODE)>(apart(sv[e / 4][e % 4]), sc, slope2, far + (float)e);
      }
      // keys out of sight: weight 0, and values 0 whatever the cache holds there
      uint32_t seen = 0;
#pragma unroll
      for (int e = 0; e < 4 * KT; ++e) {
        const int j = lane_key + e;
        const bool in = j < len && (j >= wstart || j < pre);
        x[e] = in ? x[e] : kNegInf;
        seen |= in ? 1u << e : 0u;
      }
#pragma unroll
      for (int w = 0; w < (E2 ? 8 : 4); ++w) {
        uint32_t keep = 0;
        if constexpr (E4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) keep |= (seen >> (4 * w + e)) & 1u ? 0xffu << (8 * e) : 0u;
        } else {
          keep = ((seen >> (2 * w)) & 1u ? 0xffffu : 0u) | ((seen >> (2 * w + 1)) & 1u ? 0xffff0000u : 0u);
        }
        // (an e2m1 code is always a number: it is the scales that may be anything)
        if constexpr (E2) {
#pragma unroll
          for (int t = 0; t < D / 64; ++t) st.vs[2 * t + w / 4][w % 4] &= keep;
        } else {
#pragma unroll
          for (int t = 0; t < DT; ++t) st.v[t][w] &= keep;
        }
      }
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 4 * KT; ++e) mx = fmaxf(mx, x[e]);
    mx = halves_max(rows_max(mx));
    const float m_new = fmaxf(m, mx);
    if (__any(m_new > m)) {
      const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(m - m_new);
      l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] *= alpha;
      m = m_new;
    }
    const float m0 = m == kNegInf ? 0.0f : m;
#pragma unroll
    for (int e = 0; e < 4 * KT; ++e) {
      x[e] = exp2_fast(x[e] - m0);
      l += x[e];
    }
    // for the matrix units the weights are rounded to bf16, by up to 2^-8 of each (values are
    // bf16 or less, and so is the result); their sum takes them as they are.  Those of e2m1 values
    // are multiplied with the values' scales first, and the values are their codes'.
    if constexpr (E2) {
#pragma unroll
      for (int w = 0; w < KT / 2; ++w)
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          u32x4 pr;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t vs = st.vs[2 * h + w][e];
            pr[e] = bf16_pair(x[8 * w + 2 * e] * half_of(vs, 0), x[8 * w + 2 * e + 1] * half_of(vs, 1));
          }
          const bf16x8 p = as_bf16x8(pr);
#pragma unroll
          for (int t = 4 * h; t < 4 * h + 4; ++t)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                as_bf16x8(e2m1_to_bf16(st.v[t / 2][2 * (t & 1) + w], 1.0f)), p, acc[t], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int w = 0; w < KT / 2; ++w) {
        u32x4 pr;
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[e] = bf16_pair(x[8 * w + 2 * e], x[8 * w + 2 * e + 1]);
        const bf16x8 p = as_bf16x8(pr);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          if constexpr (E4)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                as_bf16x8(e4m3_to_bf16(st.v[t][2 * w], st.v[t][2 * w + 1])), p, acc[t], 0, 0, 0);
          else
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(st.v[t]), p, acc[t], 0, 0, 0);
        }
      }
    }
  };

  // page numbers are fetched two steps ahead and before the loads of the step
  // between, so that waiting for them does not wait for those
  auto ids = [&](int i, int& kp, int& vp) {
    if (SPARSE) return;
    const int blk = step_blk(min(i, i_end - 1));
    kp = page_of(blk + kblk);
    vp = page_of(blk + vblk);
  };
  if constexpr (one_step(KV, SPARSE)) {
    // the next step's keys are loaded once this one's are used, its values likewise
    if (it < i_end) {
      Step st;
      int kp = 0, vp = 0, kn = 0, vn = 0;
      ids(it, kp, vp);
      ids(it + kDecWaves, kn, vn);
      load(st, it, kp, vp);
      while (true) {
        ids(it + 2 * kDecWaves, kp, vp);
        const bool more = it + kDecWaves < i_end;
        compute(st, it, [&]() {
          if (more) load_keys(st, it + kDecWaves, kn);
        });
        if (!more) break;
        load_values(st, it + kDecWaves, vn);
        kn = kp;
        vn = vp;
        it += kDecWaves;
      }
    }
  } else if (it < i_end) {
    const auto none = []() {};
    Step s0, s1;
    int kp0 = 0, vp0 = 0, kp1 = 0, vp1 = 0;
    ids(it, kp0, vp0);
    ids(it + kDecWaves, kp1, vp1);
    load(s0, it, kp0, vp0);
    while (true) {
      ids(it + 2 * kDecWaves, kp0, vp0);
      if (it + kDecWaves < i_end) load(s1, it + kDecWaves, kp1, vp1);
      compute(s0, it, none);
      it += kDecWaves;
      if (it >= i_end) break;
      ids(it + 2 * kDecWaves, kp1, vp1);
      if (it + kDecWaves < i_end) load(s0, it + kDecWaves, kp0, vp0);
      compute(s1, it, none);
      it += kDecWaves;
      if (it >= i_end) break;
    }
  }

  // join the four waves
  l = halves_sum(rows_sum(l));
  if (quarter == 0) {
    s_ml[0][wave][n] = m;
    s_ml[1][wave][n] = l;
  }
  __syncthreads();                   // (and the lists of a sparse call have been read)
  float M = kNegInf;
#pragma unroll
  for (int w = 0; w < kDecWaves; ++w) M = fmaxf(M, s_ml[0][w][n]);
  // a maximum of NaN scores stays -inf; their weights made l and acc NaN already
  const float M0 = M == kNegInf ? 0.0f : M;
  const float f = exp2_fast(m - M0);
  if (n < heads) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      f32x4 w;
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = f == 0.0f && l == 0.0f ? 0.0f : acc[t][r] * f;
      *reinterpret_cast<f32x4*>(&s_o[wave][n][16 * t + 4 * quarter]) = w;
    }
  }
  __syncthreads();
  const float* vscale = E4 ? c.v_scale : nullptr;
  for (int i = threadIdx.x; i < heads * (D / 4); i += kDecThreads) {
    const int h = i / (D / 4), d = 4 * (i % (D / 4)), hq = head0 + h;
    float Mh = kNegInf, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) Mh = fmaxf(Mh, s_ml[0][w][h]);
    const float Mh0 = Mh == kNegInf ? 0.0f : Mh;
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) {
      const float lw = s_ml[1][w][h];
      if (lw != 0.0f) L += lw * exp2_fast(s_ml[0][w][h] - Mh0);
      const f32x4 ow = *reinterpret_cast<const f32x4*>(&s_o[w][h][d]);
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] += ow[e];
    }
    if (sp.nsplit == 1) {
      const float f1 = L == 0.0f ? 0.0f : (E4 ? vscale[hk] : 1.0f) / L;
      u32x2 w;
      w[0] = L == 0.0f ? 0u : bf16_pair(r[0] * f1, r[1] * f1);
      w[1] = L == 0.0f ? 0u : bf16_pair(r[2] * f1, r[3] * f1);
      *reinterpret_cast<u32x2*>(o.p + (size_t)row * o.stride + (size_t)hq * D + d) = w;
      if (lse && d == 0) lse[(size_t)row * a.Hq + hq] = L == 0.0f ? kNegInf : (Mh0 + __log2f(L)) * kLn2;
    } else {
      const size_t part = ((size_t)row * a.Hq + hq) * sp.nsplit + split;
      if (L != 0.0f) *reinterpret_cast<f32x4*>(sp.o + part * D + d) = r;
      if (d == 0) {
        sp.ml[2 * part] = Mh0;
        sp.ml[2 * part + 1] = L;
      }
    }
  }
}

// One workgroup a (row, head).  Every wave finds the parts' factors
// 2^(m - M) for itself; then D/4 threads take a part's row, 16 bytes each, the
// 256 threads 8 (D = 128) or 16 parts at once, and their sums are joined in LDS in a fixed
// order.  Parts without a visible key have l = 0 and no o: what lies in its place is
// read, so that no load waits for another, and left out.  (A wave for all parts of a
// (row, head) took 56 us for 64 of them in 128 parts, this 4.8.)
constexpr int kJoinThreads = 256;

template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(SplitArgs sp, int Hq, int g,
                                                                 const float* __restrict__ v_scale, RowsOut o,
                                                                 float* __restrict__ lse,
                                                                 const int32_t* __restrict__ q_start, int S) {
  constexpr int kGroup = D / 4, kGroups = kJoinThreads / kGroup;
  __shared__ float s_f[kMaxSplit];
  __shared__ f32x4 s_o[kGroups][kGroup];
  const int lane = threadIdx.x & 63, w = blockIdx.x;
  const int row = w / Hq, h = w - row * Hq;
  if (q_start && (row < q_start[0] || row >= q_start[S])) return;   // padding
  const float* ml = sp.ml + (size_t)w * sp.nsplit * 2;
  float mv[kMaxSplit / 64], lv[kMaxSplit / 64], M = kNegInf;
#pragma unroll
  for (int i = 0; i < kMaxSplit / 64; ++i) {
    const int part = lane + 64 * i;
    mv[i] = kNegInf;
    lv[i] = 0.0f;
    if (part < sp.nsplit) {
      mv[i] = ml[2 * part];
      lv[i] = ml[2 * part + 1];
      if (lv[i] == 0.0f) mv[i] = kNegInf;
    }
    M = fmaxf(M, mv[i]);
  }
  M = wave_max(M);
  const float M0 = M == kNegInf ? 0.0f : M;
  float L = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxSplit / 64; ++i) {
    const float f = lv[i] == 0.0f ? 0.0f : exp2_fast(mv[i] - M0);
    L += lv[i] == 0.0f ? 0.0f : lv[i] * f;
    // -1: no o (a factor may itself be 0)
    if (threadIdx.x < 64) s_f[lane + 64 * i] = lv[i] == 0.0f ? -1.0f : f;
  }
  L = wave_sum(L);
  __syncthreads();
  const int grp = threadIdx.x / kGroup, d = threadIdx.x % kGroup;
  const float* po = sp.o + (size_t)w * sp.nsplit * D + 4 * d;
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int part = grp; part < sp.nsplit; part += kGroups) {
    const float f = s_f[part];
    const f32x4 v = *reinterpret_cast<const f32x4*>(po + (size_t)part * D);
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] += f == -1.0f ? 0.0f : v[e] * f;
  }
  s_o[grp][d] = r;
  __syncthreads();
  if (threadIdx.x >= kGroup) return;
#pragma unroll
  for (int i = 1; i < kGroups; ++i) {
    const f32x4 v = s_o[i][d];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] += v[e];
  }
  const float f = L == 0.0f ? 0.0f : (v_scale ? v_scale[h / g] : 1.0f) / L;
  u32x2 out = {0u, 0u};
  if (L != 0.0f) {
    out[0] = bf16_pair(r[0] * f, r[1] * f);
    out[1] = bf16_pair(r[2] * f, r[3] * f);
  }
  *reinterpret_cast<u32x2*>(o.p + (size_t)row * o.stride + (size_t)h * D + 4 * d) = out;
  if (lse && d == 0) lse[(size_t)row * Hq + h] = L == 0.0f ? kNegInf : (M0 + __log2f(L)) * kLn2;
}

// Few parts, FEW at most: D/4 threads a (row, head), 16 bytes of a part each, all
// loads at once.  A prefill of 896 rows of 32 heads in two parts: 48.2 us with the kernel
// above, 33.7 with this for up to 8, 30.8 for 2 (fewer registers, more waves).  One row of
// 16 heads in 7 parts: the kernel takes 2.9 us (6.4 where one part followed the other).
constexpr int kJoinFew = 8;

template <int D, int FEW>
__global__ void __launch_bounds__(kJoinThreads) attn_join_few_kernel(SplitArgs sp, int all, int Hq, int g,
                                                                     const float* __restrict__ v_scale, RowsOut o,
                                                                     float* __restrict__ lse,
                                                                     const int32_t* __restrict__ q_start, int S) {
  constexpr int kGroup = D / 4;
  const int w = blockIdx.x * (kJoinThreads / kGroup) + threadIdx.x / kGroup, d = threadIdx.x % kGroup;
  if (w >= all) return;
  const int row = w / Hq, h = w - row * Hq;
  if (q_start && (row < q_start[0] || row >= q_start[S])) return;   // padding
  const float* ml = sp.ml + (size_t)w * sp.nsplit * 2;
  const float* po = sp.o + (size_t)w * sp.nsplit * D + 4 * d;
  float mv[FEW], lv[FEW], M = kNegInf, L = 0.0f;
  f32x4 v[FEW], r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < FEW; ++i) {           // all loads first
    const int part = min(i, sp.nsplit - 1);
    mv[i] = ml[2 * part];
    lv[i] = ml[2 * part + 1];
    if (i < sp.nsplit) v[i] = *reinterpret_cast<const f32x4*>(po + (size_t)part * D);
  }
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    if (i >= sp.nsplit) lv[i] = 0.0f;
    M = fmaxf(M, lv[i] == 0.0f ? kNegInf : mv[i]);
  }
  const float M0 = M == kNegInf ? 0.0f : M;
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    const float f = exp2_fast(mv[i] - M0);
    L += lv[i] == 0.0f ? 0.0f : lv[i] * f;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] += lv[i] == 0.0f ? 0.0f : v[i][e] * f;
  }
  const float f = L == 0.0f ? 0.0f : (v_scale ? v_scale[h / g] : 1.0f) / L;
  u32x2 out = {0u, 0u};
  if (L != 0.0f) {
    out[0] = bf16_pair(r[0] * f, r[1] * f);
    out[1] = bf16_pair(r[2] * f, r[3] * f);
  }
  *reinterpret_cast<u32x2*>(o.p + (size_t)row * o.stride + (size_t)h * D + 4 * d) = out;
  if (lse && d == 0) lse[(size_t)row * Hq + h] = L == 0.0f ? kNegInf : (M0 + __log2f(L)) * kLn2;
}

hipError_t launch_attn_join(const SplitArgs& sp, int rows, int Hq, int g, int D, const float* v_scale, RowsOut o,
                            float* lse, const BatchArgs* ragged, hipStream_t stream) {
  const int all = rows * Hq, per = kJoinThreads / (D / 4);
  const int32_t* q_start = ragged ? ragged->q_start : nullptr;
  const int S = ragged ? ragged->S : 0;
  timing_begin(stream, kSiteAttnJoin);
  if (sp.nsplit <= kJoinFew) {
    const dim3 grid((all + per - 1) / per);
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kJoinThreads), 0, stream, sp, all, Hq, g, v_scale, o, lse, q_start, S);
    };
    if (sp.nsplit == 2)
      D == 64 ? launch(attn_join_few_kernel<64, 2>) : launch(attn_join_few_kernel<128, 2>);
    else
      D == 64 ? launch(attn_join_few_kernel<64, kJoinFew>) : launch(attn_join_few_kernel<128, kJoinFew>);
  } else if (D == 64) {
    hipLaunchKernelGGL(attn_join_kernel<64>, dim3(all), dim3(kJoinThreads), 0, stream, sp, Hq, g, v_scale, o, lse,
                       q_start, S);
  } else {
    hipLaunchKernelGGL(attn_join_kernel<128>, dim3(all), dim3(kJoinThreads), 0, stream, sp, Hq, g, v_scale, o, lse,
                       q_start, S);
  }
  timing_end(stream, kSiteAttnJoin);
  return hipGetLastError();
}

// Partial rows of a query head: a call that splits has S * nsplit <=
// kDecTarget / Hkv of them, and at most kMaxSplit a sequence; prefill's bound is its own.
size_t attn_workspace_bytes(int T, int Hq, int Hkv, int D) {
  const size_t most = kDecTarget / Hkv, all = (size_t)T * kMaxSplit;
  size_t rows = (all < most ? all : most) * Hq;
  const size_t pre = attn_prefill_split_rows(T, Hq);
  if (pre > rows) rows = pre;
  return rows * (size_t)(D + 2) * sizeof(float);
}

template <int D, bool SPARSE>
static void decode_launch(RowsIn q, int rows, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a, RowsOut o,
                          float* lse, const SplitArgs& sp, int head_tiles, const SparseArgs& sparse,
                          hipStream_t stream) {
  const dim3 grid((unsigned)((size_t)rows * c.Hkv * head_tiles * sp.nsplit));
  with_kv_kind(c, [&](auto kind) {
    with_score_mode(a, [&](auto mode) {
      hipLaunchKernelGGL((attn_decode_kernel<D, decltype(kind)::value, decltype(mode)::value, SPARSE>), grid,
                         dim3(kDecThreads), 0, stream, q, b, c, a, o, lse, sp, head_tiles, sparse);
    });
  });
}

// Keys of a step, and bytes of a key and its value.
static int step_keys(const KvArgs& c) { return c.kind == MC_KV_BF16 ? 32 : 64; }
static int pair_bytes(const KvArgs& c, int D) {
  return c.kind == MC_KV_BF16 ? 4 * D : c.kind == MC_KV_E4M3 ? 2 * D : D + D / 16;
}

hipError_t launch_attn_decode(RowsIn q, int D, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a, RowsOut o,
                              float* lse, int max_len, void* ws, hipStream_t stream) {
  const int head_tiles = (a.g + kDecHeads - 1) / kDecHeads;
  if (a.window > 0 && !a.prefix && a.window < max_len) max_len = a.window;
  SplitArgs sp;
  sp.nsplit = decode_splits(b.S, c.Hkv, head_tiles, max_len, step_keys(c) * kDecWaves, pair_bytes(c, D));
  sp.o = static_cast<float*>(ws);
  sp.ml = sp.o + (size_t)b.S * a.Hq * sp.nsplit * D;
  timing_begin(stream, kSiteAttnDecode);
  if (D == 64)
    decode_launch<64, false>(q, b.S, b, c, a, o, lse, sp, head_tiles, {}, stream);
  else
    decode_launch<128, false>(q, b.S, b, c, a, o, lse, sp, head_tiles, {}, stream);
  timing_end(stream, kSiteAttnDecode);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit == 1) return err;
  return launch_attn_join(sp, b.S, a.Hq, a.g, D, c.v_scale, o, lse, nullptr, stream);
}

hipError_t launch_attn_sparse(RowsIn q, int D, const BatchArgs& b, const KvArgs& c, const ScoreArgs& a,
                              const int32_t* sel, const int32_t* count, int n_sel, RowsOut o, float* lse, void* ws,
                              hipStream_t stream) {
  const int rows = b.q_start ? b.T : b.S, head_tiles = (a.g + kDecHeads - 1) / kDecHeads;
  const int keys = (n_sel << c.lb) * kKvBlock;
  SplitArgs sp;
  sp.nsplit = decode_splits(rows, c.Hkv, head_tiles, keys, step_keys(c) * kDecWaves, pair_bytes(c, D));
  sp.o = static_cast<float*>(ws);
  sp.ml = sp.o + (size_t)rows * a.Hq * sp.nsplit * D;
  timing_begin(stream, kSiteAttnSparse);
  if (D == 64)
    decode_launch<64, true>(q, rows, b, c, a, o, lse, sp, head_tiles, {sel, count, n_sel}, stream);
  else
    decode_launch<128, true>(q, rows, b, c, a, o, lse, sp, head_tiles, {sel, count, n_sel}, stream);
  timing_end(stream, kSiteAttnSparse);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit == 1) return err;
  return launch_attn_join(sp, rows, a.Hq, a.g, D, c.v_scale, o, lse, b.q_start ? &b : nullptr, stream);
}

}  // namespace mc
