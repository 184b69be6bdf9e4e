// Attention with a sliding window, first tokens that stay visible (sinks) and a
// learned relative position bias by buckets; shared key-value heads, padded
// sequences; forward and backward.
//
//   p_i = len_k - len_q + i                       position of query row i
//   visible(i, j): j < len_k, [j <= p_i,] and [|p_i - j| < window or j < sinks]
//   x_ij = scale q_i.k_j + table[bucket[clamp(j - p_i, -R, R) + R]][head]
//   P = softmax of x over the visible keys (a row without any: all zero), O = P V
//   dP = dO V^T, D_i = sum_j P_ij dP_ij, dS = P (dP - D)
//   dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO, dtable[t][h] += sum of dS over
//   the pairs of bucket t
//
// One pass over the visible key tiles with the running maximum and sum of the
// softmax; tiles outside every row's window are never touched, whole tiles inside
// it take no mask.  The score block is held transposed (one query, or key, per
// lane) as in k_attention.hip.  The storage types differ in an Ops struct: how a
// tile gets to LDS, how a score block and a product with the tile's transpose are
// formed.  bf16 products run on MFMA 32x32x16, P and dS rounded to bf16 on their
// way into the second product (they are never stored; every sum stays in fp32);
// fp32 ones on MFMA 32x32x2 in fp32 throughout.
//
// Times beside the kernels are traced launches in the first ten passes after a pause, where nothing else is said.
// Under load for some hundred launches the card is up to a fifth faster: the case of 8192 tokens and window 1024
// then takes 172 us forward, 227 for dQ, 296 for dK/dV and 11 for its join.
#include <algorithm>
#include <type_traits>

#include "attn_core.h"
#include "common.h"
#include "kernels.h"

namespace rg {

// A table entry at or below this hides its bucket (the type's lowest value and
// -infinity alike): its pairs are not visible.
constexpr float kHidden = -1e30f;

// ================================================================ who sees whom
struct Seq {
  int lq, lk, off;  // queries, keys, position of query 0
};
__device__ __forceinline__ Seq seq_of(const MaskedAttnArgs& a, int b) {
  Seq s;
  s.lq = a.len_q ? min(max(a.len_q[b], 0), a.Sq) : a.Sq;
  s.lk = a.len_k ? min(max(a.len_k[b], 0), a.Sk) : a.Sk;
  s.off = s.lk - s.lq;
  return s;
}

struct Mask {
  int lk, causal, window, sinks;  // window 0: none
  __device__ __forceinline__ Mask(const MaskedAttnArgs& a, int lk_)
      : lk(lk_), causal(a.causal), window(a.window), sinks(a.sinks) {}
};
// The visible ones among consecutive rows: one interval (and, for a query, the first `sinks`
// keys), so a test is a subtraction and a comparison or two.  No branches: what follows in a
// wave has matrix instructions and transpose reads, which take all 64 lanes, so no lane
// may leave on its own.
struct Visible {
  int lo;
  unsigned n1;  // interval lo .. lo + n1
  int sinks;
  __device__ __forceinline__ Visible(int lo_, int hi, int sinks_) : lo(lo_), n1(hi - lo_), sinks(sinks_) {
    if (hi < lo_) {
      lo = 1 << 30;  // beyond every row
      n1 = 0;
    }
  }
  __device__ __forceinline__ bool has(int i) const { return ((unsigned)(i - lo) <= n1) | (i < sinks); }
};
// keys of the query at position p
__device__ __forceinline__ Visible keys_of(const Mask& m, int p) {
  int lo = 0, hi = m.lk - 1, sk = 0;
  if (m.causal) hi = min(hi, p);
  if (m.window) {
    sk = min(m.sinks, hi + 1);
    lo = max(lo, p - m.window + 1);
    hi = min(hi, p + m.window - 1);
  }
  return Visible(lo, hi, sk);
}
// query rows (row i at position off + i, lq of them) of a key; no sinks: to one every row is near
__device__ __forceinline__ Visible rows_of(const Mask& m, int key, int off, int lq) {
  int lo = 0, hi = lq - 1;
  if (m.causal) lo = max(lo, key - off);
  if (m.window && key >= m.sinks) {
    lo = max(lo, key - m.window + 1 - off);
    hi = min(hi, key + m.window - 1 - off);
  }
  return Visible(lo, key < m.lk ? hi : -1, 0);
}

// What a loop meets, by blocks of 32: blocks v0 .. v1 and those below vs hold something
// visible, f0 .. f1 and those below fs nothing else.  Worked out once per wave, so that a step
// costs a few scalar comparisons.
struct Span {
  int v0, v1, vs, f0, f1, fs;
  // 0 nothing visible, 2 everything, 1 else
  __device__ __forceinline__ int kind(int blk) const {
    const bool full = (blk >= f0 && blk <= f1) || blk < fs, some = (blk >= v0 && blk <= v1) || blk < vs;
    return full ? 2 : some ? 1 : 0;
  }
};
// key blocks for the query positions plo .. phi
__device__ __forceinline__ Span key_span(const Mask& m, int plo, int phi) {
  Span s{0, 0, 0, 0, 0, 0};
  int hi = m.lk - 1, fhi = m.lk - 1;
  if (m.causal) {
    hi = min(hi, phi);
    fhi = min(fhi, plo);
  }
  if (m.window) {
    s.v0 = max(0, plo - m.window + 1) >> 5;
    s.f0 = (max(0, phi - m.window + 1) + 31) >> 5;
    s.vs = (min(m.sinks, hi + 1) + 31) >> 5;
    s.fs = max(0, min(m.sinks, fhi + 1)) >> 5;
    if (!m.causal) {
      hi = min(hi, phi + m.window - 1);
      fhi = min(fhi, plo + m.window - 1);
    }
  }
  s.v1 = hi >> 5;
  s.f1 = ((fhi + 1) >> 5) - 1;
  return s;
}
// blocks of query rows (positions off + row, lq rows) for the keys k0 .. k0 + 31; the whole 32
// rows and keys exist in a full one
__device__ __forceinline__ Span query_span(const Mask& m, int k0, int off, int lq) {
  const int k1 = k0 + 31;
  Span s{0, 0, 0, 0, 0, 0};
  int lo = 0, hi = lq - 1, flo = 0, fhi = lq - 1;
  if (m.causal) {
    lo = max(lo, k0 - off);
    flo = max(flo, k1 - off);
  }
  if (m.window) {
    if (k0 >= m.sinks) hi = min(hi, k1 + m.window - 1 - off);
    if (k1 >= m.sinks) fhi = min(fhi, k0 + m.window - 1 - off);
    if (!m.causal) {
      if (k0 >= m.sinks) lo = max(lo, k0 - m.window + 1 - off);
      if (k1 >= m.sinks) flo = max(flo, k1 - m.window + 1 - off);
    }
  }
  if (k0 >= m.lk) hi = -1;
  if (k1 >= m.lk) fhi = -1;
  s.v0 = lo >> 5;
  s.v1 = hi >> 5;
  s.f0 = (flo + 31) >> 5;
  s.f1 = ((fhi + 1) >> 5) - 1;
  return s;
}
// the tiles of KR keys that positions plo .. phi can see: the sinks' tiles, then
// the window's
struct KeyTiles {
  int nsink, t0, n;
  __device__ __forceinline__ int at(int i) const { return i < nsink ? i : t0 + i - nsink; }
};
template <int KR>
__device__ __forceinline__ KeyTiles key_tiles(const Mask& m, int plo, int phi) {
  int hi = m.lk - 1, lo = 0, ns = 0;
  if (m.causal) hi = min(hi, phi);
  if (m.window) {
    if (!m.causal) hi = min(hi, phi + m.window - 1);
    lo = max(0, plo - m.window + 1);
    int s = min(m.sinks, m.lk);
    if (m.causal) s = min(s, phi + 1);
    ns = s > 0 ? (s + KR - 1) / KR : 0;
  }
  KeyTiles t{ns, 0, ns};
  if (hi >= lo) {
    t.t0 = lo / KR;
    t.nsink = min(ns, t.t0);
    t.n = t.nsink + max(hi / KR, ns - 1) - t.t0 + 1;  // sinks may reach past the window
  }
  return t;
}

// ================================================================ the pipeline
// Pairs of tiles stream through ST stages in LDS, ST - 1 of them under way: a stage is
// refilled once the barrier says that its readers are done, and waited for by the count of
// DMAs issued since (PER per tile and wave; memory returns them in order).  One tile ahead, as in
// k_attention.hip, the wait for memory was most of an iteration at short windows.
template <int N>
__device__ __forceinline__ void wait_dma() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
// tile i of n has landed, for every wave; `ahead` tiles are in flight behind it at most
template <int ST, int PER>
__device__ __forceinline__ void tile_ready(int i, int n) {
  static_assert(ST >= 2 && ST <= 4 && PER * (ST - 2) < 64, "vmcnt counts to 63");
  const int ahead = min(ST - 2, n - 1 - i);
  if (ST == 4 && ahead == 2) wait_dma<PER*(ST > 3 ? 2 : 0)>();
  else if (ST >= 3 && ahead == 1) wait_dma<PER*(ST > 2 ? 1 : 0)>();
  else wait_dma<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Values loaded before the loop are waited for there: left to the first use, the wait sits inside
// the loop, where every step then waits for the DMAs it has just issued.
template <typename T>
__device__ __forceinline__ void settle(T& x) {
  asm volatile("" : "+v"(x));
}

// Products that a branch follows are waited for before it.  The compiler counts wait states from a matrix
// instruction to the first use of its result along one of the ways only where both start at its block: behind the
// two branches that choose a block's constant bias it left 7 of 11, and the scores read there changed from run
// to run.  STATES: of the instruction's passes, and then some.
template <int STATES>
__device__ __forceinline__ void landed(f32x16& x) {
  static_assert(STATES > 0 && STATES <= 32, "two s_nop");
  if constexpr (STATES > 16) asm volatile("s_nop 15\n\ts_nop %1" : "+v"(x) : "n"(STATES - 17));
  else asm volatile("s_nop %1" : "+v"(x) : "n"(STATES - 1));
}

// ================================================================ storage types
// A tile is KR rows of one head in LDS.  dma() brings this wave's share (of NW) of rows 0 .. KR - 1
// from src (rows past `last` read row `last`: what they score is masked); scores() forms the block
// [32 tile rows][32 own rows] (lane = own row, register r = tile row perm_pos(r)); accum() adds
// tile^T p to acc (lane = own row, registers = head dims).
template <int DH_>
struct OpsBf16 {
  static constexpr int BLOCK_DMAS(int rows) { return rows * DH_ / 512; }  // 1 KB each
  static constexpr int DH = DH_, KR = 64, ST = DH == 64 ? 3 : 2, TILE = KR * DH, STAGE = 32 * (DH + 8), WAVES = 2;
  static constexpr int LANDS = 12;  // wait states of a product (8 passes)
  static constexpr int BLOCK = 32 * DH, DMAS = BLOCK_DMAS(32);  // elements of 32 rows, and their DMAs
  typedef bf16 E;
  struct Rows {
    bf16x8 f[DH / 16];
    __device__ __forceinline__ void settled() {
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) settle(f[i]);
    }
  };
  TileRead<DH> rd;
  __device__ __forceinline__ OpsBf16(int lane, int) : rd(lane) {}
  // the LDS read offsets are formed anew from here on: kept across a loop they spill at d_head 128
  __device__ __forceinline__ void fresh() {
    if constexpr (DH == 128) asm volatile("" : "+v"(rd.row), "+v"(rd.tr));
  }
  static __device__ __forceinline__ void load_rows(Rows& o, const E* row, bool valid, int half, int) {
    load_row_frags<DH>(row, valid, half, o.f);
  }
  // the same from a tile: rows kb * 32 + lane % 32
  __device__ __forceinline__ void tile_rows(Rows& o, const E* tile, int kb, int) const {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) o.f[i] = rd.frag(tile, kb, i);
  }
  static __device__ __forceinline__ float dot(const Rows& x, const Rows& y) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) {
      float u[8], w[8];
      unpack_frag(x.f[i], u);
      unpack_frag(y.f[i], w);
#pragma unroll
      for (int v = 0; v < 8; ++v) s += u[v] * w[v];
    }
    return s + __shfl_xor(s, 32, 64);
  }
  // byte offset of this lane in DMA i of a wave; rows past `last` give row `last`
  template <int NW>
  static __device__ __forceinline__ uint32_t dma_at(int i, long ld, int last, int, int lane, int wave) {
    constexpr int CPR = DH / 8, RPI = 64 / CPR;
    const int r = (i * NW + wave) * RPI + lane / CPR, c = (lane % CPR) ^ swz<DH>(r);
    return ((uint32_t)min(r, last) * (uint32_t)ld + c * 8) * 2;
  }
  // ... in DMA 0 of a whole tile: DMA i is i * NW * RPI rows on (the swizzle repeats after 16 rows)
  template <int NW>
  static __device__ __forceinline__ uint32_t dma_first(long ld, int dh, int lane, int wave) {
    return dma_at<NW>(0, ld, KR, dh, lane, wave);
  }
  template <int NW>
  static __device__ __forceinline__ void dma(const E* src, long ld, int last, E* dst, int dh, int lane, int wave,
                                             uint32_t first) {
    constexpr int RPI = 512 / DH, N = KR / (RPI * NW);
    static_assert(KR % (RPI * NW) == 0 && NW * RPI % 16 == 0, "whole DMA instructions per wave");
    src = uniform_ptr(src);
    const uint32_t lds = lds_addr(dst) + wave * 1024;
    if (last >= KR - 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) dma16_m0(src + i * (NW * RPI) * ld, first, lds + i * NW * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) dma16_m0(src, dma_at<NW>(i, ld, last, dh, lane, wave), lds + i * NW * 1024);
    }
  }
  // 32 rows by one wave
  static __device__ __forceinline__ void dma_block(const E* src, long ld, int last, E* dst, int dh, int lane) {
    src = uniform_ptr(src);
#pragma unroll
    for (int i = 0; i < BLOCK_DMAS(32); ++i) dma16_m0(src, dma_at<1>(i, ld, last, dh, lane, 0), lds_addr(dst) + i * 1024);
  }
  __device__ __forceinline__ void scores(f32x16& st, const E* tile, int kb, const Rows& own) const {
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) st = mfma32(rd.frag(tile, kb, s), own.f[s], st);
  }
  __device__ __forceinline__ void accum(f32x16 (&acc)[DH / 32], const E* tile, int kb, const f32x16& p) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x8 pf = pack8(p, j);
#pragma unroll
      for (int db = 0; db < DH / 32; ++db) acc[db] = mfma32(rd.perm(tile, db, kb, j), pf, acc[db]);
    }
  }
  static __device__ __forceinline__ void rotate_back(f32x16 (&acc)[DH / 32], const float2* tab, int pos, int half) {
    if (tab) unrotate<DH>(acc, pos, tab, half);
  }
  static __device__ __forceinline__ void store(const f32x16 (&acc)[DH / 32], float scale, int lane, E* stage, E* dst,
                                               long ld, bool nt, int n, int) {
    store_rows_staged<DH>(acc, scale, lane >> 5, lane, stage, dst, ld, nt, n);
  }
};

// Head dims dh <= DHM; columns dh .. DHM - 1 of a tile repeat column dh - 1 and meet
// zeros in the own rows.
template <int DHM>
struct OpsF32 {
  static constexpr int BLOCK_DMAS(int rows) { return rows * DHM / 64; }  // 64 floats each
  static constexpr int DH = DHM, KR = 32, ST = DHM == 64 ? 4 : 3, P = DHM + 4, TILE = KR * P, STAGE = 32 * P, WAVES = 1;
  static constexpr int LANDS = 20;  // wait states of a product (16 passes)
  static constexpr int BLOCK = TILE, DMAS = BLOCK_DMAS(KR);
  typedef float E;
  struct Rows {
    float f[DHM / 2];  // dims half * DHM / 2 + i
    // zero from dim n on; by integer masks, as comparisons would take a scalar pair per element
    __device__ __forceinline__ void cut(int half, int n) {
#pragma unroll
      for (int i = 0; i < DHM / 2; ++i)
        f[i] = __int_as_float(__float_as_int(f[i]) & ((half * (DHM / 2) + i - n) >> 31));
    }
    __device__ __forceinline__ void settled() {
#pragma unroll
      for (int i = 0; i < DHM / 2; ++i) settle(f[i]);
    }
  };
  int row, col, half;
  __device__ __forceinline__ OpsF32(int lane, int) {
    half = lane >> 5;
    row = (lane & 31) * P + half * (DHM / 2);
    col = lane & 31;
  }
  __device__ __forceinline__ void fresh() {}
  static __device__ __forceinline__ void load_rows(Rows& o, const E* src, bool valid, int half, int dh) {
#pragma unroll
    for (int i = 0; i < DHM / 2; ++i) o.f[i] = src[min(half * (DHM / 2) + i, dh - 1)];
    o.cut(half, valid ? dh : 0);
  }
  // dims dh .. DHM - 1 hold what the tile holds there: zero them in one operand of a product
  __device__ __forceinline__ void tile_rows(Rows& o, const E* tile, int, int dh) const {
#pragma unroll
    for (int i = 0; i < DHM / 8; ++i) {
      const float4 t = *reinterpret_cast<const float4*>(tile + row + 4 * i);
      o.f[4 * i] = t.x;
      o.f[4 * i + 1] = t.y;
      o.f[4 * i + 2] = t.z;
      o.f[4 * i + 3] = t.w;
    }
    o.cut(half, dh);
  }
  static __device__ __forceinline__ float dot(const Rows& x, const Rows& y) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < DHM / 2; ++i) s = fmaf(x.f[i], y.f[i], s);
    return s + __shfl_xor(s, 32, 64);
  }
  // 4 B per lane: any alignment of the rows will do
  template <int NW>
  static __device__ __forceinline__ uint32_t dma_at(int i, long ld, int last, int dh, int lane, int wave) {
    constexpr int CPR = DHM / 64;
    const int n = i * NW + wave;
    return ((uint32_t)min(n / CPR, last) * (uint32_t)ld + min(n % CPR * 64 + lane, dh - 1)) * 4;
  }
  template <int NW>
  static __device__ __forceinline__ uint32_t dma_first(long ld, int dh, int lane, int wave) {
    return dma_at<NW>(0, ld, KR, dh, lane, wave);
  }
  template <int NW>
  static __device__ __forceinline__ void dma(const E* src, long ld, int last, E* dst, int dh, int lane, int wave,
                                             uint32_t first) {
    constexpr int CPR = DHM / 64, N = KR * CPR / NW;
    static_assert(KR * CPR % NW == 0 && NW % CPR == 0, "whole DMA instructions per wave, each of one part of the rows");
    src = uniform_ptr(src);
    const uint32_t lds = lds_addr(dst) + (wave / CPR * P + wave % CPR * 64) * 4;
    if (last >= KR - 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) dma4_m0(src + i * (NW / CPR) * ld, first, lds + i * (NW / CPR) * P * 4);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) dma4_m0(src, dma_at<NW>(i, ld, last, dh, lane, wave), lds + i * (NW / CPR) * P * 4);
    }
  }
  static __device__ __forceinline__ void dma_block(const E* src, long ld, int last, E* dst, int dh, int lane) {
    constexpr int CPR = DHM / 64;
    src = uniform_ptr(src);
#pragma unroll
    for (int i = 0; i < BLOCK_DMAS(KR); ++i)
      dma4_m0(src, dma_at<1>(i, ld, last, dh, lane, 0), lds_addr(dst) + (i / CPR * P + i % CPR * 64) * 4);
  }
  __device__ __forceinline__ void scores(f32x16& st, const E* tile, int kb, const Rows& own) const {
    (void)kb;  // a tile is one block
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
    for (int i = 0; i < DHM / 8; ++i) {
      const float4 t = *reinterpret_cast<const float4*>(tile + row + 4 * i);
      st = mfma32_f32(t.x, own.f[4 * i], st);
      st = mfma32_f32(t.y, own.f[4 * i + 1], st);
      st = mfma32_f32(t.z, own.f[4 * i + 2], st);
      st = mfma32_f32(t.w, own.f[4 * i + 3], st);
    }
  }
  __device__ __forceinline__ void accum(f32x16 (&acc)[DHM / 32], const E* tile, int kb, const f32x16& p) const {
    (void)kb;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int db = 0; db < DHM / 32; ++db)
        acc[db] = mfma32_f32(tile[perm_pos(r, half) * P + db * 32 + col], p[r], acc[db]);
  }
  static __device__ __forceinline__ void rotate_back(f32x16 (&)[DHM / 32], const float2*, int, int) {}
  static __device__ __forceinline__ void store(const f32x16 (&acc)[DHM / 32], float scale, int lane, E* stage, E* dst,
                                               long ld, bool, int n, int dh) {
    const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int db = 0; db < DHM / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = acc[db][4 * g + q] * scale;
        St<float>::st4(stage + l32 * P, db * 32 + 8 * g + 4 * half, v);
      }
    for (int r = 0; r < min(n, 32); ++r)
#pragma unroll
      for (int c = 0; c < DHM; c += 64)
        if (c + lane < dh) dst[r * ld + c + lane] = stage[r * P + c + lane];
  }
};

// ================================================================ the bias
// The bias of one head by relative position, times log2 e, from -R to R.  Beyond R it
// is constant, so a block past it reads one value.
// All NT threads go through the loop together, the last ones on the last entry: after a loop that
// lanes leave one by one, the compiler has been seen to save a register (to an accumulation
// register, the scalar ones being spilled there too) before it restored the execution mask.
template <int NT>
__device__ __forceinline__ void load_bias(const MaskedAttnArgs& a, int h, float* dst) {
  const int W = 2 * a.R + 1;
  for (int i0 = 0; i0 < W; i0 += NT) {
    const int i = min(i0 + (int)threadIdx.x, W - 1);
    const int t = min(max(a.bucket[i], 0), a.nb - 1);
    const float v = a.table[(long)t * a.H + h];
    dst[i] = v <= kHidden ? -INFINITY : v * kLog2e;
  }
}
// x = st * sl2 + bias for a block whose register r has relative position rel0 + sgn * perm_pos(r)
// in this lane; relmin .. relmax over the wave's block
template <int SGN>
__device__ __forceinline__ void add_bias(f32x16& st, float sl2, const float* bias, int R, int rel0, int relmin,
                                         int relmax, int half) {
  if (relmin >= R || relmax <= -R) {
    const float b = bias[relmin >= R ? 2 * R : 0];
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = fmaf(st[r], sl2, b);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int rel = rel0 + SGN * perm_pos(r, half);
      st[r] = fmaf(st[r], sl2, bias[min(max(rel, -R), R) + R]);
    }
  }
}

// x shifted by N lanes within rows of 16, zeros coming in: lane i gets lane i + N (N > 0) or i - |N|
template <int N>
__device__ __forceinline__ float row_shift(float x) {
  if constexpr (N == 0) return x;
  constexpr int ctrl = N > 0 ? 0x100 + N : 0x110 - N;
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xf, 0xf, true));
}
// adds register R's part of a block to the diagonals v[j] (add_diag below)
template <int R>
__device__ __forceinline__ void diag_part(const f32x16& ds, float (&v)[3]) {
  if constexpr (R < 16) {
    constexpr int kap = 8 * ((R >> 2) & 1) + (R & 3), k16 = R >> 3;
    v[k16] += row_shift<kap>(ds[R]);
    if constexpr (kap > 0) v[k16 + 1] += row_shift<kap - 16>(ds[R]);
    diag_part<R + 1>(ds, v);
  }
}
// Sums of a 32 x 32 block of dS (lane = query, register = key) along its diagonals, added to
// the wave's own array diag[rel + R]; what is at or beyond +-R goes to this lane's hi / lo.  Register
// r holds key k = 16 k16 + kap + 4 half, so shifting it by kap lanes puts the values of
// one q - k = c + 16 (lane / 16 % 2 - k16) - 4 half on one lane c of each row of 16, and
// what a row's end cuts off, shifted the other way, those 16 further: 30 additions give each
// lane three diagonals' sums, one exchange across 16 lanes two, which no other lane of
// its half shares.  The halves then add one after the other; a wave's LDS operations run in
// order, so the sums' order is fixed.
__device__ __forceinline__ void add_diag(const f32x16& ds, int base, int R, float* diag, float& lo, float& hi,
                                         int lane) {
  if (base - 31 >= R || base + 31 <= -R) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += ds[r];
    if (base > 0) hi += s;
    else lo += s;
    return;
  }
  float v[3] = {0.f, 0.f, 0.f};
  diag_part<0>(ds, v);
  // q - k + 4 half: v[0] lane, v[1] lane - 16, v[2] lane - 32
  const int half = lane >> 5, l32 = lane & 31;
  const float x = __shfl_xor(v[1], 16, 64);
  const float sum[2] = {v[0] + (l32 < 16 ? x : 0.f), v[2] + (l32 < 16 ? 0.f : x)};
  const int rel[2] = {base - l32 + 4 * half, base - l32 + 4 * half + 32};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (rel[j] >= R) hi += sum[j];
    else if (rel[j] <= -R) lo += sum[j];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (half == h) {
      float old[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) old[j] = abs(rel[j]) < R ? diag[rel[j] + R] : 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (abs(rel[j]) < R) diag[rel[j] + R] = old[j] + sum[j];
    }
    // to one lane the two steps are alternatives: nothing but this keeps them apart
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

// Rows that see nothing, or lie past the lengths, are zeros whatever the others hold: their products with
// weights of zero are NaN where a tile has infinities.
template <int N>
__device__ __forceinline__ void clear_if(bool dead, f32x16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = dead ? 0.f : acc[i][r];
}

// ================================================================ forward
// The running maximum (base 2) moves only when some row's new one is more than 8 above it:
// until then P is at most 2^8, which costs fp32 sums and bf16 products nothing, and the
// wave keeps its sums as they are.
template <int N>
__device__ __forceinline__ void move_max(float& mrun, float& lrun, f32x16 (&oacc)[N], float mx) {
  if (__any(mx > mrun + 8.f)) {
    const float mnew = fmaxf(mrun, mx);
    const float alpha = mnew == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mrun - mnew);
    mrun = mnew;
    lrun *= alpha;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[d][r] *= alpha;
  }
}

// One workgroup per 128 queries of a head, 32 per wave; the four share the key tiles.  Bound by
// issue: at 32 heads on 8 of 128, 8192 causal tokens, window 1024, 200 us (0.43 of the matrix rate of
// a large product): matrix unit 35 %, vector unit 40 % busy with two waves per SIMD, which meet in the
// same phase about as often as not; exponentials take half as long as the products.  LDS is 20 % busy,
// and more fragments read ahead change nothing.
template <class O, bool BIAS, int NW>
__global__ __launch_bounds__(64 * NW, O::WAVES) void attn_masked_fwd(MaskedAttnArgs a) {
  typedef typename O::E E;
  constexpr int DH = O::DH, KR = O::KR, TILE = O::TILE;
  constexpr int ST = O::ST, PER = 2 * O::BLOCK_DMAS(KR) / NW;
  __shared__ __attribute__((aligned(1024))) E sm[ST * 2 * TILE];  // [stage][K, V]
  extern __shared__ float sbias[];
  static_assert(ST * 2 * TILE >= NW * O::STAGE, "the O rows fit the tiles' space");
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // what a wave skips, it skips whole
  const int nq = (a.Sq + 32 * NW - 1) / (32 * NW);
  int qb, bh;
  heavy_first(blockIdx.x, nq, a.B * a.H, qb, bh);
  qb = nq - 1 - qb;
  const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hkv);
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const int qw0 = qb * 32 * NW, q0 = qw0 + wave * 32, q = q0 + l32, p = sq.off + q;
  const bool qv = q < sq.lq;
  const int plo = sq.off + q0, phi = sq.off + min(q0 + 31, sq.lq - 1);
  const Span span = key_span(mask, plo, phi);
  const Visible seen = keys_of(mask, p);
  KeyTiles kt{0, 0, 0};
  if (qw0 < sq.lq) kt = key_tiles<KR>(mask, sq.off + qw0, sq.off + min(qw0 + 32 * NW, sq.lq) - 1);
  const float sl2 = kLog2e * a.scale;
  const E* K = static_cast<const E*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const E* V = static_cast<const E*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const O ops(lane, a.dh);
  const uint32_t kfirst = O::template dma_first<NW>(a.k.t, a.dh, lane, wave);
  const uint32_t vfirst = O::template dma_first<NW>(a.v.t, a.dh, lane, wave);
  auto issue = [&](int i) {
    const int k0 = kt.at(i) * KR, last = sq.lk - 1 - k0;
    E* dst = sm + (i % ST) * 2 * TILE;
    O::template dma<NW>(K + (long)k0 * a.k.t, a.k.t, last, dst, a.dh, lane, wave, kfirst);
    O::template dma<NW>(V + (long)k0 * a.v.t, a.v.t, last, dst + TILE, a.dh, lane, wave, vfirst);
  };
  for (int i = 0; i < min(ST - 1, kt.n); ++i) issue(i);
  typename O::Rows qf;
  O::load_rows(qf, static_cast<const E*>(a.q.p) + b * a.q.b + (long)(qv ? q : 0) * a.q.t + h * a.q.h, qv, half, a.dh);
  if (BIAS) load_bias<64 * NW>(a, h, sbias);

  f32x16 oacc[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float mrun = -INFINITY, lrun = 0.f;

  qf.settled();
  for (int i = 0; i < kt.n; ++i) {
    tile_ready<ST, PER>(i, kt.n);
    if (i + ST - 1 < kt.n) issue(i + ST - 1);
    const int k0 = kt.at(i) * KR;
    if (q0 >= sq.lq) continue;  // wave-uniform, as all of this
    int most = 0, least = 2;
#pragma unroll
    for (int kb = 0; kb < KR / 32; ++kb) {
      const int kind = span.kind(k0 / 32 + kb);
      most = max(most, kind);
      least = min(least, kind);
    }
    if (most == 0) continue;
    const E* sK = sm + (i % ST) * 2 * TILE;
    const E* sV = sK + TILE;
    f32x16 sc[KR / 32];
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KR / 32; ++kb) {
      ops.scores(sc[kb], sK, kb, qf);
      if (BIAS || kb == KR / 32 - 1) landed<O::LANDS>(sc[kb]);
      if (BIAS)
        add_bias<1>(sc[kb], sl2, sbias, a.R, k0 + kb * 32 - p, k0 + kb * 32 - phi, k0 + kb * 32 + 31 - plo, half);
    }
    if (least < 2) {
#pragma unroll
      for (int kb = 0; kb < KR / 32; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sc[kb][r] = seen.has(k0 + kb * 32 + perm_pos(r, half)) ? sc[kb][r] : -INFINITY;
    }
#pragma unroll
    for (int kb = 0; kb < KR / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[kb][r]);
    // without a bias the scale (positive) is folded into the exponent's FMA
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * (BIAS ? 1.f : sl2);
    move_max(mrun, lrun, oacc, mx);
    const float mfin = mrun == -INFINITY ? 0.f : mrun;  // nothing visible yet: exp2(-inf - 0) = 0
    float rs = 0.f;
#pragma unroll
    for (int kb = 0; kb < KR / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[kb][r] = __builtin_amdgcn_exp2f(BIAS ? sc[kb][r] - mfin : fmaf(sc[kb][r], sl2, -mfin));
        rs += sc[kb][r];
      }
    lrun += rs + __shfl_xor(rs, 32, 64);
#pragma unroll
    for (int kb = 0; kb < KR / 32; ++kb) ops.accum(oacc, sV, kb, sc[kb]);
  }
  tiles_ready();  // the tiles' space now takes the O rows
  if (q0 >= a.Sq) return;
  const bool sees = qv && lrun != 0.f;  // a sum that is NaN stays one
  const float inv = 1.f / (sees ? lrun : 1.f);
  clear_if(!sees, oacc);
  O::store(oacc, inv, lane, sm + wave * O::STAGE,
           static_cast<E*>(a.o.p) + b * a.o.b + (long)q0 * a.o.t + h * a.o.h, a.o.t,
           stream_out((long)a.B * a.Sq * a.H * DH * (long)sizeof(E)), a.Sq - q0, a.dh);
  if (a.lse && q < a.Sq && half == 0)
    a.lse[(long)bh * a.Sq + q] = sees ? mrun + log2f(lrun) : -INFINITY;
}

// ================================================================ a few queries, many keys
// Bound by the bytes of the visible keys and values.  The queries of a key-value head (every token
// of every query head of its group) are the 32 rows of one score block, so its keys
// are read once for all of them; the keys are dealt to workgroups, and inside one, tile by
// tile, to waves that run on their own: tiles of 32 keys that only their wave reads, two deep
// by DMA, no barrier.  The waves' (maximum, sum, O) are joined in LDS, the workgroups' by
// attn_few_join.
// Now: 4 x 32 heads on 8 of 128, window 32768: 86 us (5.3 TB/s) and 5 for the join; 32 heads, window
// 1024: 10 and 4.  Before (attn_masked_fwd, no split): 876 and 29 us.
struct FewWork {
  int split, rb;  // workgroups over the keys, blocks of 32 rows
};
// the rest of a table's bias for one lane: constant beyond +-R
struct LaneBias {
  float lo, hi;
  static __device__ __forceinline__ float at(const MaskedAttnArgs& a, int i, int h) {
    const float v = a.table[(long)min(max(a.bucket[i], 0), a.nb - 1) * a.H + h];
    return v <= kHidden ? -INFINITY : v * kLog2e;
  }
};

template <class O, bool BIAS, int NW>
__global__ __launch_bounds__(64 * NW, 1) void attn_few_fwd(MaskedAttnArgs a, FewWork w) {
  typedef typename O::E E;
  constexpr int DH = O::DH, BLOCK = O::BLOCK;
  __shared__ __attribute__((aligned(1024))) E sm[NW][4 * BLOCK];  // per wave: [buffer][K, V]; later its O
  __shared__ float sM[NW][32], sS[NW][32];
  static_assert(4 * BLOCK * sizeof(E) >= 32 * DH * 4, "a wave's O fits its tiles' space");
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blk = xcd_block(blockIdx.x, gridDim.x), rb = blk % w.rb, split = blk / w.rb % w.split, bh = blk / w.rb / w.split;
  const int grp = a.H / a.Hkv, b = bh / a.Hkv, hk = bh % a.Hkv;
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const int row = rb * 32 + l32, tok = row / grp, h = hk * grp + row % grp, p = sq.off + tok;
  const bool qv = tok < sq.lq;
  const int tok0 = rb * 32 / grp, plo = sq.off + tok0, phi = sq.off + min((rb * 32 + 31) / grp, sq.lq - 1);
  const Span span = key_span(mask, plo, phi);
  const Visible seen = keys_of(mask, p);
  KeyTiles kt{0, 0, 0};
  if (tok0 < sq.lq) kt = key_tiles<32>(mask, plo, phi);
  const int per = (kt.n + w.split - 1) / w.split, i1 = min(kt.n, (split + 1) * per);
  const float sl2 = kLog2e * a.scale;
  const E* K = static_cast<const E*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const E* V = static_cast<const E*>(a.v.p) + b * a.v.b + hk * a.v.h;
  O ops(lane, a.dh);
  E* tiles = sm[wave];
  auto issue = [&](int i, int buf) {
    const int k0 = kt.at(i) * 32, last = sq.lk - 1 - k0;
    E* dst = tiles + buf * 2 * BLOCK;
    O::dma_block(K + (long)k0 * a.k.t, a.k.t, last, dst, a.dh, lane);
    O::dma_block(V + (long)k0 * a.v.t, a.v.t, last, dst + BLOCK, a.dh, lane);
  };
  int i = split * per + wave;
  if (i < i1) issue(i, 0);
  typename O::Rows qf;
  O::load_rows(qf, static_cast<const E*>(a.q.p) + b * a.q.b + (long)(qv ? tok : 0) * a.q.t + h * a.q.h, qv, half, a.dh);
  LaneBias lb{0.f, 0.f};
  if (BIAS) lb = LaneBias{LaneBias::at(a, 0, h), LaneBias::at(a, 2 * a.R, h)};

  f32x16 oacc[DH / 32];
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[d][r] = 0.f;
  float mrun = -INFINITY, lrun = 0.f;
  qf.settled();
  if (BIAS) {
    settle(lb.lo);
    settle(lb.hi);
  }
  for (int buf = 0; i < i1; i += NW, buf ^= 1) {
    // the other buffer's reads have ended; its next tile is under way while this one is waited for,
    // where the counter of loads in flight (63 at most) can tell the two apart
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if constexpr (2 * O::DMAS <= 32) {
      if (i + NW < i1) {
        issue(i + NW, buf ^ 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * O::DMAS) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (i + NW < i1) issue(i + NW, buf ^ 1);
    }
    const int k0 = kt.at(i) * 32, kind = span.kind(k0 / 32);
    if (kind == 0) continue;
    const E* sK = tiles + buf * 2 * BLOCK;
    f32x16 sc;
    ops.scores(sc, sK, 0, qf);
    landed<O::LANDS>(sc);
    if (BIAS) {
      if (k0 - phi >= a.R || k0 + 31 - plo <= -a.R) {
        const float c = k0 - phi >= a.R ? lb.hi : lb.lo;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = fmaf(sc[r], sl2, c);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int rel = k0 + perm_pos(r, half) - p;
          sc[r] = fmaf(sc[r], sl2, LaneBias::at(a, min(max(rel, -a.R), a.R) + a.R, h));
        }
      }
    }
    if (kind == 1) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = seen.has(k0 + perm_pos(r, half)) ? sc[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * (BIAS ? 1.f : sl2);
    move_max(mrun, lrun, oacc, mx);
    const float mfin = mrun == -INFINITY ? 0.f : mrun;
    float rs = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(BIAS ? sc[r] - mfin : fmaf(sc[r], sl2, -mfin));
      rs += sc[r];
    }
    lrun += rs + __shfl_xor(rs, 32, 64);
    ops.accum(oacc, sK + BLOCK, 0, sc);
  }

  // join the waves: O in the accumulators' own order
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  float4* so = reinterpret_cast<float4*>(tiles) + lane;
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      so[(d * 4 + g) * 64] = make_float4(oacc[d][4 * g], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]);
  if (half == 0) {
    sM[wave][l32] = mrun;
    sS[wave][l32] = lrun;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f, f[NW];
#pragma unroll
  for (int k = 0; k < NW; ++k) M = qv ? fmaxf(M, sM[k][l32]) : -INFINITY;
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    f[k] = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sM[k][l32] - M);
    L = fmaf(sS[k][l32], f[k], L);
  }
  if (tok >= a.Sq) return;
  if (!qv) L = 0.f;
  const float inv = 1.f / L;
  float* po = a.part + ((long)blk * 32 + l32) * DH;
  E* o = static_cast<E*>(a.o.p) + b * a.o.b + (long)tok * a.o.t + h * a.o.h;
  for (int d = wave; d < DH / 32; d += NW)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float4 x = reinterpret_cast<const float4*>(sm[k])[(d * 4 + g) * 64 + lane];
        v[0] = fmaf(x.x, f[k], v[0]);
        v[1] = fmaf(x.y, f[k], v[1]);
        v[2] = fmaf(x.z, f[k], v[2]);
        v[3] = fmaf(x.w, f[k], v[3]);
      }
      const int c = d * 32 + 8 * g + 4 * half;
      if (w.split > 1) {
        St<float>::st4(po, c, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.dh) St<E>::st(o, c + e, L != 0.f ? v[e] * inv : 0.f);
      }
    }
  if (wave == 0 && half == 0) {
    if (w.split > 1) reinterpret_cast<float2*>(a.part + (long)gridDim.x * 32 * DH)[(long)blk * 32 + l32] = make_float2(M, L);
    else if (a.lse) a.lse[((long)b * a.H + h) * a.Sq + tok] = L != 0.f ? M + log2f(L) : -INFINITY;
  }
}

// joins a row's partial results (at most 64) in order; one wave per row
template <class O>
__global__ __launch_bounds__(256) void attn_few_join(MaskedAttnArgs a, FewWork w) {
  typedef typename O::E E;
  constexpr int DH = O::DH;
  const int lane = threadIdx.x & 63, grp = a.H / a.Hkv, rows = a.Sq * grp;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (long)a.B * a.Hkv * rows) return;
  const int bh = (int)(id / rows), row = (int)(id % rows), b = bh / a.Hkv, hk = bh % a.Hkv;
  const long blk0 = ((long)bh * w.split) * w.rb + row / 32, n = (long)a.B * a.Hkv * w.split * w.rb;
  const float2 ml = lane < w.split ? reinterpret_cast<const float2*>(a.part + n * 32 * DH)[(blk0 + (long)lane * w.rb) * 32 + row % 32]
                                   : make_float2(-INFINITY, 0.f);
  const float M = wave_max(ml.x), f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M), L = wave_sum(ml.y * f);
  float acc[DH / 64];
#pragma unroll
  for (int d = 0; d < DH / 64; ++d) acc[d] = 0.f;
  for (int s0 = 0; s0 < w.split; s0 += 8) {  // eight loads in flight; past the last one with weight 0
    float v[8][DH / 64], fs[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = min(s0 + k, w.split - 1);
      const float* src = a.part + ((blk0 + (long)s * w.rb) * 32 + row % 32) * DH + lane;
#pragma unroll
      for (int d = 0; d < DH / 64; ++d) v[k][d] = src[64 * d];
      fs[k] = s0 + k < w.split ? __shfl(f, s, 64) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int d = 0; d < DH / 64; ++d) acc[d] = fmaf(v[k][d], fs[k], acc[d]);
  }
  const int tok = row / grp, h = hk * grp + row % grp;
  E* o = static_cast<E*>(a.o.p) + b * a.o.b + (long)tok * a.o.t + h * a.o.h;
#pragma unroll
  for (int d = 0; d < DH / 64; ++d)
    if (lane + 64 * d < a.dh) St<E>::st(o, lane + 64 * d, L != 0.f ? acc[d] / L : 0.f);
  if (a.lse && lane == 0) a.lse[((long)b * a.H + h) * a.Sq + tok] = L != 0.f ? M + log2f(L) : -INFINITY;
}

// ================================================================ backward
// exponent offset of a row that sees nothing: exp2(x - inf) = 0
__device__ __forceinline__ float lse_or_inf(float l) { return l == -INFINITY ? INFINITY : l; }

// An lse is off by half its last digit, and P = exp2(x - lse) by that factor: 2^-18 at 128, but with entries of
// -1e9 in all that a row sees its whole logarithm of the sum is lost, and P no longer sums to one.  Where a block
// of 32 rows has one beyond 128 the passes divide by the sum of P; elsewhere that is a test and a branch (dK/dV
// with the bias, bf16 64: 2 %).  Without a bias x is q.k, whose own products' rounding is as much.
__device__ __forceinline__ bool is_far(float lse) { return fabsf(lse) > 128.f && fabsf(lse) < INFINITY; }
__device__ __forceinline__ float inv_sum(float sum) { return sum > 0.f ? 1.f / sum : 1.f; }
__device__ __forceinline__ float sum16(const f32x16& p) {
  float s = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) s += p[r];
  return s;
}
template <int N>
__device__ __forceinline__ void scale_by(float f, f32x16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] *= f;
}

// st = P and dp = dP of a block (lane = query, registers = keys k0 ..) against tiles of K and V
template <class O, bool BIAS>
__device__ __forceinline__ void p_and_dp(const O& ops, f32x16& st, f32x16& dp, const typename O::E* sK,
                                         const typename O::E* sV, int kb, const typename O::Rows& qf,
                                         const typename O::Rows& df, float sl2, const float* bias, int R, int k0, int p,
                                         int plo, int phi, bool whole, const Visible& seen, float lse, int half) {
  ops.scores(st, sK, kb, qf);
  ops.scores(dp, sV, kb, df);
  landed<O::LANDS>(st);
  landed<O::LANDS>(dp);
  if (BIAS) add_bias<1>(st, sl2, bias, R, k0 - p, k0 - phi, k0 + 31 - plo, half);
  if (!whole) {  // a row past len_q has lse = +inf
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = seen.has(k0 + perm_pos(r, half)) ? st[r] : -INFINITY;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) st[r] = __builtin_amdgcn_exp2f(BIAS ? st[r] - lse : fmaf(st[r], sl2, -lse));
}
// st = P and dp = dS of a block (lane = key, registers = query rows q0 ..) against tiles of Q and
// dO; stat: (lse, D) of those rows; inv(i): one over row q0 + i's sum of P, where one of the 32 is_far
template <class O, bool BIAS, class Inv>
__device__ __forceinline__ void p_and_ds(const O& ops, f32x16& st, f32x16& dp, const typename O::E* sQ,
                                         const typename O::E* sO, int qb, const typename O::Rows& kf,
                                         const typename O::Rows& vf, float sl2, const float* bias, int R, int q0, int off,
                                         int key, int k0, bool whole, const Visible& seen, const float2* stat, int half,
                                         const Inv& inv) {
  ops.scores(st, sQ, qb, kf);
  ops.scores(dp, sO, qb, vf);
  landed<O::LANDS>(st);
  landed<O::LANDS>(dp);
  if (BIAS) {
    const int plo = off + q0;
    add_bias<-1>(st, sl2, bias, R, key - plo, k0 - plo - 31, k0 + 31 - plo, half);
  }
  if (!whole) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      st[r] = (unsigned)(q0 + perm_pos(r, half) - seen.lo) <= seen.n1 ? st[r] : -INFINITY;
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {  // queries q0 + 8g + 4*half + 0..3
    const float4* ld = reinterpret_cast<const float4*>(stat + 8 * g + 4 * half);
    const float4 x = ld[0], y = ld[1];
    const float lv[4] = {x.x, x.z, y.x, y.z}, sv[4] = {x.y, x.w, y.y, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * g + e;
      st[r] = __builtin_amdgcn_exp2f(BIAS ? st[r] - lv[e] : fmaf(st[r], sl2, -lv[e]));
      dp[r] = st[r] * (dp[r] - sv[e]);
    }
  }
  if (BIAS && __any(is_far(stat[threadIdx.x & 31].x))) {
    const int own = __float_as_int(inv(threadIdx.x & 31));  // handed round by lane: registers are scarce here
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int f0 = __builtin_amdgcn_readlane(own, perm_pos(r, 0)), f1 = __builtin_amdgcn_readlane(own, perm_pos(r, 1));
      const float f = __int_as_float(half ? f1 : f0);
      st[r] *= f;
      dp[r] *= f;
    }
  }
}
// a workgroup's sums along the diagonals leave as one row of the workspace: the waves' arrays
// follow the bias in LDS, what lay beyond +-R is in the lanes' lo and hi
__device__ __forceinline__ void close_diag(float* diag, int W, float lo, float hi, int lane) {
  lo = wave_sum(lo);
  hi = wave_sum(hi);
  if (lane == 0) {
    diag[0] += lo;
    diag[W - 1] += hi;
  }
}
template <int NW>
__device__ __forceinline__ void put_diag(const float* sbias, int W, float* out) {
  for (int i0 = 0; i0 < W; i0 += 64 * NW) {  // all threads, as in load_bias
    const int i = min(i0 + (int)threadIdx.x, W - 1);
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += sbias[(1 + w) * W + i];
    out[i] = s;
  }
}

// dQ pass (lane = query); writes (lse, D).  DTAB: dtable is wanted, and D is formed from
// P and dP themselves in a first sweep over the tiles: the sums over dS cancel, and a D
// from the stored (rounded) O would leave an error of that rounding in them.  That sweep
// is two of the pass's five products.  Bound by issue, as the forward: 8192 tokens, window 1024
// 255 us, matrix unit 39 %, vector unit 34 % busy; with the table's gradient (1777 tokens, 2 x 16 heads,
// window 500) 81 us.  The two sweeps are two loops, so that dQ holds no registers in the first: as one loop
// with a flag 45 registers spilled and the same took 109.
template <class O, bool BIAS, bool DTAB, int NW>
__global__ __launch_bounds__(64 * NW, O::WAVES) void attn_masked_bwd_dq(MaskedAttnArgs a) {
  typedef typename O::E E;
  constexpr int DH = O::DH, KR = O::KR, TILE = O::TILE;
  constexpr int ST = O::ST, PER = 2 * O::BLOCK_DMAS(KR) / NW;
  __shared__ __attribute__((aligned(1024))) E sm[ST * 2 * TILE];  // [stage][K, V]
  extern __shared__ float sbias[];                                // bias, then (DTAB) one diagonal array per wave
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // what a wave skips, it skips whole
  const int nq = (a.Sq + 32 * NW - 1) / (32 * NW);
  int qb, bh;
  heavy_first(blockIdx.x, nq, a.B * a.H, qb, bh);
  qb = nq - 1 - qb;
  const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hkv);
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const int qw0 = qb * 32 * NW, q0 = qw0 + wave * 32, q = q0 + l32, p = sq.off + q;
  const bool qv = q < sq.lq;
  const int plo = sq.off + q0, phi = sq.off + min(q0 + 31, sq.lq - 1);
  const Span span = key_span(mask, plo, phi);
  const Visible seen = keys_of(mask, p);
  KeyTiles kt{0, 0, 0};
  if (qw0 < sq.lq) kt = key_tiles<KR>(mask, sq.off + qw0, sq.off + min(qw0 + 32 * NW, sq.lq) - 1);
  const float sl2 = kLog2e * a.scale;
  const E* K = static_cast<const E*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const E* V = static_cast<const E*>(a.v.p) + b * a.v.b + hk * a.v.h;
  O ops(lane, a.dh);
  const int nit = DTAB ? 2 * kt.n : kt.n;  // DTAB: the tiles twice
  const uint32_t kfirst = O::template dma_first<NW>(a.k.t, a.dh, lane, wave);
  const uint32_t vfirst = O::template dma_first<NW>(a.v.t, a.dh, lane, wave);
  auto issue = [&](int i) __attribute__((always_inline)) {
    const int k0 = kt.at(DTAB && i >= kt.n ? i - kt.n : i) * KR, last = sq.lk - 1 - k0;
    E* dst = sm + (i % ST) * 2 * TILE;
    O::template dma<NW>(K + (long)k0 * a.k.t, a.k.t, last, dst, a.dh, lane, wave, kfirst);
    O::template dma<NW>(V + (long)k0 * a.v.t, a.v.t, last, dst + TILE, a.dh, lane, wave, vfirst);
  };
  for (int i = 0; i < min(ST - 1, nit); ++i) issue(i);
  const long row = qv ? q : 0;
  typename O::Rows qf, df;
  O::load_rows(qf, static_cast<const E*>(a.q.p) + b * a.q.b + row * a.q.t + h * a.q.h, qv, half, a.dh);
  O::load_rows(df, static_cast<const E*>(a.dout.p) + b * a.dout.b + row * a.dout.t + h * a.dout.h, qv, half, a.dh);
  float dsum = 0.f;
  if (!DTAB) {
    typename O::Rows of;
    O::load_rows(of, static_cast<const E*>(a.o.p) + b * a.o.b + row * a.o.t + h * a.o.h, qv, half, a.dh);
    dsum = O::dot(of, df);
  }
  float lse = qv ? lse_or_inf(a.lse[(long)bh * a.Sq + row]) : INFINITY;
  const int W = 2 * a.R + 1;
  float* diag = sbias + (1 + wave) * W;
  if (BIAS) load_bias<64 * NW>(a, h, sbias);
  if (DTAB)
    for (int i = 0; i < W; i += 64) diag[min(i + lane, W - 1)] = 0.f;  // all lanes, as in load_bias
  float dlo = 0.f, dhi = 0.f;

  qf.settled();
  df.settled();
  settle(lse);
  settle(dsum);
  const bool far = BIAS && __any(is_far(lse));
  float psum = 0.f, inv = 1.f;
  f32x16 dq[DH / 32];
  // the key tiles once, as iterations from .. of the pipeline; first: for D alone
  auto sweep = [&](auto first, int from) __attribute__((always_inline)) {
    for (int t = 0; t < kt.n; ++t) {
      const int i = from + t;
      tile_ready<ST, PER>(i, nit);
      if (i + ST - 1 < nit) issue(i + ST - 1);
      if (q0 >= sq.lq) continue;
      const E* sK = sm + (i % ST) * 2 * TILE;
      const E* sV = sK + TILE;
      // one key block at a time (not unrolled): keeps the kernel within its registers
#pragma unroll 1
      for (int kb = 0; kb < KR / 32; ++kb) {
        const int k0 = kt.at(t) * KR + kb * 32;
        const int kind = span.kind(k0 / 32);
        if (kind == 0) continue;  // wave-uniform
        ops.fresh();
        f32x16 st, dp;
        p_and_dp<O, BIAS>(ops, st, dp, sK, sV, kb, qf, df, sl2, sbias, a.R, k0, p, plo, phi, kind == 2, seen, lse, half);
        if constexpr (first) {
#pragma unroll
          for (int r = 0; r < 16; ++r) dsum = fmaf(st[r], dp[r], dsum);
          if (far) psum += sum16(st);
        } else {
          if (far) {
            if (DTAB)
#pragma unroll
              for (int r = 0; r < 16; ++r) st[r] *= inv;
            else psum += sum16(st);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) st[r] *= dp[r] - dsum;  // dS
          if (DTAB) add_diag(st, k0 - sq.off - q0, a.R, diag, dlo, dhi, lane);
          ops.accum(dq, sK, kb, st);
        }
      }
    }
  };
  if constexpr (DTAB) {
    sweep(std::true_type{}, 0);
    dsum += __shfl_xor(dsum, 32, 64);
    if (far) {
      inv = inv_sum(psum + __shfl_xor(psum, 32, 64));
      dsum *= inv;
    }
  }
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[i][r] = 0.f;
  sweep(std::false_type{}, DTAB ? __builtin_amdgcn_readfirstlane(kt.n) : 0);
  const bool dead = lse == INFINITY;  // nothing visible, or past the length
  if (dead) dsum = 0.f;
  clear_if(dead, dq);
  if (far) {
    if (!DTAB) {
      inv = inv_sum(psum + __shfl_xor(psum, 32, 64));
      scale_by(inv, dq);
    }
    if (q < a.Sq && half == 0) a.inv[(long)bh * a.Sq + q] = inv;
  }
  // the row statistics that the dK/dV pass reads
  if (q < a.Sq && half == 0) a.stat[(long)bh * a.Sq + q] = make_float2(lse, dsum);
  if (DTAB) close_diag(diag, W, dlo, dhi, lane);
  tiles_ready();  // the tiles' space now takes the dQ rows
  if (DTAB) put_diag<NW>(sbias, W, a.diag + ((long)(b * nq + qb) * a.H + h) * W);
  if (q0 >= a.Sq) return;
  O::rotate_back(dq, a.rope_tab, min(q, a.Sq - 1), half);
  O::store(dq, a.scale, lane, sm + wave * O::STAGE,
           static_cast<E*>(a.dq.p) + b * a.dq.b + (long)q0 * a.dq.t + h * a.dq.h, a.dq.t,
           stream_out((long)a.B * a.Sq * a.H * DH * (long)sizeof(E)), a.Sq - q0, a.dh);
}

// The same for calls whose 32-row blocks would hold fewer than half of the SIMDs: a workgroup takes one of
// them, and its waves every fourth (second) block of its keys each, from tiles of their own as
// in attn_few_fwd; D and dQ are joined in LDS.  4 heads on 2 of 128, 1824 tokens, with the
// table's gradient: 69 us, 147 with one wave per block.
template <class O, bool BIAS, bool DTAB, int NW>
__global__ __launch_bounds__(64 * NW, 1) void attn_few_dq(MaskedAttnArgs a) {
  typedef typename O::E E;
  constexpr int DH = O::DH, BLOCK = O::BLOCK;
  __shared__ __attribute__((aligned(1024))) E sm[NW][4 * BLOCK];  // per wave: [buffer][K, V]; later its dQ
  __shared__ float sD[NW][32], sP[NW][32];
  extern __shared__ float sbias[];  // bias, then (DTAB) one diagonal array per wave
  static_assert(4 * BLOCK * sizeof(E) >= 32 * DH * 4 && 4 * BLOCK >= O::STAGE, "a wave's dQ fits its tiles' space");
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nq = (a.Sq + 31) / 32, blk = xcd_block(blockIdx.x, gridDim.x), qb = blk % nq, bh = blk / nq;
  const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hkv);
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const int q0 = qb * 32, q = q0 + l32, p = sq.off + q;
  const bool qv = q < sq.lq;
  const int plo = sq.off + q0, phi = sq.off + min(q0 + 31, sq.lq - 1);
  const Span span = key_span(mask, plo, phi);
  const Visible seen = keys_of(mask, p);
  KeyTiles kt{0, 0, 0};
  if (q0 < sq.lq) kt = key_tiles<32>(mask, plo, phi);
  const float sl2 = kLog2e * a.scale;
  const int W = 2 * a.R + 1;
  const E* K = static_cast<const E*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const E* V = static_cast<const E*>(a.v.p) + b * a.v.b + hk * a.v.h;
  O ops(lane, a.dh);
  E* tiles = sm[wave];
  auto issue = [&](int i, int buf) {
    const int k0 = kt.at(i) * 32, last = sq.lk - 1 - k0;
    E* dst = tiles + buf * 2 * BLOCK;
    O::dma_block(K + (long)k0 * a.k.t, a.k.t, last, dst, a.dh, lane);
    O::dma_block(V + (long)k0 * a.v.t, a.v.t, last, dst + BLOCK, a.dh, lane);
  };
  if (wave < kt.n) issue(wave, 0);
  const long row = qv ? q : 0;
  typename O::Rows qf, df;
  O::load_rows(qf, static_cast<const E*>(a.q.p) + b * a.q.b + row * a.q.t + h * a.q.h, qv, half, a.dh);
  O::load_rows(df, static_cast<const E*>(a.dout.p) + b * a.dout.b + row * a.dout.t + h * a.dout.h, qv, half, a.dh);
  float dsum = 0.f, dlo = 0.f, dhi = 0.f;
  if (!DTAB) {
    typename O::Rows of;
    O::load_rows(of, static_cast<const E*>(a.o.p) + b * a.o.b + row * a.o.t + h * a.o.h, qv, half, a.dh);
    dsum = O::dot(of, df);
  }
  float lse = qv ? lse_or_inf(a.lse[(long)bh * a.Sq + row]) : INFINITY;
  float* diag = sbias + (1 + wave) * W;
  if (BIAS) load_bias<64 * NW>(a, h, sbias);
  if (DTAB)
    for (int i = 0; i < W; i += 64) diag[min(i + lane, W - 1)] = 0.f;  // all lanes, as in load_bias
  f32x16 dq[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[i][r] = 0.f;
  qf.settled();
  df.settled();
  settle(lse);
  settle(dsum);
  const bool far = BIAS && __any(is_far(lse));  // of the workgroup: its waves have the same rows
  float psum = 0.f, inv = 1.f;
  auto join_psum = [&] {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) sum += sP[k][l32];
    inv = inv_sum(sum);
  };
  __syncthreads();  // the bias

#pragma unroll 1
  for (int sweep = DTAB ? 0 : 1; sweep < 2; ++sweep) {
#pragma unroll 1
    for (int i = wave, buf = 0; i < kt.n; i += NW, buf ^= 1) {
      // as in attn_few_fwd
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if constexpr (2 * O::DMAS <= 32) {
        if (i + NW < kt.n) {
          issue(i + NW, buf ^ 1);
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * O::DMAS) : "memory");
        } else {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (i + NW < kt.n) issue(i + NW, buf ^ 1);
      }
      const int k0 = kt.at(i) * 32, kind = span.kind(k0 / 32);
      if (kind == 0) continue;  // wave-uniform
      const E* sK = tiles + buf * 2 * BLOCK;
      f32x16 st, dp;
      p_and_dp<O, BIAS>(ops, st, dp, sK, sK + BLOCK, 0, qf, df, sl2, sbias, a.R, k0, p, plo, phi, kind == 2, seen, lse,
                        half);
      if (DTAB && sweep == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dsum = fmaf(st[r], dp[r], dsum);
        if (far) psum += sum16(st);
        continue;
      }
      if (far) {
        if (DTAB)
#pragma unroll
          for (int r = 0; r < 16; ++r) st[r] *= inv;
        else psum += sum16(st);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] *= dp[r] - dsum;  // dS
      if (DTAB) add_diag(st, k0 - plo, a.R, diag, dlo, dhi, lane);
      ops.accum(dq, sK, 0, st);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (DTAB && sweep == 0) {
      if (wave < kt.n) issue(wave, 0);
      dsum += __shfl_xor(dsum, 32, 64);
      psum += __shfl_xor(psum, 32, 64);
      if (half == 0) {
        sD[wave][l32] = dsum;
        sP[wave][l32] = psum;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      dsum = 0.f;
#pragma unroll
      for (int k = 0; k < NW; ++k) dsum += sD[k][l32];
      if (far) {
        join_psum();
        dsum *= inv;
      }
    }
  }
  const bool dead = lse == INFINITY;
  if (dead) dsum = 0.f;
  if (wave == 0 && half == 0 && q < a.Sq) a.stat[(long)bh * a.Sq + q] = make_float2(lse, dsum);
  if (DTAB) close_diag(diag, W, dlo, dhi, lane);
  if (!DTAB && far) {
    psum += __shfl_xor(psum, 32, 64);
    if (half == 0) sP[wave][l32] = psum;
  }
  float4* so = reinterpret_cast<float4*>(tiles) + lane;
  if (wave > 0) {
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        so[(d * 4 + g) * 64] = make_float4(dq[d][4 * g], dq[d][4 * g + 1], dq[d][4 * g + 2], dq[d][4 * g + 3]);
  }
  __syncthreads();
  if (DTAB) put_diag<NW>(sbias, W, a.diag + ((long)(b * nq + qb) * a.H + h) * W);
  if (wave > 0) return;
#pragma unroll
  for (int k = 1; k < NW; ++k)
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = reinterpret_cast<const float4*>(sm[k])[(d * 4 + g) * 64 + lane];
        dq[d][4 * g] += x.x;
        dq[d][4 * g + 1] += x.y;
        dq[d][4 * g + 2] += x.z;
        dq[d][4 * g + 3] += x.w;
      }
  clear_if(dead, dq);
  if (far) {
    if (!DTAB) {
      join_psum();
      scale_by(inv, dq);
    }
    if (q < a.Sq && half == 0) a.inv[(long)bh * a.Sq + q] = inv;
  }
  O::rotate_back(dq, a.rope_tab, min(q, a.Sq - 1), half);
  O::store(dq, a.scale, lane, sm[0], static_cast<E*>(a.dq.p) + b * a.dq.b + (long)q0 * a.dq.t + h * a.dq.h, a.dq.t, false,
           a.Sq - q0, a.dh);
}

// Work of the dK/dV pass.  A block of 32 NW keys meets the query tiles that see it, for every
// query head of its group: `iters` iterations at most.  Blocks that hold sinks (all of them
// without a window) are seen by every later query, so they are dealt to several
// workgroups each, and so are the others when there are too few of them to fill the GPU;
// such workgroups leave fp32 partial sums, which attn_masked_dkdv_join adds in order.
// 8192 causal tokens, 32 heads on 8, window 1024, 4 sinks: 353 us and 12 for the join; with one
// workgroup per block 3704 us.
struct KeyWork {
  int nk, nfar;       // key blocks, and how many of them (the first) are the sinks'
  int s_far, s_near;  // workgroups per block
  int c_far, c_near;  // iterations of each
  __host__ __device__ long items() const { return (long)nfar * s_far + (long)(nk - nfar) * s_near; }
  // the item that is dispatched n-th: the longer ones first, so that the others fill the gaps at the
  // end.  8192 tokens, window 1024, 4 sinks: 353 us, 390 us in order and in quarters (key_work)
  __device__ __forceinline__ int in_order(int n) const {
    const int near = (nk - nfar) * s_near;
    return c_far >= c_near ? n : n < near ? nfar * s_far + n : n - near;
  }
  // items that leave partial sums (far blocks are split at least as finely)
  __host__ __device__ long slots() const { return s_near > 1 ? items() : s_far > 1 ? (long)nfar * s_far : 0; }
};
struct KeyItem {
  int kb, split, n, c;  // block, which of its n workgroups, iterations of each
  __device__ __forceinline__ KeyItem(const KeyWork& w, int item) {
    const int far = w.nfar * w.s_far, t = item - far;
    const bool f = item < far;
    kb = f ? item / w.s_far : w.nfar + t / w.s_near;
    split = f ? item % w.s_far : t % w.s_near;
    n = f ? w.s_far : w.s_near;
    c = f ? w.c_far : w.c_near;
  }
};
// the query tiles of KR rows that see keys kw0 .. kw0 + nkeys - 1: the first, and how many
template <int KR>
__device__ __forceinline__ void query_tiles(const MaskedAttnArgs& a, const Seq& sq, int kw0, int nkeys, int& qt0,
                                            int& nt) {
  qt0 = nt = 0;
  if (kw0 >= sq.lk) return;
  const int kw1 = min(kw0 + nkeys, sq.lk) - 1;
  int qlo = 0, qhi = sq.lq - 1;
  if (a.causal) qlo = max(0, kw0 - sq.off);
  if (a.window && kw0 >= a.sinks) {
    qhi = min(qhi, kw1 + a.window - 1 - sq.off);
    if (!a.causal) qlo = max(0, kw0 - a.window + 1 - sq.off);
  }
  if (qhi < qlo) return;
  qt0 = qlo / KR;
  nt = qhi / KR - qt0 + 1;
}
// Whether the iterations i0 .. i1 - 1 (query tile i % nt, from qt0) touch any block of `span`: a wave
// without any leaves no partial sums, and the join reads none.
template <int KR>
__device__ __forceinline__ bool touches(const Span& span, int qt0, int nt, int i0, int i1) {
  const int t0 = span.v0 / (KR / 32) - qt0, t1 = (span.v1 >= 0 ? span.v1 / (KR / 32) : -1) - qt0;
  if (span.v1 < span.v0 || i1 <= i0) return false;
  const int a = i0 % nt, b = a + (i1 - i0) - 1;  // tiles a .. b, taken modulo nt
  return i1 - i0 >= nt || (t0 <= b && t1 >= a) || (b >= nt && t0 <= b - nt);
}
// item and batch-head of a workgroup: items in order of weight over all heads of an XCD
__device__ __forceinline__ void key_item(int lin, int items, int nbh, int& item, int& bh) {
  const int n = items * nbh, P = n / 8;
  if (n % 8 || P % items) {
    const int blk = xcd_block(lin, n);
    item = blk % items;
    bh = blk / items;
    return;
  }
  const int x = lin % 8, o = lin / 8, per = P / items;
  item = o / per;
  bh = x * per + o % per;
}

// dK/dV pass (lane = key): the query heads of the key's group one after another.  At head dim 128
// dK, dV and the own rows of K and V take 192 of 256 registers, so a fragment from LDS is waited for
// before the next is asked for: waves wait 57 % of the time, the matrix unit is 34 % busy.  With 512
// registers and one wave per SIMD: 460 us where this takes 390.  bf16, head dim
// 64, without a bias: held to 168 registers (169 otherwise), three waves fit a SIMD; 4 x 16 heads on 4
// of 2048 tokens, both passes: 188 us, 209 with two.
template <class O, bool BIAS, int NW>
__global__ __launch_bounds__(64 * NW, O::DH == 64 && O::KR == 64 && !BIAS ? 3 : O::WAVES) void attn_masked_bwd_dkdv(MaskedAttnArgs a, KeyWork w) {
  typedef typename O::E E;
  constexpr int DH = O::DH, KR = O::KR, TILE = O::TILE;
  constexpr int ST = O::ST, PER = 2 * O::BLOCK_DMAS(KR) / NW + 1;
  __shared__ __attribute__((aligned(1024))) E sm[ST * 2 * TILE];  // [stage][Q, dO]
  __shared__ __attribute__((aligned(1024))) float2 sS[ST][KR];   // (lse, D) of the tile's rows
  extern __shared__ float sbias[];  // two heads' bias
  static_assert(NW % (KR / 32) == 0, "32 rows' statistics per DMA");
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // what a wave skips, it skips whole
  const int grp = a.H / a.Hkv;
  int item, bh;
  key_item(blockIdx.x, (int)w.items(), a.B * a.Hkv, item, bh);
  item = w.in_order(item);
  const KeyItem ki(w, item);
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const int kw0 = ki.kb * 32 * NW, k0 = kw0 + wave * 32, key = k0 + l32;
  const bool kv = key < sq.lk;
  int qt0, nt;
  query_tiles<KR>(a, sq, kw0, 32 * NW, qt0, nt);
  const Span span = query_span(mask, k0, sq.off, sq.lq);
  const Visible seen = rows_of(mask, key, sq.off, sq.lq);
  const int i0 = ki.n > 1 ? ki.split * ki.c : 0, i1 = ki.n > 1 ? min(nt * grp, i0 + ki.c) : nt * grp;
  if (ki.n > 1 && i0 >= i1) return;  // the join counts the same way
  const float sl2 = kLog2e * a.scale;
  const int W = 2 * a.R + 1;
  O ops(lane, a.dh);
  int h = hk * grp, t = 0;  // head and query tile (of nt) that is issued next
  if (nt > 0) {
    h += i0 / nt;
    t = i0 % nt;
  }
  const uint32_t qfirst = O::template dma_first<NW>(a.q.t, a.dh, lane, wave);
  const uint32_t ofirst = O::template dma_first<NW>(a.dout.t, a.dh, lane, wave);
  // brings the tile of (h, t) into a stage and moves on to the next one
  int issued = i0;
  auto issue = [&]() {
    const int r0 = (qt0 + t) * KR, last = sq.lq - 1 - r0, stage = (issued - i0) % ST;
    E* dst = sm + stage * 2 * TILE;
    O::template dma<NW>(static_cast<const E*>(a.q.p) + b * a.q.b + h * a.q.h + (long)r0 * a.q.t, a.q.t, last, dst, a.dh,
                        lane, wave, qfirst);
    O::template dma<NW>(static_cast<const E*>(a.dout.p) + b * a.dout.b + h * a.dout.h + (long)r0 * a.dout.t, a.dout.t,
                        last, dst + TILE, a.dh, lane, wave, ofirst);
    // 32 rows per DMA; waves of the same remainder bring the same ones, so that every wave counts alike
    const int s0 = wave % (KR / 32) * 32;
    dma4_m0(uniform_ptr(a.stat + ((long)b * a.H + h) * a.Sq + r0), (uint32_t)(min(s0 + lane / 2, last) * 8 + lane % 2 * 4),
            lds_addr(sS[stage]) + s0 * 8);
    ++issued;
    if (++t == nt) {
      t = 0;
      ++h;
    }
  };
  while (issued < min(i1, i0 + ST - 1)) issue();
  // head and query tile of the iteration that is computed, and its bias
  int hc = hk * grp + (nt > 0 ? i0 / nt : 0), tc = nt > 0 ? i0 % nt : 0, hb = 0;
  if (BIAS && i0 < i1) load_bias<64 * NW>(a, hc, sbias);
  typename O::Rows kf, vf;
  const long row = kv ? key : 0;
  O::load_rows(kf, static_cast<const E*>(a.k.p) + b * a.k.b + row * a.k.t + hk * a.k.h, kv, half, a.dh);
  O::load_rows(vf, static_cast<const E*>(a.v.p) + b * a.v.b + row * a.v.t + hk * a.v.h, kv, half, a.dh);
  f32x16 dk[DH / 32], dv[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[i][r] = dv[i][r] = 0.f;

  kf.settled();
  vf.settled();
  for (int i = i0; i < i1; ++i) {
    const int stage = (i - i0) % ST, qt = qt0 + tc, hb_now = hb, h_now = hc;
    tile_ready<ST, PER>(i - i0, i1 - i0);
    if (issued < i1) issue();
    if (++tc == nt) {
      tc = 0;
      ++hc;
      hb ^= 1;
      // goes where the last head's was: read for the last time before this barrier
      if (BIAS && i + 1 < i1) load_bias<64 * NW>(a, hc, sbias + hb * W);
    }
    const E* sQ = sm + stage * 2 * TILE;
    const E* sO = sQ + TILE;
    const float* bias = sbias + hb_now * W;
#pragma unroll 1
    for (int qb = 0; qb < KR / 32; ++qb) {
      const int q0 = qt * KR + qb * 32;
      const int kind = span.kind(q0 / 32);
      if (kind == 0) continue;  // wave-uniform
      ops.fresh();
      f32x16 st, dp;
      p_and_ds<O, BIAS>(ops, st, dp, sQ, sO, qb, kf, vf, sl2, bias, a.R, q0, sq.off, key, k0, kind == 2, seen,
                        sS[stage] + qb * 32, half,
                        [&](int r) { return a.inv[((long)b * a.H + h_now) * a.Sq + min(q0 + r, a.Sq - 1)]; });
      ops.accum(dv, sO, qb, st);
      ops.accum(dk, sQ, qb, dp);
    }
  }
  if (ki.n > 1) {  // in the accumulators' own order, 1 KB per store
    if (!touches<KR>(span, qt0, nt, i0, i1)) return;
    float4* dst = reinterpret_cast<float4*>(a.part + (((long)bh * w.slots() + item) * NW + wave) * (2 * 32 * DH)) + lane;
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        dst[(i * 4 + g) * 64] = make_float4(dk[i][4 * g], dk[i][4 * g + 1], dk[i][4 * g + 2], dk[i][4 * g + 3]);
        dst[(DH / 8 + i * 4 + g) * 64] = make_float4(dv[i][4 * g], dv[i][4 * g + 1], dv[i][4 * g + 2], dv[i][4 * g + 3]);
      }
    return;
  }
  tiles_ready();  // the tiles' space now takes the dK, then the dV rows
  if (k0 >= a.Sk) return;
  clear_if(!kv, dk);
  clear_if(!kv, dv);
  E* stage = sm + wave * O::STAGE;
  const bool nt_out = stream_out((long)a.B * a.Sk * a.Hkv * DH * (long)sizeof(E));
  O::rotate_back(dk, a.rope_tab, min(key, a.Sk - 1), half);
  O::store(dk, a.scale, lane, stage, static_cast<E*>(a.dk.p) + b * a.dk.b + (long)k0 * a.dk.t + hk * a.dk.h, a.dk.t,
           nt_out, a.Sk - k0, a.dh);
  O::store(dv, 1.f, lane, stage, static_cast<E*>(a.dv.p) + b * a.dv.b + (long)k0 * a.dv.t + hk * a.dv.h, a.dv.t,
           nt_out, a.Sk - k0, a.dh);
}

// Adds a split block's partial sums and writes its rows: one workgroup per 32 keys, output and
// pair of dim blocks (d, d + DH / 64: what a rotation mixes).  Its four waves take every fourth
// split each, then wave 0 adds the four, always in this order.
template <class O, int NW>
__global__ __launch_bounds__(256) void attn_masked_dkdv_join(MaskedAttnArgs a, KeyWork w, int blocks) {
  typedef typename O::E E;
  constexpr int DH = O::DH, ND = DH / 32;
  __shared__ float4 part[3][8][64];
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = blockIdx.x % NW, kb = blockIdx.x / NW % blocks, bh = blockIdx.x / NW / blocks;
  const bool is_v = blockIdx.y & 1;
  const int d0 = blockIdx.y >> 1, b = bh / a.Hkv, hk = bh % a.Hkv;
  const int kw0 = kb * 32 * NW, k0 = kw0 + wave * 32, key = k0 + l32;
  if (k0 >= a.Sk) return;  // the whole workgroup
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const Span span = query_span(mask, k0, sq.off, sq.lq);
  int qt0, nt;
  query_tiles<O::KR>(a, sq, kw0, 32 * NW, qt0, nt);
  const int item = kb < w.nfar ? kb * w.s_far : w.nfar * w.s_far + (kb - w.nfar) * w.s_near;
  const int c = kb < w.nfar ? w.c_far : w.c_near, nit = nt * (a.H / a.Hkv), n = (nit + c - 1) / c;
  float4 acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  const float4* src = reinterpret_cast<const float4*>(a.part + (((long)bh * w.slots() + item) * NW + wave) * (2 * 32 * DH)) +
                      (is_v ? DH / 8 * 64 : 0) + lane;
  const long step = (long)NW * 2 * 32 * DH / 4;
  for (int s = sub; s < n; s += 4) {
    if (!touches<O::KR>(span, qt0, nt, s * c, min(nit, s * c + c))) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 v = src[s * step + ((d0 + i / 4 * (ND / 2)) * 4 + i % 4) * 64];
      acc[i].x += v.x;
      acc[i].y += v.y;
      acc[i].z += v.z;
      acc[i].w += v.w;
    }
  }
  if (sub)
#pragma unroll
    for (int i = 0; i < 8; ++i) part[sub - 1][i][lane] = acc[i];
  __syncthreads();
  if (sub || key >= a.Sk) return;
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 v = part[k][i][lane];
      acc[i].x += v.x;
      acc[i].y += v.y;
      acc[i].z += v.z;
      acc[i].w += v.w;
    }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (key >= sq.lk) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);  // as clear_if
  const View& o = is_v ? a.dv : a.dk;
  E* dst = static_cast<E*>(o.p) + b * o.b + (long)key * o.t + hk * o.h;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float x[2][4] = {{acc[g].x, acc[g].y, acc[g].z, acc[g].w}, {acc[4 + g].x, acc[4 + g].y, acc[4 + g].z, acc[4 + g].w}};
    const int at = d0 * 32 + 8 * g + 4 * half;
    if (!is_v)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x0 = x[0][e] * a.scale, x1 = x[1][e] * a.scale;
        float cs = 1.f, sn = 0.f;
        if (a.rope_tab) rope_cs(a.rope_tab, key, at + e, DH, &cs, &sn);
        x[0][e] = x0 * cs + x1 * sn;
        x[1][e] = x1 * cs - x0 * sn;
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int dim = i * (DH / 2) + at;
      if constexpr (sizeof(E) == 2) {
        St<E>::st4(dst, dim, x[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (dim + e < a.dh) St<E>::st(dst, dim + e, x[i][e]);
      }
    }
  }
}

// Both passes of a (batch, head) whose queries and keys fit one workgroup's LDS, without shared
// heads: bound by latency, so Q, dO, K and V are brought once, all at a time, and the dK/dV pass
// finds them, the statistics and the bias where the dQ pass left them.  384 of 128 x 128, head
// dim 64, with the table's gradient: 22.6 us, 36.4 as two kernels.
template <class O, bool BIAS, bool DTAB, int ROWS>
__global__ __launch_bounds__(256, O::DH == 64 && sizeof(typename O::E) == 2 ? 2 : 1) void attn_masked_bwd_small(MaskedAttnArgs a) {
  typedef typename O::E E;
  constexpr int DH = O::DH, KR = O::KR, TILE = O::TILE, NW = 4, NT = ROWS / KR;
  __shared__ __attribute__((aligned(1024))) E sm[4 * NT * TILE];  // Q, dO, K, V
  __shared__ __attribute__((aligned(16))) float2 sS[ROWS];        // (lse, D)
  __shared__ float sInv[ROWS];
  extern __shared__ float sbias[];                                // bias, then (DTAB) one diagonal array per wave
  static_assert(4 * NT * TILE >= NW * O::STAGE, "the rows fit the tiles' space on their way out");
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = xcd_block(blockIdx.x, gridDim.x), b = bh / a.H, h = bh % a.H;
  const Seq sq = seq_of(a, b);
  const Mask mask(a, sq.lk);
  const float sl2 = kLog2e * a.scale;
  const int W = 2 * a.R + 1;
  O ops(lane, a.dh);
  auto bring = [&](const View& v, int rows, E* dst) {
    const E* src = static_cast<const E*>(v.p) + b * v.b + h * v.h;
    const uint32_t first = O::template dma_first<NW>(v.t, a.dh, lane, wave);
    for (int r0 = 0; r0 < rows; r0 += KR)
      O::template dma<NW>(src + (long)r0 * v.t, v.t, rows - 1 - r0, dst + r0 / KR * TILE, a.dh, lane, wave, first);
  };
  E *sQ = sm, *sO = sm + NT * TILE, *sK = sm + 2 * NT * TILE, *sV = sm + 3 * NT * TILE;
  bring(a.k, sq.lk, sK);
  bring(a.q, sq.lq, sQ);
  bring(a.v, sq.lk, sV);
  bring(a.dout, sq.lq, sO);
  const int q0 = wave * 32, q = q0 + l32, p = sq.off + q;
  const bool qv = q < sq.lq;
  const long row = qv ? q : 0;
  typename O::Rows of;
  if (!DTAB)
    O::load_rows(of, static_cast<const E*>(a.o.p) + b * a.o.b + row * a.o.t + h * a.o.h, qv, half, a.dh);
  float lse = qv ? lse_or_inf(a.lse[(long)bh * a.Sq + row]) : INFINITY;
  float* diag = sbias + (1 + wave) * W;
  if (BIAS) load_bias<64 * NW>(a, h, sbias);
  if (DTAB)
    for (int i = 0; i < W; i += 64) diag[min(i + lane, W - 1)] = 0.f;  // all lanes, as in load_bias
  tiles_ready();

  // queries q0 .. q0 + 31 against every key
  f32x16 dq[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[i][r] = 0.f;
  float dsum = 0.f, dlo = 0.f, dhi = 0.f, psum = 0.f, inv = 1.f;
  const bool far = BIAS && __any(is_far(lse));
  if (q0 < sq.lq) {
    const int plo = sq.off + q0, phi = sq.off + min(q0 + 31, sq.lq - 1);
    const Span span = key_span(mask, plo, phi);
    const Visible seen = keys_of(mask, p);
    typename O::Rows qf, df;
    ops.tile_rows(qf, sQ + q0 / KR * TILE, q0 / 32 % (KR / 32), a.dh);
    ops.tile_rows(df, sO + q0 / KR * TILE, q0 / 32 % (KR / 32), a.dh);
    if (!DTAB) dsum = O::dot(of, df);
    auto block = [&](int k0, int kind, f32x16& st, f32x16& dp) {
      p_and_dp<O, BIAS>(ops, st, dp, sK + k0 / KR * TILE, sV + k0 / KR * TILE, k0 / 32 % (KR / 32), qf, df, sl2, sbias, a.R,
                        k0, p, plo, phi, kind == 2, seen, lse, half);
    };
    auto add = [&](int k0, f32x16& st, const f32x16& dp) {
      if (far) {
        if (DTAB)
#pragma unroll
          for (int r = 0; r < 16; ++r) st[r] *= inv;
        else psum += sum16(st);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] *= dp[r] - dsum;  // dS
      if (DTAB) add_diag(st, k0 - sq.off - q0, a.R, diag, dlo, dhi, lane);
      ops.accum(dq, sK + k0 / KR * TILE, k0 / 32 % (KR / 32), st);
    };
    if constexpr (DTAB) {  // D from P and dP, as in the dQ pass, which stay in registers here
      f32x16 st[ROWS / 32], dp[ROWS / 32];
#pragma unroll
      for (int i = 0; i < ROWS / 32; ++i) {
        if (span.kind(i) == 0) continue;
        block(i * 32, span.kind(i), st[i], dp[i]);
#pragma unroll
        for (int r = 0; r < 16; ++r) dsum = fmaf(st[i][r], dp[i][r], dsum);
        if (far) psum += sum16(st[i]);
      }
      dsum += __shfl_xor(dsum, 32, 64);
      if (far) {
        inv = inv_sum(psum + __shfl_xor(psum, 32, 64));
        dsum *= inv;
      }
#pragma unroll
      for (int i = 0; i < ROWS / 32; ++i)
        if (span.kind(i) != 0) add(i * 32, st[i], dp[i]);
    } else {
#pragma unroll 1
      for (int k0 = 0; k0 < sq.lk; k0 += 32) {
        const int kind = span.kind(k0 / 32);
        if (kind == 0) continue;
        f32x16 st, dp;
        block(k0, kind, st, dp);
        add(k0, st, dp);
      }
    }
  }
  if (lse == INFINITY) dsum = 0.f;
  clear_if(lse == INFINITY, dq);
  if (!DTAB && far) {
    inv = inv_sum(psum + __shfl_xor(psum, 32, 64));
    scale_by(inv, dq);
  }
  if (q < ROWS && half == 0) {
    sS[q] = make_float2(lse, dsum);
    sInv[q] = inv;
  }
  if (DTAB) close_diag(diag, W, dlo, dhi, lane);
  __syncthreads();
  if (DTAB) put_diag<NW>(sbias, W, a.diag + (long)bh * W);

  // keys k0 .. k0 + 31 against every query
  const int k0 = wave * 32, key = k0 + l32;
  f32x16 dk[DH / 32], dv[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[i][r] = dv[i][r] = 0.f;
  if (k0 < sq.lk) {
    const Span span = query_span(mask, k0, sq.off, sq.lq);
    const Visible seen = rows_of(mask, key, sq.off, sq.lq);
    typename O::Rows kf, vf;
    ops.tile_rows(kf, sK + k0 / KR * TILE, k0 / 32 % (KR / 32), a.dh);
    ops.tile_rows(vf, sV + k0 / KR * TILE, k0 / 32 % (KR / 32), a.dh);
#pragma unroll 1
    for (int r0 = 0; r0 < sq.lq; r0 += 32) {
      const int kind = span.kind(r0 / 32), qb = r0 / 32 % (KR / 32), t = r0 / KR * TILE;
      if (kind == 0) continue;
      f32x16 st, dp;
      p_and_ds<O, BIAS>(ops, st, dp, sQ + t, sO + t, qb, kf, vf, sl2, sbias, a.R, r0, sq.off, key, k0, kind == 2, seen,
                        sS + r0, half, [&](int r) { return sInv[r0 + r]; });
      ops.accum(dv, sO + t, qb, st);
      ops.accum(dk, sQ + t, qb, dp);
    }
  }
  clear_if(key >= sq.lk, dk);
  clear_if(key >= sq.lk, dv);
  __syncthreads();  // the tiles' space now takes the rows on their way out
  E* stage = sm + wave * O::STAGE;
  const bool nt = stream_out((long)a.B * max(a.Sq, a.Sk) * a.H * DH * (long)sizeof(E));
  if (q0 < a.Sq) {
    O::rotate_back(dq, a.rope_tab, min(q, a.Sq - 1), half);
    O::store(dq, a.scale, lane, stage, static_cast<E*>(a.dq.p) + b * a.dq.b + (long)q0 * a.dq.t + h * a.dq.h, a.dq.t, nt,
             a.Sq - q0, a.dh);
  }
  if (k0 < a.Sk) {
    O::rotate_back(dk, a.rope_tab, min(key, a.Sk - 1), half);
    O::store(dk, a.scale, lane, stage, static_cast<E*>(a.dk.p) + b * a.dk.b + (long)k0 * a.dk.t + h * a.dk.h, a.dk.t, nt,
             a.Sk - k0, a.dh);
    O::store(dv, 1.f, lane, stage, static_cast<E*>(a.dv.p) + b * a.dv.b + (long)k0 * a.dv.t + h * a.dv.h, a.dv.t, nt,
             a.Sk - k0, a.dh);
  }
}

// dtable[t][h] += the sums of dS over the relative positions of bucket t, from the dQ pass's
// partial sums diag[row][head][W]: one workgroup per head; 256 positions at a time over the rows (as
// many rows at a time as 1024 threads hold positions), then a wave per bucket.  In a
// fixed order; in 64 bits, which costs nothing here.  Bound by the latency of its loads: eight
// are in flight at a time, past the last row too (with weight 0), and the buckets beside them.
__global__ __launch_bounds__(1024) void attn_bias_grad(MaskedAttnArgs a, int rows) {
  __shared__ double part[1024], sum[2 * ATTN_MAX_DISTANCE + 1];
  __shared__ int bucket[2 * ATTN_MAX_DISTANCE + 1];
  const int W = 2 * a.R + 1, h = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int span = min(256, (W + 63) / 64 * 64), groups = 1024 / span, g = threadIdx.x / span, at = threadIdx.x % span;
  for (int i0 = 0; i0 < W; i0 += span) {
    const int i = i0 + at;
    double s = 0.0;
    if (g < groups && i < W) {
      if (g == 0) bucket[i] = min(max(a.bucket[i], 0), a.nb - 1);
      for (int r0 = g; r0 < rows; r0 += 8 * groups) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = a.diag[((long)min(r0 + k * groups, rows - 1) * a.H + h) * W + i];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += r0 + k * groups < rows ? (double)v[k] : 0.0;
      }
    }
    part[threadIdx.x] = s;
    __syncthreads();
    if (g == 0 && i < W) {
      for (int k = 1; k < groups; ++k) s += part[k * span + at];
      sum[i] = s;
    }
    __syncthreads();
  }
  for (int t = wave; t < a.nb; t += 16) {
    double s = 0.0;
    for (int i = lane; i < W; i += 64)
      if (bucket[i] == t) s += sum[i];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) a.dtable[(long)t * a.H + h] += (float)s;
  }
}

// ================================================================ launchers
constexpr int MA_NW = 4;

static long blocks_of(int n) { return (n + 32 * MA_NW - 1) / (32 * MA_NW); }

// keys that a query block may see, at most about
static long key_reach(const MaskedAttnArgs& a) {
  return a.window ? std::min<long>(a.Sk, (long)a.Sq + (a.causal ? 1 : 2) * (long)a.window + a.sinks) : a.Sk;
}
// for attn_few_dq: 32-row blocks hold fewer than half of the SIMDs, and see keys for two waves
static bool few_blocks(const MaskedAttnArgs& a) {
  return (long)a.B * a.H * ((a.Sq + 31) / 32) < 512 && key_reach(a) >= 64;
}

// HIP takes fewer than 2^32 threads in a launch's x dimension, and workgroups here have 256 (attn_bias_grad, one
// workgroup of 1024 per head, stays below that)
constexpr long MAX_WGS = (1l << 24) - 1;

static size_t al256(size_t n) { return (n + 255) & ~(size_t)255; }

// Workgroups of the dK/dV pass: two per CU hide each other's barriers, so blocks are split
// until there are 512, but no finer than four iterations (bf16 with the bias, 8 heads of 64, 1000 tokens: 20 us and 5 for the
// join, 19 and 7 with two; 4 heads on 2 of 128, 1824 tokens: 40 and 8, 34 and 9 with two), fp32, whose products
// take 8 times as long, one (2 x 2 heads of 96, 557 tokens, window 183: 35 and 7, 75 and 6 with four).
static KeyWork key_work(int dtype, const MaskedAttnArgs& a) {
  const int KR = dtype == DT_BF16 ? 64 : 32, grp = a.H / a.Hkv, rows = 32 * MA_NW;
  KeyWork w;
  w.nk = (int)blocks_of(a.Sk);
  w.nfar = a.window ? (int)std::min<long>(w.nk, (a.sinks + rows - 1) / rows) : w.nk;
  const long far = (long)grp * ((a.Sq + KR - 1) / KR);
  const long span = (long)rows + (a.causal ? 1l : 2l) * a.window;
  const long near = a.window ? std::min(far, grp * (span / KR + 2)) : far;
  const long least = dtype == DT_BF16 ? 4 : 1;
  const bool has_near = w.nfar < w.nk;
  const long wgs = (long)w.nk * a.B * a.Hkv, nfar = (long)w.nfar * a.B * a.Hkv, longest = has_near ? near : far;
  // Not into more than 64 pieces, which the join adds one after the other (whole backward, here and below, under
  // load: fp32, 8 heads of 64 on 1, 512 tokens: 71 us, 89 with up to 128, 649 unsplit), nor the far ones into more than 2048 workgroups, as
  // their partial sums take 64 or 128 KB each.
  const long want = std::max(1l, std::min({(512 + wgs - 1) / wgs, longest / least, 64l}));
  const long c_least = std::max({least, (far + 63) / 64, (far * nfar + 2047) / 2048});
  w.c_near = (int)((longest + want - 1) / want);
  w.s_near = has_near ? (int)((near + w.c_near - 1) / w.c_near) : 1;
  long c = far;
  // All of them far: nothing else fills gaps, so they are dealt as the others are (16 heads of 128, 2048 tokens:
  // 154 us, 232 in eighths of that).  Causal ones in two pieces alone cannot even out their unequal
  // lengths: quarters of that (32 heads on 8 of 128, 4096 tokens: 585 us, 640 in two pieces; 16 heads of 64, 2048
  // tokens: 99.6 and 97.5).
  if (!has_near) c = std::max(a.causal && want == 2 ? (far + 7) / 8 : (long)w.c_near, c_least);
  // A far block is left whole up to twice a near one's length (the join costs as much), else
  // dealt out in eighths of that, so that they fill the gaps: 512 near workgroups of 80
  // iterations are one round of the GPU, and far ones as long would begin another.  With the
  // join, 8192 tokens and window 1024: halves 430 us, quarters 383, eighths 365.
  // At least as many pieces as of a near one: KeyWork::slots.
  else if (w.s_near > 1 || far > 2 * near) c = std::min(std::max((long)(w.c_near + 7) / 8, c_least), far / w.s_near);
  w.c_far = (int)std::min(far, c);
  w.s_far = w.nfar ? (int)((far + w.c_far - 1) / w.c_far) : 1;
  if (w.items() * a.B * a.Hkv > MAX_WGS) {
    w.s_far = w.s_near = 1;
    w.c_far = w.c_near = (int)far;
  }
  return w;
}

struct BwdSpace {
  size_t inv, diag, part, total;
};
static BwdSpace bwd_space(int dtype, const MaskedAttnArgs& a, bool dtable) {
  BwdSpace s;
  s.inv = al256((size_t)a.B * a.H * a.Sq * 8);
  s.diag = s.inv + al256((size_t)a.B * a.H * a.Sq * 4);
  s.part = s.diag + (dtable ? al256((size_t)a.B * (few_blocks(a) ? (a.Sq + 31) / 32 : blocks_of(a.Sq)) * a.H *
                                     (2 * a.R + 1) * 4) : 0);
  const int dh = a.dh <= 64 ? 64 : 128;
  s.total = s.part + al256((size_t)a.B * a.Hkv * key_work(dtype, a).slots() * MA_NW * 2 * 32 * dh * 4);
  return s;
}

// A few queries against many keys: the rows of a key-value head fill one block, or the blocks
// are one round of workgroups (two per CU at head dims up to 64; fp32 ones gain there in two rounds
// as well), over a loop that gives each wave some of it.  16 heads on 4 of 128, 256 queries on 1024 and 8192
// keys: 16.4 and 51 us here, 26.5 and 170 in attn_masked_fwd; 8 heads of 64, 100 on 100 5.8 and 6.9, 64 on 64
// 5.8 and 5.3; 2 x 16 heads on 4 of 128, 300 on 300 (304 blocks) 16.8 and 11.5; over 8192 keys two rounds are
// no worse (512 blocks: 163 and 172).
static bool few(const MaskedAttnArgs& a) {
  const long rows = (long)a.Sq * (a.H / a.Hkv), blocks = a.B * a.Hkv * ((rows + 31) / 32);
  return rows <= 32 || (blocks <= (a.dh <= 64 ? 512 : 256) && key_reach(a) >= 96) || (blocks <= 512 && key_reach(a) >= 4096);
}
// At least 256 workgroups where there are tiles for their four waves (64 heads, window
// 1024: 13.9 us with both kernels; with two tiles for each wave 14.8); none split below 512 keys, as the join
// takes 4 us.  Rounded up: where the blocks of rows do not divide 256, head dim 128 (one workgroup per CU) runs a second,
// nearly empty round (32 heads on 8, 16384 keys: 3.9 TB/s of them at batch 3, 5.4 at batch 4).
static FewWork few_work(const MaskedAttnArgs& a) {
  FewWork w;
  w.rb = (a.Sq * (a.H / a.Hkv) + 31) / 32;
  const long wgs = (long)a.B * a.Hkv * w.rb;
  const long reach = key_reach(a);
  w.split = reach < 512 ? 1 : (int)std::max(1l, std::min({64l, (256 + wgs - 1) / wgs, reach / 128}));
  return w;
}

bool masked_attn_fits(int dtype, const MaskedAttnArgs& a) {
  long most = std::max(blocks_of(a.Sq) * a.H, blocks_of(a.Sk) * a.Hkv) * a.B;
  if (few(a)) {
    const FewWork w = few_work(a);
    most = std::max(most, (long)a.B * a.Hkv * w.split * w.rb);
    if (w.split > 1) most = std::max(most, ((long)a.B * a.H * a.Sq + 3) / 4);
  }
  const KeyWork w = key_work(dtype, a);
  if (w.slots()) most = std::max(most, (long)a.B * a.Hkv * (w.s_near > 1 ? w.nk : w.nfar) * MA_NW);
  return most <= MAX_WGS;
}

void masked_attn_bytes(int dtype, const MaskedAttnArgs& a, bool dtable, size_t* fwd, size_t* bwd) {
  *fwd = 0;
  if (few(a)) {
    const FewWork w = few_work(a);
    const int dh = a.dh <= 64 ? 64 : 128;
    if (w.split > 1) *fwd = (size_t)a.B * a.Hkv * w.split * w.rb * 32 * (dh + 2) * 4;
  }
  *bwd = bwd_space(dtype, a, dtable).total;
}

void masked_attn_workspace(int dtype, MaskedAttnArgs& a, void* ws) {
  const BwdSpace s = bwd_space(dtype, a, a.dtable != nullptr);
  char* p = static_cast<char*>(ws);
  a.stat = reinterpret_cast<float2*>(p);
  a.inv = reinterpret_cast<float*>(p + s.inv);
  a.diag = reinterpret_cast<float*>(p + s.diag);
  a.part = reinterpret_cast<float*>(p + s.part);
}

// NW: waves whose private tiles fit the LDS of a CU
template <class O, int NW>
static hipError_t few_ops(const MaskedAttnArgs& a, hipStream_t s) {
  const FewWork w = few_work(a);
  const dim3 grid((unsigned)((long)a.B * a.Hkv * w.split * w.rb)), block(64 * NW);
  if (a.table) RG_LAUNCH((attn_few_fwd<O, true, NW>), grid, block, 0, s, a, w);
  else RG_LAUNCH((attn_few_fwd<O, false, NW>), grid, block, 0, s, a, w);
  if (w.split > 1)
    RG_LAUNCH((attn_few_join<O>), dim3((unsigned)(((long)a.B * a.H * a.Sq + 3) / 4)), dim3(256), 0, s, a, w);
  return hipGetLastError();
}
template <class O>
static hipError_t fwd_ops(const MaskedAttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(blocks_of(a.Sq) * a.B * a.H)), block(64 * MA_NW);
  if (a.table) RG_LAUNCH((attn_masked_fwd<O, true, MA_NW>), grid, block, (2 * a.R + 1) * 4, s, a);
  else RG_LAUNCH((attn_masked_fwd<O, false, MA_NW>), grid, block, 0, s, a);
  return hipGetLastError();
}
// ROWS: queries, and keys, that the LDS of attn_masked_bwd_small holds
template <class O, int ROWS>
static bool fits_small(const MaskedAttnArgs& a) {
  const size_t lds = sizeof(typename O::E) * 4 * (ROWS / O::KR) * O::TILE + ROWS * 12 +
                     (a.table ? (size_t)(2 * a.R + 1) * 4 * (a.dtable ? 5 : 1) : 0);
  return a.H == a.Hkv && a.Sq <= ROWS && a.Sk <= ROWS && lds <= 160 * 1024;
}
template <class O, int NW>
static bool launch_few_dq(const MaskedAttnArgs& a, hipStream_t s) {
  const int W4 = (2 * a.R + 1) * 4;
  const size_t lds = sizeof(typename O::E) * NW * 4 * O::BLOCK + NW * 256 + (a.table ? (size_t)W4 * (a.dtable ? 1 + NW : 1) : 0);
  const long wgs = (long)a.B * a.H * ((a.Sq + 31) / 32);
  // one and a half rounds of the CUs at most, but over long loops: 348 workgroups of one per CU (fp32, 29 x 2 heads
  // of 191, with the table's gradient) take 41 us, 51 in the other kernel; 448 (bf16, 4 x 8 heads of 430) 25.7 and
  // 20.2; 408 (bf16, 3 heads of 4323, with the table's gradient) 248 and 293
  if (!few_blocks(a) || lds > 160 * 1024 || (wgs > 384 * (long)(160 * 1024 / lds) && key_reach(a) < 1024)) return false;
  const dim3 grid((unsigned)wgs), block(64 * NW);
  if (!a.table) RG_LAUNCH((attn_few_dq<O, false, false, NW>), grid, block, 0, s, a);
  else if (!a.dtable) RG_LAUNCH((attn_few_dq<O, true, false, NW>), grid, block, W4, s, a);
  else RG_LAUNCH((attn_few_dq<O, true, true, NW>), grid, block, (1 + NW) * W4, s, a);
  return true;
}
// FNW: as few_ops' NW
template <class O, int ROWS, int FNW>
static hipError_t bwd_ops(int dtype, const MaskedAttnArgs& a, hipStream_t s) {
  if (fits_small<O, ROWS>(a)) {
    const dim3 grid((unsigned)(a.B * a.H)), block(256);
    const int W4 = (2 * a.R + 1) * 4;
    if (!a.table) RG_LAUNCH((attn_masked_bwd_small<O, false, false, ROWS>), grid, block, 0, s, a);
    else if (!a.dtable) RG_LAUNCH((attn_masked_bwd_small<O, true, false, ROWS>), grid, block, W4, s, a);
    else {
      RG_LAUNCH((attn_masked_bwd_small<O, true, true, ROWS>), grid, block, 5 * W4, s, a);
      RG_LAUNCH(attn_bias_grad, dim3(a.H), dim3(1024), 0, s, a, a.B);
    }
    return hipGetLastError();
  }
  const KeyWork w = key_work(dtype, a);
  const dim3 gq((unsigned)(blocks_of(a.Sq) * a.B * a.H)), gk((unsigned)(w.items() * a.B * a.Hkv)), block(64 * MA_NW);
  const int W = 2 * a.R + 1;
  const bool few_dq = launch_few_dq<O, FNW>(a, s);
  if (!few_dq) {
    if (!a.table) RG_LAUNCH((attn_masked_bwd_dq<O, false, false, MA_NW>), gq, block, 0, s, a);
    else if (!a.dtable) RG_LAUNCH((attn_masked_bwd_dq<O, true, false, MA_NW>), gq, block, W * 4, s, a);
    else RG_LAUNCH((attn_masked_bwd_dq<O, true, true, MA_NW>), gq, block, (1 + MA_NW) * W * 4, s, a);
  }
  if (a.table) RG_LAUNCH((attn_masked_bwd_dkdv<O, true, MA_NW>), gk, block, 2 * W * 4, s, a, w);
  else RG_LAUNCH((attn_masked_bwd_dkdv<O, false, MA_NW>), gk, block, 0, s, a, w);
  if (a.dtable)
    RG_LAUNCH(attn_bias_grad, dim3(a.H), dim3(1024), 0, s, a, (int)(a.B * (few_dq ? (a.Sq + 31) / 32 : blocks_of(a.Sq))));
  const int split = w.s_near > 1 ? w.nk : w.s_far > 1 ? w.nfar : 0;
  if (split)
    RG_LAUNCH((attn_masked_dkdv_join<O, MA_NW>), dim3((unsigned)(a.B * a.Hkv * split * MA_NW), 2 * O::DH / 64),
              dim3(256), 0, s, a, w, split);
  return hipGetLastError();
}

hipError_t launch_masked_attn_fwd(int dtype, const MaskedAttnArgs& a, hipStream_t s) {
  if (few(a)) {
    if (dtype == DT_BF16) return a.dh == 64 ? few_ops<OpsBf16<64>, 4>(a, s) : few_ops<OpsBf16<128>, 4>(a, s);
    return a.dh <= 64 ? few_ops<OpsF32<64>, 4>(a, s) : few_ops<OpsF32<128>, 2>(a, s);
  }
  if (dtype == DT_BF16) return a.dh == 64 ? fwd_ops<OpsBf16<64>>(a, s) : fwd_ops<OpsBf16<128>>(a, s);
  return a.dh <= 64 ? fwd_ops<OpsF32<64>>(a, s) : fwd_ops<OpsF32<128>>(a, s);
}
hipError_t launch_masked_attn_bwd(int dtype, const MaskedAttnArgs& a, hipStream_t s) {
  if (dtype == DT_BF16) return a.dh == 64 ? bwd_ops<OpsBf16<64>, 128, 4>(dtype, a, s) : bwd_ops<OpsBf16<128>, 128, 4>(dtype, a, s);
  return a.dh <= 64 ? bwd_ops<OpsF32<64>, 128, 4>(dtype, a, s) : bwd_ops<OpsF32<128>, 64, 2>(dtype, a, s);
}

}  // namespace rg
