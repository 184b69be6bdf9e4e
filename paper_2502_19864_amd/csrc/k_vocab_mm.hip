// The vocabulary head's products in bf16: logits h w^T with their statistics, dh = P w, dw = P^T h
// (k_vocab.hip has the formulas and what runs between them).
//
// One kernel on MFMA 32x32x16, whose operands may lie either way in memory: [rows][k], as h and w do for the
// logits, or [k][rows], as w does for dh and both of P and h do for dw.  So nothing is transposed in memory, where
// a copy of w or P would cost as much as reading it twice.  Tiles come by DMA, two to four stages deep, 64 k
// wide.  In LDS an operand keeps its order:
//  * [rows][64]: chunk c (16 B) of row r at c ^ (r / 2) % 8, so the 16 rows that one pass of a fragment read
//    touches hit all banks once;
//  * [64][rows]: read by transposing loads, four k of 32 columns at a time; the 64-byte group of the columns
//    at its number ^ k % 4, so those four rows lie in different banks.
// Rows past the operands' ends are clamped (their results are not stored) and k past the end meets zeros
// in the other operand: hc and P are padded with them.
#include <type_traits>
#include <utility>

#include "common.h"
#include "kernels.h"
#include "vocab_peak.h"

namespace rg {

template <int N>
__device__ __forceinline__ void wait_dma() {  // vmcnt <= N and lgkmcnt == 0
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | ((N >> 4) << 14));
}
__device__ __forceinline__ void wg_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ND fragment reads of the next k-step spread evenly between the NM MFMAs of this one
template <int ND, int NM, int... Q>
__device__ __forceinline__ void spread_reads(std::integer_sequence<int, Q...>) {
  ([] {
    constexpr int n = (Q + 1) * ND / NM - Q * ND / NM;
    if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(0x100, n, 0);  // DS read
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                       // MFMA
  }(), ...);
}

// One operand of a product: R rows (of the tile) by 64 k, KMAJOR: [rows][k] in memory.
template <int R, int NW, bool KMAJOR>
struct Operand {
  static constexpr int L = R / (8 * NW);            // DMA instructions per wave and tile
  static constexpr int CPR = KMAJOR ? 8 : R / 8;    // chunks per LDS row
  static constexpr int RPI = 64 / CPR;              // LDS rows per instruction
  static_assert(L * 8 * NW == R && (KMAJOR || R >= 128), "whole instructions; four groups of columns");
  const char* base;   // the tile's first element
  long step;          // bytes per k-tile
  uint32_t off[L];    // per-lane byte offsets within a k-tile
  int row[L], chunk[L];
  uint32_t ld2;
  // rows0: first row; rows: how many there are (KMAJOR: clamped one by one, else in chunks of 8)
  __device__ __forceinline__ void init(const bf16* p, long ld, int rows0, int rows, int wave, int lane) {
    ld2 = (uint32_t)ld * 2;
    if constexpr (KMAJOR) {
      base = reinterpret_cast<const char*>(p + (long)rows0 * ld);
      step = 128;
    } else {
      base = reinterpret_cast<const char*>(p + rows0);
      step = ld * 128;
    }
    base = uniform_ptr(base);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int r = (i * NW + wave) * RPI + lane / CPR, pos = lane % CPR;
      if constexpr (KMAJOR) {
        chunk[i] = pos ^ ((r >> 1) & 7);
        row[i] = min(rows0 + r, rows - 1) - rows0;
      } else {
        chunk[i] = min(pos ^ ((r & 3) << 2), (rows - rows0 + 7) / 8 - 1);
        row[i] = r;
      }
      off[i] = (uint32_t)row[i] * ld2 + chunk[i] * 16;
    }
  }
  // instruction i of k-tile kt; left: k of this tile that the operand has (a whole tile: 64)
  __device__ __forceinline__ void dma(int i, int kt, int left, uint32_t lds, int wave_u) const {
    uint32_t o = off[i];
    if (left < 64) {
      if constexpr (KMAJOR) o -= max(0, chunk[i] - (left / 8 - 1)) * 16;
      else o -= max(0, row[i] - (left - 1)) * ld2;
    }
    dma16_m0(base + (long)kt * step, o, lds + (i * NW + wave_u) * 1024);
  }
};

// Fragments of F blocks of 32 rows from first row r0 of the tile in LDS
template <int R, int F, bool KMAJOR>
struct Frags {
  uint32_t at[KMAJOR ? 1 : F];
  __device__ __forceinline__ void init(int r0, int lane) {
    if constexpr (KMAJOR) {
      at[0] = (r0 + (lane & 31)) * 128;
    } else {
      const int g = lane >> 4, r = lane & 15;
#pragma unroll
      for (int i = 0; i < F; ++i)
        at[i] = (8 * (g >> 1) + (r >> 2)) * (R * 2) + (((r0 / 32 + i) ^ (r >> 2)) * 4 + 2 * (g & 1) + ((r & 3) >> 1)) * 16 + (r & 1) * 8;
    }
  }
  __device__ __forceinline__ void read(const char* tile, int ks, int lane, bf16x8 (&f)[F]) const {
    if constexpr (KMAJOR) {
      const char* p = tile + at[0] + 16 * ((2 * ks + (lane >> 5)) ^ ((lane >> 1) & 7));
#pragma unroll
      for (int i = 0; i < F; ++i) f[i] = *reinterpret_cast<const bf16x8*>(p + i * 32 * 128);
    } else {
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const char* p = tile + at[i] + ks * 16 * (R * 2);
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)p));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(p + 4 * R * 2)));
        f[i] = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
      }
    }
  }
};

constexpr int stage_rows(int bm, int row_bytes, int lds_bytes) {
  int r = bm;
  while (r > 32 && r * row_bytes > lds_bytes) r /= 2;
  return r;
}

struct VocabProduct {
  const bf16* A; long lda;
  const bf16* B; long ldb;
  int M, N;        // M: of dw (the logits and dh have the rows that count)
  int K;           // k of the logits (d) and of dh (V)
  int slots;       // dh: workgroups of one round
};
// dh's k (the vocabulary) is dealt to several workgroups per tile where the tiles of the rows that count leave CUs
// idle, eight k-tiles at least to each
__host__ __device__ inline int dh_splits(int slots, int tiles, int V) {
  const int by_slots = slots / tiles, by_k = V / 512, s = by_slots < by_k ? by_slots : by_k;
  return s < 1 ? 1 : s;
}

// The tile of C[m][n] = sum_k A(m, k) B(n, k) that a workgroup makes, by XCD: workgroups are dealt round-robin to the eight
// XCDs; each takes a contiguous run of a raster in bands of GROUP tile rows, so what its L2 holds is shared.
template <int GROUP>
__device__ __forceinline__ bool vocab_tile(int g, int ntm, int ntn, int& tm, int& tn) {
  const int n = ntm * ntn;
  if (g >= n) return false;
  const int x = g & 7, q = n >> 3, r = n & 7;
  g = x * q + min(x, r) + (g >> 3);
  const int band = g / (GROUP * ntn), first = band * GROUP, size = min(ntm - first, GROUP), in = g - band * GROUP * ntn;
  tm = first + in % size;
  tn = in / size;
  return true;
}

template <int BM, int BN, int WM, int WN, int NS, bool KA, bool KB, Prod E>
__global__ __launch_bounds__(64 * WM * WN) void vocab_mm_k(VocabArgs a, VocabProduct p) {
  constexpr int NW = WM * WN, NT = 64 * NW, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32, KS = 4;
  using OA = Operand<BM, NW, KA>;
  using OB = Operand<BN, NW, KB>;
  constexpr int LPT = OA::L + OB::L, STAGE = (BM + BN) * 128, CP = BN + 4;
  constexpr int ND = FM * (KA ? 1 : 2) + FN * (KB ? 1 : 2);
  static_assert(FM * 32 * WM == BM && FN * 32 * WN == BN && NS >= 2 && NS <= 4 && LPT * (NS - 1) < 64, "tile");
  constexpr int EPI_MIN = (BM == 256 && BN == 256 ? 128 : 64) * CP * 4;
  constexpr int LDS = EPI_MIN > NS * STAGE ? EPI_MIN : NS * STAGE;
  constexpr int RPP = stage_rows(BM, CP * 4, LDS);
  static_assert(BM % RPP == 0 && RPP * CP * 4 <= LDS && LDS <= 160 * 1024, "epilogue passes");
  __shared__ __attribute__((aligned(1024))) char smem[LDS];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / WN, wn = wave % WN;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int cnt = __builtin_amdgcn_readfirstlane(piece_rows(a));
  const int M = E == Prod::Dw ? p.M : cnt, N = p.N;
  const int K = E == Prod::Dw ? cnt : p.K;
  const int ntm = (M + BM - 1) / BM, ntn = (N + BN - 1) / BN;
  int splits = 1, split = 0;
  if constexpr (E == Prod::Dh) {
    if (ntm == 0) return;
    splits = __builtin_amdgcn_readfirstlane(dh_splits(p.slots, ntm * ntn, p.K));
    split = __builtin_amdgcn_readfirstlane(blockIdx.x / (ntm * ntn));
    if (split >= splits) return;
  }
  int tm, tn;
  if (!vocab_tile<4>((int)blockIdx.x - split * ntm * ntn, ntm, ntn, tm, tn)) return;
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int nk_all = (K + 63) / 64;
  const int kt0 = E == Prod::Dh ? (int)((long)nk_all * split / splits) : 0;
  const int kt1 = E == Prod::Dh ? (int)((long)nk_all * (split + 1) / splits) : nk_all;
  const int nk = kt1 - kt0;

  OA oa;
  OB ob;
  oa.init(p.A, p.lda, m0, M, wave, lane);
  ob.init(p.B, p.ldb, n0, N, wave, lane);
  // part q of `of` of k-tile kt's DMA instructions.  A (hc in the logits, P) has zeros up to whole k-tiles; B has not.
  auto issue = [&](int kt, int slot, int q, int of) {
    const uint32_t l0 = lds_addr(smem) + slot * STAGE;
    const int left = min(64, K - (kt0 + kt) * 64);
#pragma unroll
    for (int i = LPT * q / of; i < LPT * (q + 1) / of; ++i) {
      if (i < OA::L) oa.dma(i, kt0 + kt, 64, l0, wave_u);
      else ob.dma(i - OA::L, kt0 + kt, left, l0 + BM * 128, wave_u);
    }
  };
  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  Frags<BM, FM, KA> ra;
  Frags<BN, FN, KB> rb;
  ra.init(wm * TM, lane);
  rb.init(wn * TN, lane);
  bf16x8 fa[2][FM], fb[2][FN];
  auto read_frags = [&](int slot, int ks, int buf) {
    ra.read(smem + slot * STAGE, ks, lane, fa[buf]);
    rb.read(smem + slot * STAGE + BM * 128, ks, lane, fb[buf]);
  };
  auto wait_tiles = [&](int n) {  // at most n k-tiles still in flight
    if constexpr (NS >= 4) { if (n >= 3) { wait_dma<3 * LPT>(); return; } }
    if constexpr (NS >= 3) { if (n >= 2) { wait_dma<2 * LPT>(); return; } }
    if (n >= 1) { wait_dma<LPT>(); return; }
    wait_dma<0>();
  };
  // A finished stage is refilled in pieces, the first right after the barrier that frees it
  constexpr int PARTS = NS >= 3 ? KS : 2;
  auto step = [&](auto S, int kt) {
    constexpr int s = decltype(S)::value, sn = (s + 1) % NS, sp = (s + NS - 1) % NS;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 1 < KS) {
        if (ks + 1 < PARTS && kt > 0 && kt - 1 + NS < nk) issue(kt - 1 + NS, sp, ks + 1, PARTS);
        read_frags(s, ks + 1, (ks + 1) & 1);
      } else if (kt + 1 < nk) {
        wait_tiles(min(NS - 2, nk - 2 - kt));
        wg_barrier();
        if (kt + NS < nk) issue(kt + NS, s, 0, PARTS);
        read_frags(sn, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma32(fb[ks & 1][j], fa[ks & 1][i], acc[i][j]);
      spread_reads<ND, FM * FN>(std::make_integer_sequence<int, FM * FN>{});
    }
  };
  if (nk > 0) {
#pragma unroll
    for (int t = 0; t < NS; ++t)
      if (t < nk) issue(t, t, 0, 1);
    wait_tiles(min(NS, nk) - 1);
    wg_barrier();
    read_frags(0, 0, 0);
    for (int kt = 0; kt < nk; kt += NS) {
      step(std::integral_constant<int, 0>{}, kt);
      if (kt + 1 < nk) step(std::integral_constant<int, 1>{}, kt + 1);
      if constexpr (NS > 2) if (kt + 2 < nk) step(std::integral_constant<int, 2>{}, kt + 2);
      if constexpr (NS > 3) if (kt + 3 < nk) step(std::integral_constant<int, 3>{}, kt + 3);
    }
  }
  wait_dma<0>();
  wg_barrier();  // every wave is done with the operands

  // Lane l holds of each 32x32 block row l % 32, columns 8 g + 4 (l / 32) + 0..3, g = 0..3.
  const int l32 = lane & 31, half = lane >> 5;
  float* cf = reinterpret_cast<float*>(smem);
  if constexpr (E == Prod::Stats || E == Prod::Logits) {
    float* sm = cf;                                  // [BM][WN] maxima, sums, places
    float* sl = cf + BM * WN;
    int* sa = reinterpret_cast<int*>(cf + 2 * BM * WN);
    const int c0 = n0 + wn * TN + 4 * half;
    const bool edge = n0 + BN > N;
    auto col = [&](int j, int r) { return c0 + j * 32 + 8 * (r / 4) + r % 4; };
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = wm * TM + i * 32 + l32;
      const int lab = a.lab_c && m0 + row < M ? a.lab_c[a.row0 + m0 + row] : -1;
      if (lab >= n0 && lab < n0 + BN) {  // few lanes
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (col(j, r) == lab) a.target[a.row0 + m0 + row] = acc[i][j][r];
      }
      float m = -INFINITY;
      if (edge) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, col(j, r) < N ? acc[i][j][r] : -INFINITY);
      } else {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
      }
      m = fmaxf(m, __shfl_xor(m, 32));
      const float z = m == -INFINITY ? 0.f : m;
      float l = 0.f;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = exp_below(acc[i][j][r] - z);
          l += !edge || col(j, r) < N ? e : 0.f;
        }
      l += __shfl_xor(l, 32);
      int at = INT32_MAX;
      if (a.part_at) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (acc[i][j][r] == m && (!edge || col(j, r) < N)) at = min(at, col(j, r));
        at = min(at, __shfl_xor(at, 32));
      }
      if (half == 0) {
        sm[row * WN + wn] = m;
        sl[row * WN + wn] = l;
        sa[row * WN + wn] = at;
      }
    }
    __syncthreads();
    for (int row = tid; row < BM; row += NT) {
      if (m0 + row >= M) break;
      Peak q{sm[row * WN], sl[row * WN], sa[row * WN]};
#pragma unroll
      for (int w = 1; w < WN; ++w) q = join(q, Peak{sm[row * WN + w], sl[row * WN + w], sa[row * WN + w]});
      a.part[(long)(m0 + row) * a.tiles + tn] = make_float2(q.m, q.l);
      if (a.part_at) a.part_at[(long)(m0 + row) * a.tiles + tn] = min(q.at, N - 1);
    }
    if constexpr (E == Prod::Stats) return;
    __syncthreads();
  }
  // the tile through LDS, RPP rows at a time, so that stores are whole rows' pieces of 16 bytes
  constexpr int CPR = BN / 8;
#pragma unroll
  for (int pass = 0; pass < BM / RPP; ++pass) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if ((wm * TM + i * 32) / RPP != pass) continue;  // wave-uniform
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(cf + (wm * TM + i * 32 + l32 - pass * RPP) * CP + wn * TN + j * 32 + 8 * g + 4 * half) =
              make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
    }
    __syncthreads();
    if constexpr (E == Prod::Logits) {
      for (int idx = tid; idx < RPP * CPR * 2; idx += NT) {
        const int row = idx / (CPR * 2), c = idx % (CPR * 2) * 4, m = m0 + pass * RPP + row, n = n0 + c;
        if (m < M && n < a.Vp) *reinterpret_cast<float4*>(a.logits + (long)m * a.Vp + n) = *reinterpret_cast<const float4*>(cf + row * CP + c);
      }
    } else {
      for (int idx = tid; idx < RPP * CPR; idx += NT) {
        const int row = idx / CPR, c = idx % CPR * 8, m = m0 + pass * RPP + row, n = n0 + c;
        if (m >= M || n >= N) continue;
        float v[8];
        *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(cf + row * CP + c);
        *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(cf + row * CP + c + 4);
        if constexpr (E == Prod::Dh) {
          if (splits > 1) {
            float* o = a.dh_part + (((long)split * ntm + tm) * ntn + tn) * (BM * BN) + (pass * RPP + row) * BN + c;
            *reinterpret_cast<float4*>(o) = *reinterpret_cast<float4*>(v);
            *reinterpret_cast<float4*>(o + 4) = *reinterpret_cast<float4*>(v + 4);
          } else {
            *reinterpret_cast<bf16x8*>(static_cast<bf16*>(a.dh) + (long)a.idx[a.row0 + m] * a.lddh + n) = pack_frag(v);
          }
        } else {
          float* o = a.dw_acc + (long)m * a.ld_acc + n;
          if (!a.first) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += o[e];
          }
          if (a.last) {
            *reinterpret_cast<bf16x8*>(static_cast<bf16*>(a.dw) + (long)m * a.lddw + n) = pack_frag(v);
          } else {
            *reinterpret_cast<float4*>(o) = *reinterpret_cast<float4*>(v);
            *reinterpret_cast<float4*>(o + 4) = *reinterpret_cast<float4*>(v + 4);
          }
        }
      }
    }
    if (pass + 1 < BM / RPP) __syncthreads();
  }
}

// dh of a piece from its splits' sums, in their order; tiles are bt x bt
__global__ __launch_bounds__(256) void vocab_dh_sum_k(VocabArgs a, VocabProduct p, int bt) {
  const int cnt = piece_rows(a), cols = p.N / 8, i = blockIdx.x * 256 + threadIdx.x, m = i / cols, n = i % cols * 8;
  if (m >= cnt) return;
  const int ntn = (p.N + bt - 1) / bt, tiles = (cnt + bt - 1) / bt * ntn, splits = dh_splits(p.slots, tiles, p.K);
  if (splits == 1) return;
  const float* q = a.dh_part + (long)(m / bt * ntn + n / bt) * bt * bt + (m % bt) * bt + n % bt;
  float v[8] = {};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    float x[8];
    *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(q + (long)s * tiles * bt * bt);
    *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(q + (long)s * tiles * bt * bt + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  *reinterpret_cast<bf16x8*>(static_cast<bf16*>(a.dh) + (long)a.idx[a.row0 + m] * a.lddh + n) = pack_frag(v);
}

static int tiles_of(int x, int t) { return (x + t - 1) / t; }

template <int BM, int BN, int WM, int WN, int NS, bool KA, bool KB, Prod E>
static void go(const VocabArgs& a, VocabProduct p, hipStream_t s) {
  int wgs = tiles_of(E == Prod::Dw ? p.M : a.rows, BM) * tiles_of(p.N, BN);
  if (E == Prod::Dh && wgs < p.slots) wgs = p.slots;
  RG_LAUNCH((vocab_mm_k<BM, BN, WM, WN, NS, KA, KB, E>), dim3(wgs), dim3(64 * WM * WN), 0, s, a, p);
}

int vocab_mm_bn(int rows, int d, int V) { return rows > 128 && V > 128 && d >= 2048 ? 256 : 128; }
static int dh_tile(int rows) { return rows > 128 ? 256 : 128; }
static int dh_slots(int rows) { return rows > 128 ? 256 : 512; }

size_t vocab_dh_part_bytes(int rows, int d, int V) {
  const int t = dh_tile(rows), slots = dh_slots(rows);
  const long tiles = (long)tiles_of(rows, t) * tiles_of(d, t);
  // one tile to all of them: whichever rows count, splits times tiles are at most slots
  const long most = tiles * dh_splits(slots, 1, V);
  return (size_t)(most < slots ? most : slots) * t * t * 4;
}

void launch_vocab_logits_bf16(const VocabArgs& a, bool keep, hipStream_t s) {
  VocabProduct p{};
  p.A = static_cast<const bf16*>(a.hc) + (long)a.row0 * a.dp;
  p.lda = a.dp;
  p.B = static_cast<const bf16*>(a.w);
  p.ldb = a.ldw;
  p.N = a.V;
  p.K = a.d;
  if (a.bn == 256) {
    if (keep) go<256, 256, 4, 2, 2, true, true, Prod::Logits>(a, p, s);
    else go<256, 256, 4, 2, 2, true, true, Prod::Stats>(a, p, s);
  } else {
    if (keep) go<128, 128, 2, 2, 2, true, true, Prod::Logits>(a, p, s);
    else go<128, 128, 2, 2, 2, true, true, Prod::Stats>(a, p, s);
  }
}
void launch_vocab_dh_bf16(const VocabArgs& a, hipStream_t s) {
  VocabProduct p{};
  p.A = static_cast<const bf16*>(a.P);
  p.lda = a.Vp;
  p.B = static_cast<const bf16*>(a.w);
  p.ldb = a.ldw;
  p.N = a.d;
  p.K = a.V;
  p.slots = dh_slots(a.n);
  const int t = dh_tile(a.n);
  if (t == 256) go<256, 256, 4, 2, 2, true, false, Prod::Dh>(a, p, s);
  else go<128, 128, 2, 2, 2, true, false, Prod::Dh>(a, p, s);
  if (dh_splits(p.slots, 1, a.V) > 1)
    RG_LAUNCH(vocab_dh_sum_k, dim3((unsigned)(((long)a.rows * (a.d / 8) + 255) / 256)), dim3(256), 0, s, a, p, t);
}
void launch_vocab_dw_bf16(const VocabArgs& a, hipStream_t s) {
  VocabProduct p{};
  p.A = static_cast<const bf16*>(a.P);
  p.lda = a.Vp;
  p.B = static_cast<const bf16*>(a.hc) + (long)a.row0 * a.dp;
  p.ldb = a.dp;
  p.M = a.V;
  p.N = a.d;
  if (a.n > 128) go<256, 256, 4, 2, 2, false, false, Prod::Dw>(a, p, s);
  else go<128, 128, 2, 2, 2, false, false, Prod::Dw>(a, p, s);
}

}  // namespace rg
