// The vocabulary head's products in bf16: logits h w^T with their statistics, dh = P w, dw = P^T h
// (k_vocab.hip has the formulas and what runs between them).
//
// One kernel on MFMA 32x32x16, whose operands may lie either way in memory: [rows][k], as h and w do for the
// logits, or [k][rows], as w does for dh and both of P and h do for dw.  So nothing is transposed in memory, where
// a copy of w or P would cost as much as reading it twice.  Tiles come by DMA, two stages deep, 64 k
// wide.  In LDS an operand keeps its order:
//  * [rows][64]: chunk c (16 B) of row r at c ^ (r / 2) % 8, so the 16 rows that one pass of a fragment read
//    touches hit all banks once;
//  * [64][rows]: read by transposing loads, four k of 32 columns at a time; the 64-byte group of the columns
//    at its number ^ k % 4, so those four rows lie in different banks.
// Rows past the operands' ends are clamped (their results are not stored).  k past the end meets zeros in A: hc and P are
// padded with them.  In w of the logits it is zeros too, as an infinity read again there would make a NaN; where B is [k][rows] it is its
// last row again, whose infinities have made their columns NaN already.
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

// One operand of a product: R rows (of the tile) by BK k, KMAJOR: [rows][k] in memory.
template <int R, int BK, int NW, bool KMAJOR>
struct Operand {
  static constexpr int L = R * BK / (512 * NW);     // DMA instructions per wave and tile
  static constexpr int CPR = (KMAJOR ? BK : R) / 8; // chunks per LDS row
  static constexpr int RPI = 64 / CPR;              // LDS rows per instruction
  static constexpr int SWD = 16 / CPR;              // KMAJOR: rows of one swizzle
  static_assert(L * 512 * NW == R * BK && (KMAJOR || R >= 128), "whole instructions; four groups of columns");
  const char* base;   // the tile's first element
  long step;          // bytes per k-tile
  uint32_t off[L];    // per-lane byte offsets within a k-tile
  uint32_t ld2;
  // first of `rows` rows: those past the end are clamped (KMAJOR: one by one, else in chunks of 8)
  __device__ __forceinline__ void init(const bf16* p, long ld, int first, int rows, int wave, int lane) {
    ld2 = (uint32_t)ld * 2;
    base = uniform_ptr(reinterpret_cast<const char*>(KMAJOR ? p + (long)first * ld : p + first));
    step = KMAJOR ? BK * 2 : ld * (BK * 2);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int r = (i * NW + wave) * RPI + lane / CPR, pos = lane % CPR;
      if constexpr (KMAJOR) off[i] = (uint32_t)min(r, rows - 1 - first) * ld2 + (pos ^ (r / SWD % CPR)) * 16;
      else off[i] = (uint32_t)r * ld2 + min(pos ^ ((r & 3) << 2), (rows - first + 7) / 8 - 1) * 16;
    }
  }
  // instruction i of k-tile kt; left: k of this tile that the operand has (BK: all), past them come zeros (KMAJOR) or the last one again.
  // Zeros are there once the wave has waited for its LDS operations, as it does for the DMA.
  __device__ __forceinline__ void dma(int i, int kt, int left, uint32_t lds, int wave, int wave_u, int lane) const {
    uint32_t o = off[i];
    if (left < BK) {
      if constexpr (KMAJOR) {
        int at = lane;
        asm volatile("" : "+v"(at));  // worked out here, not kept over the products
        if ((at % CPR ^ (((i * NW + wave_u) * RPI + at / CPR) / SWD % CPR)) >= left / 8) {
          lds_zero16(lds + (i * NW + wave_u) * 1024 + at * 16);
          return;
        }
      } else {
        o -= max(0, (i * NW + wave) * RPI + lane / CPR - (left - 1)) * ld2;
      }
    }
    dma16_m0(base + (long)kt * step, o, lds + (i * NW + wave_u) * 1024);
  }
};

// Fragments of F blocks of 32 rows from first row r0 of the tile in LDS
template <int R, int BK, int F, bool KMAJOR>
struct Frags {
  uint32_t at[KMAJOR ? 1 : F];
  __device__ __forceinline__ void init(int r0, int lane) {
    if constexpr (KMAJOR) {
      at[0] = (r0 + (lane & 31)) * (BK * 2);
    } else {
      const int g = lane >> 4, r = lane & 15;
#pragma unroll
      for (int i = 0; i < F; ++i)
        at[i] = (8 * (g >> 1) + (r >> 2)) * (R * 2) + (((r0 / 32 + i) ^ (r >> 2)) * 4 + 2 * (g & 1) + ((r & 3) >> 1)) * 16 + (r & 1) * 8;
    }
  }
  __device__ __forceinline__ void read(const char* tile, int ks, int lane, bf16x8 (&f)[F]) const {
    if constexpr (KMAJOR) {
      constexpr int CPR = BK / 8;
      const char* p = tile + at[0] + 16 * ((2 * ks + (lane >> 5)) ^ ((lane & 31) / (16 / CPR) % CPR));
#pragma unroll
      for (int i = 0; i < F; ++i) f[i] = *reinterpret_cast<const bf16x8*>(p + i * 32 * (BK * 2));
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

struct VocabProduct {
  const bf16* A; long lda;
  const bf16* B; long ldb;
  int M, N;        // M: of dw (the logits and dh have the rows that count)
  int K;           // k of the logits (d) and of dh (V)
  int slots;       // dh, dw: workgroups of one round
};
// Of k to a share.  2^18 terms are 2^14 additions in a chain; if each leans by half a step of fp32, that is 2^-11 of the sum, below the
// rounding to bf16.
constexpr int MM_LEAST = 512, MM_LONGEST = 1 << 18;

// four columns of a row of dw, summed over the pieces, which are in dloss' unit
__device__ __forceinline__ void add_dw(const VocabArgs& a, int m, int n, float unit, f32x4 v) {
  f32x4* o = reinterpret_cast<f32x4*>(a.dw_acc + (long)m * a.ld_acc + n);
  if (!a.first) v += *o;
  if (!a.last) {
    *o = v;
    return;
  }
  *reinterpret_cast<uint2*>(static_cast<bf16*>(a.dw) + (long)m * a.lddw + n) =
      make_uint2(f2bf2(v[0] * unit, v[1] * unit), f2bf2(v[2] * unit, v[3] * unit));
}

// Workgroups stay: one round of the GPU, each over its tiles.  While a tile is stored the first k-tiles of the next are
// on their way, and its stores drain under the next one's products (2048 x 32000 logits, d 4096: 1.08 times less than a workgroup per tile).
// So the epilogue has no LDS but 4 KB per wave beside the stages, and no barrier: each wave sends its 32 x 32 blocks
// through its own, in 16-byte pieces at c ^ row % 8, and stores whole 128-byte lines (64-byte runs: 2048 x 32000 logits 480 us instead of
// 452); the logits' statistics are per wave too, one (maximum, sum) for BN / WN columns.
template <int BM, int BN, int WM, int WN>
constexpr int MM_LDS = 2 * (BM + BN) * 64 * 2 + WM * WN * 4096;
template <int BM, int BN, int WM, int WN, bool KA, bool KB, Prod E>
__global__ __launch_bounds__(64 * WM * WN, 2) void vocab_mm_k(VocabArgs a, VocabProduct p) {
  __shared__ __attribute__((aligned(1024))) char smem[MM_LDS<BM, BN, WM, WN>];
  auto wg = [] { return blockIdx.x; };
  auto wgs = [] { return gridDim.x; };
#include "vocab_mm_body.h"
}

// both gradients, dh by the first n_dh workgroups
template <bool KA, Prod E>
__device__ __forceinline__ void vocab_mm_grad(VocabArgs a, VocabProduct p, char* smem, int number, int of) {
  auto wg = [=] { return number; };
  auto wgs = [=] { return of; };
  constexpr int BM = 128, BN = 128, WM = 2, WN = 2;
  constexpr bool KB = false;
#include "vocab_mm_body.h"
}
__global__ __launch_bounds__(256) void vocab_mm_grads_k(VocabArgs a, VocabProduct dh, VocabProduct dw, int n_dh) {
  __shared__ __attribute__((aligned(1024))) char smem[MM_LDS<128, 128, 2, 2>];
  if ((int)blockIdx.x < n_dh) vocab_mm_grad<true, Prod::Dh>(a, dh, smem, blockIdx.x, n_dh);
  else vocab_mm_grad<false, Prod::Dw>(a, dw, smem, blockIdx.x - n_dh, gridDim.x - n_dh);
}

// dh or dw of a piece from its shares; tiles are bt x bt.  G threads take every G-th share of eight columns each, and are
// added up in their order.
template <Prod E, int G>
__global__ __launch_bounds__(256) void vocab_shares_k(VocabArgs a, VocabProduct p, int bt) {
  __shared__ float red[G > 1 ? 256 : 1][9];
  const int cnt = piece_rows(a), M = E == Prod::Dw ? p.M : cnt, K = E == Prod::Dw ? cnt : p.K;
  const int cols = p.N / 8, g = threadIdx.x % G, i = blockIdx.x * (256 / G) + threadIdx.x / G, m = i / cols, n = i % cols * 8;
  const int ntn = (p.N + bt - 1) / bt, tiles = (M + bt - 1) / bt * ntn, splits = tiles ? k_shares(p.slots, tiles, K, MM_LEAST, MM_LONGEST) : 1;
  if (splits == 1) return;
  const bool in = m < M;
  float v[8] = {};
  if (in) {
    const float* q = a.shares + (long)(m / bt * ntn + n / bt) * bt * bt + (m % bt) * bt + n % bt;
#pragma unroll 4
    for (int s = g; s < splits; s += G) {
      float x[8];
      *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(q + (long)s * tiles * bt * bt);
      *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(q + (long)s * tiles * bt * bt + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
  }
  if constexpr (G > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) red[threadIdx.x][e] = v[e];
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int o = 1; o < G; ++o)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += red[threadIdx.x + o][e];
  }
  if (!in) return;
  if constexpr (E == Prod::Dh) {
    float c[8];
    unpack_frag(*reinterpret_cast<const bf16x8*>(p.B + (long)a.lab_c[a.row0 + m] * p.ldb + n), c);
    const float left = row_left(a, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += left * c[e];
  }
  const float unit = dloss_unit(a);
  if (E == Prod::Dw && !(a.first && a.last)) {
    add_dw(a, m, n, unit, f32x4{v[0], v[1], v[2], v[3]});
    add_dw(a, m, n + 4, unit, f32x4{v[4], v[5], v[6], v[7]});
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= unit;
  bf16* o = E == Prod::Dh ? static_cast<bf16*>(a.dh) + (long)a.idx[a.row0 + m] * a.lddh : static_cast<bf16*>(a.dw) + (long)m * a.lddw;
  *reinterpret_cast<bf16x8*>(o + n) = pack_frag(v);
}

// ---------------------------------------------------------------- few rows
// Statistics of the logits of up to 32 rows: w is read once, by far the most of the work, and straight into registers. A
// wave makes 16 classes at a time by MFMA 16x16x32, its A operand 16 rows of w, B the rows of h, kept in LDS for all
// waves.  STEPS loads of 1 KB are in flight per wave while the last STEPS are multiplied, over the ends of the blocks of classes
// too.  Where classes are few, KS waves share a block's k.  One (maximum, sum, place) per row and workgroup is left.
template <int NB, int KS, int LDSB>
__global__ __launch_bounds__(512, LDSB > 65536 ? 2 : 4) void vocab_few_k(VocabArgs a, int pitch) {
  constexpr int STEPS = 8, KC = 32 * STEPS, NW = 8, GRP = NW / KS;  // GRP groups of KS waves
  __shared__ __attribute__((aligned(16))) char smem[LDSB];
  __shared__ float red[NW][NB][16 * 17];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = wave / KS, ks = wave % KS;
  const int chunks = (a.d + KC - 1) / KC, mine = (chunks - ks + KS - 1) / KS;  // of k: ks, ks + KS, ..
  const bf16* h = static_cast<const bf16*>(a.h);
  for (int i = tid; i < a.n * (pitch / 16); i += 512) {
    const int r = i / (pitch / 16), k = i % (pitch / 16) * 8;
    *reinterpret_cast<uint4*>(smem + r * pitch + k * 2) =
        k < a.d ? *reinterpret_cast<const uint4*>(h + (long)r * a.ldh + k) : make_uint4(0, 0, 0, 0);
  }
  const int blocks = (a.V + 15) / 16, stride = gridDim.x * GRP;
  const int first = grp * gridDim.x + blockIdx.x;  // few blocks go to as many workgroups
  int blk = first, c = 0;                          // what is loaded next
  // KS waves meet at barriers, so all groups of a workgroup go as many rounds
  const int rounds = max(0, (blocks - (KS > 1 ? (int)blockIdx.x : first) + stride - 1) / stride);
  const bf16* w = static_cast<const bf16*>(a.w);
  bf16x8 x[2][STEPS];
  auto load = [&](bf16x8 (&y)[STEPS]) {
    const bf16* row = w + (long)min(blk * 16 + l16, a.V - 1) * a.ldw;
    const int k0 = (ks + c * KS) * KC + g4 * 8;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {  // past d: the row's first elements, which mul leaves out
      const int k = k0 + s * 32;
      y[s] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(row + (k < a.d ? k : 0)));
    }
    if (++c >= mine) {
      c = 0;
      blk += stride;
    }
  };
  const char* hb[NB];
  int lab[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int r = b * 16 + l16;
    hb[b] = smem + min(r, a.n - 1) * pitch + g4 * 16;
    lab[b] = a.labels && r < a.n ? a.labels[r] : -1;
  }
  f32x4 acc[NB];
  Peak p[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    p[b] = Peak{-INFINITY, 0.f, INT32_MAX};
  }
  __syncthreads();
  // the four logits of this lane, classes v .. v + 3, into its running statistics
  auto take = [&](int b, int v, const f32x4& s) {
    float m = p[b].m;
    int at = p[b].at;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < a.V) {
        if (s[e] > m) {
          m = s[e];
          at = v + e;
        }
        if (v + e == lab[b]) a.target[b * 16 + l16] = s[e];
      }
    const float z = m == -INFINITY ? 0.f : m;
    float l = p[b].l * exp_below(p[b].m - z);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < a.V) l += exp_below(s[e] - z);
    p[b] = Peak{m, l, at};
  };
  auto mul = [&](const bf16x8 (&y)[STEPS], int kc) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bf16x8 part = kc * KC + s * 32 + g4 * 8 < a.d ? y[s] : zero_frag();
#pragma unroll
      for (int b = 0; b < NB; ++b)
        acc[b] = mfma16(part, *reinterpret_cast<const bf16x8*>(hb[b] + kc * (KC * 2) + s * 64), acc[b]);
    }
  };
  const int steps = rounds * mine;
  int done = 0, at_blk = first;  // what is multiplied
  auto finish = [&] {
    if (++done < mine) return;
    done = 0;
    if constexpr (KS > 1) {  // the shares, in their order
      __syncthreads();
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[wave][b][(4 * g4 + e) * 17 + l16] = acc[b][e];
      __syncthreads();
    }
    if (ks == 0 && at_blk < blocks) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4 s = acc[b];
        if constexpr (KS > 1)
#pragma unroll
          for (int q = 1; q < KS; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += red[wave + q][b][(4 * g4 + e) * 17 + l16];
        take(b, at_blk * 16 + 4 * g4, s);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    at_blk += stride;
  };
  if constexpr (KS > 1) {
    // every wave of the workgroup passes the same number of barriers: a round each
    for (int r = 0; r < rounds; ++r) {
      const int have = blk < blocks ? mine : 0;
      if (have) load(x[0]);
      for (int i = 0; i < have; i += 2) {
        if (i + 1 < have) load(x[1]);
        mul(x[0], ks + i * KS);
        if (i + 1 < have) {
          if (i + 2 < have) load(x[0]);
          mul(x[1], ks + (i + 1) * KS);
        }
      }
      done = mine;
      finish();
    }
  } else {
    if (steps) load(x[0]);
    for (int i = 0; i < steps; i += 2) {
      if (i + 1 < steps) load(x[1]);
      mul(x[0], done);
      finish();
      if (i + 1 < steps) {
        if (i + 2 < steps) load(x[0]);
        mul(x[1], done);
        finish();
      }
    }
  }
  // lanes of a row, then waves
  __syncthreads();
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) p[b] = join(p[b], Peak{__shfl_xor(p[b].m, o), __shfl_xor(p[b].l, o), __shfl_xor(p[b].at, o)});
    if (lane < 16) {
      red[wave][b][l16 * 3] = p[b].m;
      red[wave][b][l16 * 3 + 1] = p[b].l;
      red[wave][b][l16 * 3 + 2] = __int_as_float(p[b].at);
    }
  }
  __syncthreads();
  if (tid < a.n) {
    Peak q{-INFINITY, 0.f, INT32_MAX};
    for (int v = 0; v < NW; ++v) {
      const float* r = red[v][tid / 16] + tid % 16 * 3;
      q = join(q, Peak{r[0], r[1], __float_as_int(r[2])});
    }
    a.part[(long)tid * a.tiles + blockIdx.x] = make_float2(q.m, q.l);
    if (a.part_at) a.part_at[(long)tid * a.tiles + blockIdx.x] = min(q.at, a.V - 1);
  }
}

// rows of h in LDS, whose 16-byte pieces of one k lie in different banks
static int few_pitch(int d) { return (d + 255) / 256 * 512 + 16; }
// up to 32 rows that fit the LDS beside the partial sums: 0 if not, else the LDS that is taken
static int few_lds(int rows, int d) {
  const long bytes = (long)rows * few_pitch(d);
  return rows > 32 || bytes > 131072 ? 0 : bytes > 49152 ? 131072 : 49152;
}
bool vocab_few(int rows, int d) { return few_lds(rows, d) > 0; }
int vocab_few_wgs(int rows, int d) { return few_lds(rows, d) > 65536 ? 256 : 512; }

template <int NB, int KS>
static void go_few(const VocabArgs& a, hipStream_t s) {
  const int pitch = few_pitch(a.d);
  if (few_lds(a.n, a.d) > 65536) RG_LAUNCH((vocab_few_k<NB, KS, 131072>), dim3(a.tiles), dim3(512), 0, s, a, pitch);
  else RG_LAUNCH((vocab_few_k<NB, KS, 49152>), dim3(a.tiles), dim3(512), 0, s, a, pitch);
}
void launch_vocab_few_bf16(const VocabArgs& a, hipStream_t s) {
  // a block of 16 classes to every wave where there are as many, else their k dealt to four
  const bool share = (a.V + 15) / 16 < a.tiles * 8 / 2;
  if (a.n <= 16) share ? go_few<1, 4>(a, s) : go_few<1, 1>(a, s);
  else share ? go_few<2, 4>(a, s) : go_few<2, 1>(a, s);
}

static int tiles_of(int x, int t) { return (x + t - 1) / t; }
constexpr int mm_slots(int tile) { return tile == 256 ? 256 : 512; }  // one or two workgroups per CU

// the workgroups that a product takes, and whether any of its tiles may be in shares
struct Grid {
  unsigned wgs;
  bool shares;
};
template <Prod E>
static Grid mm_grid(const VocabArgs& a, VocabProduct& p, int bm, int bn) {
  constexpr bool shared = E == Prod::Dh || E == Prod::Dw;
  const int M = E == Prod::Dw ? p.M : a.rows, K = E == Prod::Dw ? a.rows : p.K;
  const int tiles = tiles_of(M, bm) * tiles_of(p.N, bn);
  p.slots = mm_slots(bn);
  // dw's tiles are known here; dh's are of the rows that count, so one tile may have as many shares as there can be
  const int most = !shared ? 1 : k_shares(p.slots, E == Prod::Dw ? tiles : 1, K, MM_LEAST, MM_LONGEST);
  const long wgs = (long)tiles * most;
  return {(unsigned)(wgs < p.slots ? wgs : p.slots), most > 1};
}
template <Prod E>
static void mm_shares(const VocabArgs& a, const VocabProduct& p, int bt, hipStream_t s) {
  // one thread per eight columns where those are many, else eight
  const long items = (long)(E == Prod::Dw ? p.M : a.rows) * (p.N / 8);
  if (items >= 16384) RG_LAUNCH((vocab_shares_k<E, 1>), dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, a, p, bt);
  else RG_LAUNCH((vocab_shares_k<E, 8>), dim3((unsigned)((items + 31) / 32)), dim3(256), 0, s, a, p, bt);
}
template <int BT, int WM, int WN, bool KA, bool KB, Prod E, int BM = BT>
static void go(const VocabArgs& a, VocabProduct p, hipStream_t s) {
  const Grid g = mm_grid<E>(a, p, BM, BT);
  RG_LAUNCH((vocab_mm_k<BM, BT, WM, WN, KA, KB, E>), dim3(g.wgs), dim3(64 * WM * WN), 0, s, a, p);
  if constexpr (E == Prod::Dh || E == Prod::Dw) {
    static_assert(BM == BT, "shares are of square tiles");
    if (g.shares) mm_shares<E>(a, p, BT, s);
  }
}

// Rows and columns of the logits' tiles, by the rounds of the GPU that they take: f + r K / 64 us each, fitted to 333 to 4096
// rows, 20000 to 50000 classes, d 768 to 4096.  256 x 256 has the best rate, 192 x 256 the rows that 256 leaves over (333 x 32000, d 4096: 107 us
// against 114), 128 x 128, two to a CU, the shortest epilogue.
enum class LogitsTile { T256, T192, T128 };
static LogitsTile logits_tile(int rows, int d, int V) {
  const int k = tiles_of(d, 64);
  // up to 2^31 tiles
  auto rounds = [=](int bm, int bn, int slots) { return ((long)tiles_of(rows, bm) * tiles_of(V, bn) + slots - 1) / slots; };
  const float t256 = rounds(256, 256, 256) * (8.f + 1.7f * k);
  const float t192 = rounds(192, 256, 256) * (8.f + 1.32f * k);
  const float t128 = rounds(128, 128, 512) * (7.f + 1.05f * k);
  return t256 <= t192 && t256 <= t128 ? LogitsTile::T256 : t192 <= t128 ? LogitsTile::T192 : LogitsTile::T128;
}
int vocab_mm_bn(int rows, int d, int V) { return logits_tile(rows, d, V) == LogitsTile::T256 ? 128 : 64; }  // a wave's columns
static bool wide_dh(int rows, int d) { return rows > 128 && tiles_of(rows, 256) * tiles_of(d, 256) >= 128; }
static bool wide_dw(int rows, int d, int V) { return rows > 128 && tiles_of(V, 256) * tiles_of(d, 256) >= 128; }

size_t vocab_share_bytes(int rows, int R, int d, int V) {
  auto bytes = [](int t, long tiles, int K) {
    // whichever rows count: shares times tiles are at most a round of workgroups, but for the chains
    const long by_slots = tiles * k_shares(mm_slots(t), 1, K, MM_LEAST, MM_LONGEST), chains = (K + (long)MM_LONGEST - 1) / MM_LONGEST;
    const long most = by_slots < mm_slots(t) ? by_slots : mm_slots(t), cut = chains > 1 ? tiles * chains : 0;
    return (size_t)(most > cut ? most : cut) * t * t * 4;
  };
  const int th = wide_dh(rows, d) ? 256 : 128, tw = wide_dw(rows, d, V) ? 256 : 128;
  const size_t h = bytes(th, (long)tiles_of(R, th) * tiles_of(d, th), V);
  const size_t w = bytes(tw, (long)tiles_of(V, tw) * tiles_of(d, tw), R);
  return h > w ? h : w;
}

void launch_vocab_logits_bf16(const VocabArgs& a, bool keep, hipStream_t s) {
  VocabProduct p{};
  p.A = static_cast<const bf16*>(a.hc) + (long)a.row0 * a.dp;
  p.lda = a.dp;
  p.B = static_cast<const bf16*>(a.w);
  p.ldb = a.ldw;
  p.N = a.V;
  p.K = a.d;
  switch (logits_tile(a.n, a.d, a.V)) {
    case LogitsTile::T256:
      if (keep) go<256, 4, 2, true, true, Prod::Logits>(a, p, s);
      else go<256, 4, 2, true, true, Prod::Stats>(a, p, s);
      break;
    case LogitsTile::T192:
      if (keep) go<256, 2, 4, true, true, Prod::Logits, 192>(a, p, s);
      else go<256, 2, 4, true, true, Prod::Stats, 192>(a, p, s);
      break;
    case LogitsTile::T128:
      if (keep) go<128, 2, 2, true, true, Prod::Logits>(a, p, s);
      else go<128, 2, 2, true, true, Prod::Stats>(a, p, s);
      break;
  }
}
void launch_vocab_grads_bf16(const VocabArgs& a, hipStream_t s) {
  VocabProduct h{}, w{};
  h.A = w.A = static_cast<const bf16*>(a.logits);
  h.lda = w.lda = a.Vp;
  h.B = static_cast<const bf16*>(a.w);
  h.ldb = a.ldw;
  w.B = static_cast<const bf16*>(a.hc) + (long)a.row0 * a.dp;
  w.ldb = a.dp;
  h.N = w.N = a.d;
  h.K = w.M = a.V;
  const bool bh = wide_dh(a.n, a.d), bw = wide_dw(a.n, a.d, a.V);
  // Small gradients are bound by their latency: both in one launch where dw leaves the shares' place to dh (whole calls of 500 x 1000, d 256:
  // 31 us instead of 40; 64 x 8000, d 1024: 46 and 53; 2000 x 12000, d 256: 116 both ways)
  if (a.dh && a.dw && !bh && !bw) {
    const Grid gh = mm_grid<Prod::Dh>(a, h, 128, 128), gw = mm_grid<Prod::Dw>(a, w, 128, 128);
    if (!gw.shares) {
      RG_LAUNCH(vocab_mm_grads_k, dim3(gh.wgs + gw.wgs), dim3(256), 0, s, a, h, w, (int)gh.wgs);
      if (gh.shares) mm_shares<Prod::Dh>(a, h, 128, s);
      return;
    }
  }
  if (a.dh) bh ? go<256, 4, 2, true, false, Prod::Dh>(a, h, s) : go<128, 2, 2, true, false, Prod::Dh>(a, h, s);
  if (a.dw) bw ? go<256, 4, 2, false, false, Prod::Dw>(a, w, s) : go<128, 2, 2, false, false, Prod::Dw>(a, w, s);
}

}  // namespace rg
