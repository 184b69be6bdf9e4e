// The vocabulary head with softmax cross entropy: s = h w^T over w [V][d], and from
// it the loss of every row, the gradients of h and w, or the likeliest column.
//
//   lse_n = log sum_v exp s_nv          loss_n = lse_n - s[n][label]
//   P_nv  = g_n (exp(s_nv - lse_n) - [v = label])
//   dh    = P w                         dw = P^T h
//
// A row counts when its label is in [0, V).  Rows that count are gathered first, in
// order, so that the products run over them alone (masked-token training labels one
// position in seven) and whatever stands in the others reaches nothing.  The number is
// known on the device only: grids are sized for all rows, and tiles past it end at once.
//
// The logits of a piece of the rows are held while they are needed, in fp32 or, with bf16 tensors, in fp16 below their
// tile's maximum.  Pieces of the vocabulary would need no more memory, but lse needs all columns before P has any: the product h w^T would run twice, 8 n V d
// operations instead of 6.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "vocab_peak.h"

namespace rg {

// ---------------------------------------------------------------- rows that count
constexpr int PICK_ROWS = 4;       // of h per workgroup, one per wave
constexpr int PICK_DIRECT = 16384; // labels that a workgroup counts by itself; beyond, blocks of 1024 are counted first

__device__ __forceinline__ bool counts(const VocabArgs& a, int lab) { return lab >= 0 && lab < a.V; }

// sum over the 256 threads of a workgroup; red: 4 ints
__device__ __forceinline__ int wg_sum(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0] + red[1] + red[2] + red[3];
  __syncthreads();
  return v;
}

__global__ __launch_bounds__(256) void vocab_count_k(VocabArgs a) {
  __shared__ int red[4];
  int v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = blockIdx.x * 1024 + i * 256 + threadIdx.x;
    v += n < a.n && counts(a, a.labels[n]) ? 1 : 0;
  }
  v = wg_sum(v, red);
  if (threadIdx.x == 0) a.block_count[blockIdx.x] = v;
}

// a row whose pieces are not aligned, zeros from d to dp: eight elements in flight per lane
template <typename T>
__device__ __forceinline__ void copy_row(T* dst, const T* src, int d, int dp, int lane) {
  for (int k0 = lane; k0 < dp; k0 += 512) {
    T x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = src[min(k0 + j * 64, d - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k0 + j * 64 < dp) dst[k0 + j * 64] = k0 + j * 64 < d ? x[j] : T(0);
  }
}

// A stable compaction: hc[i] is the i-th row that counts, zeros past d; without labels, every row.  A workgroup
// takes PICK_ROWS rows of h and counts the labels before them.  The results of rows that do not count are written here.
template <typename T>
__global__ __launch_bounds__(256) void vocab_pick_k(VocabArgs a, bool wide) {
  __shared__ int red[4];
  const int r0 = blockIdx.x * PICK_ROWS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = r0;
  if (a.labels) {
    int v = 0, n = threadIdx.x;
    if (a.block_count) {
      for (int b = threadIdx.x; b < r0 / 1024; b += 256) v += a.block_count[b];
      n += r0 / 1024 * 1024;
    }
    for (; n < r0; n += 256) v += counts(a, a.labels[n]) ? 1 : 0;
    before = wg_sum(v, red);
  }
  for (int i = wave; i < PICK_ROWS && r0 + i < a.n; i += 4) {
    const int n = r0 + i;
    int at = n;
    if (a.labels) {
      const int lab = lane <= i ? a.labels[r0 + lane] : -1;  // the rows up to this one
      const uint64_t vote = __ballot(lane <= i && counts(a, lab));
      const int mine = __shfl(lab, i);
      at = before + __popcll(vote) - 1;
      if (n == a.n - 1 && lane == 0) *a.n_counted = at + 1;
      if (!counts(a, mine)) {
        if (lane == 0) a.loss[n] = a.lse[n] = 0.f;
        if (a.dh) {
          T* dst = static_cast<T*>(a.dh) + (long)n * a.lddh;
          if constexpr (sizeof(T) == 2) {
            for (int k = lane * 8; k < a.d; k += 512) *reinterpret_cast<uint4*>(dst + k) = make_uint4(0, 0, 0, 0);
          } else {
            for (int k = lane; k < a.d; k += 64) dst[k] = T(0);
          }
        }
        continue;
      }
      if (lane == 0) {
        a.idx[at] = n;
        a.lab_c[at] = mine;
        if (a.dloss) a.g_c[at] = a.dloss[n];
      }
    }
    const T* src = static_cast<const T*>(a.h) + (long)n * a.ldh;
    T* dst = static_cast<T*>(a.hc) + (long)at * a.dp;
    constexpr int E = 16 / sizeof(T);
    if (wide) {
      for (int k0 = lane * E; k0 < a.dp; k0 += 512 * E) {  // eight pieces in flight
        uint4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int k = k0 + j * 64 * E;
          x[j] = k < a.d ? *reinterpret_cast<const uint4*>(src + k) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int k = k0 + j * 64 * E;
          if (k < a.dp) *reinterpret_cast<uint4*>(dst + k) = x[j];
        }
      }
    } else {
      copy_row(dst, src, a.d, a.dp, lane);
    }
  }
}

// ---------------------------------------------------------------- products in fp32
// C[m][n] = sum_k A(m, k) B(n, k) by MFMA 32x32x2 f32.  KA: A is [M][K], else [K][M]; KB likewise.  The logits' tiles leave
// (maximum, sum); dh's k (the vocabulary) is dealt to several workgroups where its tiles are few.
//
// Sums over a vocabulary are long: 300,000 terms in one chain of the matrix unit were off by 9 sqrt(n) roundings. So
// a chain ends after LONG terms, and the chains are added up.
struct F32Product {
  const float* A; long lda;
  const float* B; long ldb;
  int M, N, K;     // M of dw, k of the logits and of dh; the others are the rows that count
};
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));  // w may lie anywhere: a load of four floats asks for 4 bytes
// Shares of the k of bt x bt tiles of dh or dw, for 512 workgroups, two to a CU.  Wide tiles that come to little more than one
// per CU take three each, as most CUs would wait for those with two (1189 x 4070 of 2786: 289 us and 11 more to add them up, 400 unshared).
constexpr int F32_SLOTS = 512;
__host__ __device__ inline int f32_splits(int bt, int tiles, int K) {
  const int slots = bt == 128 && tiles > 256 && tiles * 3 <= 2 * F32_SLOTS ? 2 * F32_SLOTS : F32_SLOTS;
  return k_shares(slots, tiles, K, 512, 1 << 30);  // chains are cut in the kernels
}

template <Prod E>
__device__ __forceinline__ void f32_gradient(const VocabArgs& a, int m, int n, float v) {
  if constexpr (E == Prod::Dh) {
    static_cast<float*>(a.dh)[(long)a.idx[a.row0 + m] * a.lddh + n] = v;
  } else {
    float* o = static_cast<float*>(a.dw) + (long)m * a.lddw + n;
    *o = a.first ? v : *o + v;
  }
}
// the tile's sums, cf[row * CP + column], into what the product is for
template <int BT, int CP, Prod E>
__device__ __forceinline__ void f32_epilogue(const VocabArgs& a, const F32Product& p, const float* cf, int M, int N, int m0, int n0,
                                             int tile, int split, int splits, int tiles) {
  const int tid = threadIdx.x;
  if constexpr (E == Prod::Stats || E == Prod::Logits) {
    constexpr int TPR = 256 / BT, CPT = BT / TPR;  // threads per row, columns of each: t, t + TPR, ..
    const int row = tid / TPR, t = tid % TPR, m = m0 + row;
    const int lab = a.lab_c && m < M ? a.lab_c[a.row0 + m] : -1;
    Peak q{-INFINITY, 0.f, INT32_MAX};
#pragma unroll 8
    for (int i = 0; i < CPT; ++i) {
      const int c = i * TPR + t;
      const float s = n0 + c < N ? cf[row * CP + c] : -INFINITY;
      if (s > q.m) {
        q.m = s;
        q.at = n0 + c;
      }
      if (n0 + c == lab) a.target[a.row0 + m] = s;
    }
    const float z = q.m == -INFINITY ? 0.f : q.m;
#pragma unroll 8
    for (int i = 0; i < CPT; ++i) {
      const int c = i * TPR + t;
      if (n0 + c < N) q.l += exp_below(cf[row * CP + c] - z);
    }
#pragma unroll
    for (int o = 1; o < TPR; o <<= 1) q = join(q, Peak{__shfl_xor(q.m, o), __shfl_xor(q.l, o), __shfl_xor(q.at, o)});
    if (m < M && t == 0) {
      a.part[(long)m * a.tiles + n0 / BT] = make_float2(q.m, q.l);
      if (a.part_at) a.part_at[(long)m * a.tiles + n0 / BT] = min(q.at, N - 1);
    }
    if constexpr (E == Prod::Logits)
      for (int i = tid; i < BT * BT / 4; i += 256) {
        const int r = i / (BT / 4), c = i % (BT / 4) * 4;
        if (m0 + r < M && n0 + c < a.Vp)
          *reinterpret_cast<float4*>(static_cast<float*>(a.logits) + (long)(m0 + r) * a.Vp + n0 + c) = *reinterpret_cast<const float4*>(cf + r * CP + c);
      }
  } else {
    float* part = a.shares + ((long)split * tiles + tile) * (BT * BT);
    for (int i = tid; i < BT * BT; i += 256) {
      const int r = i / BT, c = i % BT, m = m0 + r, n = n0 + c;
      if (m >= M || n >= N) continue;
      const float v = cf[r * CP + c];
      if (splits > 1) part[i] = v;
      else f32_gradient<E>(a, m, n, v);
    }
  }
}

// 128 x 128 tiles, 32 k at a time: registers -> LDS, four waves of 64 x 64, two workgroups per CU.  LDS keeps [k][row], rows of odd k
// turned by 32 columns, so that the two k of an MFMA lie in different banks.  The loop has no branch: rows and k past the ends read
// the last ones again.  Such rows are not stored, and such k meet zeros of A: hc and P are padded with them to whole tiles of
// 64.  In the logits they are zeros of w too, as an infinity read again would make a NaN.  A piece of B that reaches past the end
// of its row is read from where it ends there, and moved (1189 x 2786, d 4070: 309 us of logits, 300 at d 4096; single loads 508).  d >= 4.
// 4096 x 16000, d 2048: 132 TF (a tile of 16 k with guarded loads: 115; torch.mm 154).
// PADDED: A, which has whole tiles of k
template <bool KM, bool PADDED>
struct F32Operand {
  const char* base;  // uniform: three elements before the tile's first
  long step;         // bytes per 32 k
  uint32_t off[4];   // of this thread's four pieces of four
  int past;          // how far a piece was moved back to end with its row (not KM)
  uint32_t ld4;
  __device__ __forceinline__ void init(const float* X, long ld, int r0, int rows, int k0) {
    const int tid = threadIdx.x;
    ld4 = (uint32_t)ld * 4;
    base = reinterpret_cast<const char*>((KM ? X + (long)r0 * ld + k0 : X + (long)k0 * ld + r0) - 3);
    step = KM ? 128 : ld * 128;
    const int c = min((tid & 31) * 4, rows - 4 - r0);  // -3 at least
    past = KM || PADDED ? 0 : (tid & 31) * 4 - c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KM) off[i] = (uint32_t)min(tid & 127, rows - 1 - r0) * ld4 + ((tid >> 7) * 16 + 4 * i + 3) * 4;
      else off[i] = (uint32_t)((tid >> 5) + 8 * i) * ld4 + (c + 3) * 4;
    }
  }
  // tile t from k0 on; left: k of it that there are
  __device__ __forceinline__ void fetch(int t, int left, f32x4 (&v)[4]) const {
    const char* b = base + t * step;
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t o = off[i];
      int move = past;
      if (!PADDED && left < 32) {
        if constexpr (KM) {
          move = max(0, (tid >> 7) * 16 + 4 * i - (left - 4));
          o -= move * 4;
        } else {
          o -= max(0, (tid >> 5) + 8 * i - (left - 1)) * ld4;
        }
      }
      v[i] = *reinterpret_cast<const f32x4_a4*>(b + o);
      if (!PADDED && (!KM || left < 32)) {
        if (move & 2) v[i].x = v[i].z, v[i].y = v[i].w;
        if (move & 1) v[i].x = v[i].y, v[i].y = v[i].z, v[i].z = v[i].w;
        if constexpr (KM) {
          const int k = (tid >> 7) * 16 + 4 * i;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][e] = k + e < left ? v[i][e] : 0.f;
        }
      }
    }
  }
};
template <bool KM>
__device__ __forceinline__ void f32_put(float* s, const f32x4 (&v)[4]) {
  const int tid = threadIdx.x;
  if constexpr (KM) {
    float* even = s + (tid >> 7) * 16 * 128 + (tid & 127);
    float* odd = s + (tid >> 7) * 16 * 128 + ((tid & 127) ^ 32);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      even[(4 * i) * 128] = v[i].x;
      odd[(4 * i + 1) * 128] = v[i].y;
      even[(4 * i + 2) * 128] = v[i].z;
      odd[(4 * i + 3) * 128] = v[i].w;
    }
  } else {
    // rows 8 i + tid / 32, of the parity of tid / 32
    float* d = s + (tid >> 5) * 128 + (((tid & 31) * 4) ^ (32 * ((tid >> 5) & 1)));
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(d + i * 8 * 128) = v[i];
  }
}

template <bool KA, bool KB, Prod E>
__global__ __launch_bounds__(256, 2) void vocab_f32_k(VocabArgs a, F32Product p) {
  constexpr int BT = 128, BK = 32, CP = BT + 4, LONG = 1024, TILE = BK * BT;
  __shared__ __attribute__((aligned(16))) float smem[BT * CP];
  static_assert(4 * TILE <= BT * CP, "two buffers");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
  const int cnt = piece_rows(a);
  const int M = E == Prod::Dw ? p.M : cnt, N = p.N;
  const int tn = (N + BT - 1) / BT, tiles = (M + BT - 1) / BT * tn;
  const int Kall = E == Prod::Dw ? cnt : p.K;
  const int splits = (E == Prod::Dh || E == Prod::Dw) && tiles ? f32_splits(BT, tiles, Kall) : 1;
  if ((int)blockIdx.x >= tiles * splits) return;
  const int split = blockIdx.x / tiles;
  int tm, tc;
  vocab_tile<4>(blockIdx.x - split * tiles, (M + BT - 1) / BT, tn, tm, tc);
  const int tile = tm * tn + tc, m0 = tm * BT, n0 = tc * BT;
  const int nkt = (Kall + BK - 1) / BK, t0 = (int)((long)nkt * split / splits), t1 = (int)((long)nkt * (split + 1) / splits);
  // A is padded; what B has
  const int Mp = KA ? M : a.Vp;
  const int Nb = E == Prod::Dw ? a.dp : N;
  f32x16 acc[2][2], sum[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = sum[i][j][r] = 0.f;
  auto settle = [&] {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sum[i][j][r] += acc[i][j][r];
          acc[i][j][r] = 0.f;
        }
  };
  f32x4 ra[4], rb[4];
  F32Operand<KA, true> oa;
  F32Operand<KB, false> ob;
  auto fetch = [&](int t) {
    t = min(t, t1 - 1);
    oa.fetch(t - t0, 32, ra);
    ob.fetch(t - t0, Kall - t * BK, rb);
  };
  auto put = [&](int buf) {
    f32_put<KA>(smem + buf * 2 * TILE, ra);
    f32_put<KB>(smem + (buf * 2 + 1) * TILE, rb);
  };
  if (t0 < t1) {
    oa.init(p.A, p.lda, m0, Mp, t0 * BK);
    ob.init(p.B, p.ldb, n0, Nb, t0 * BK);
    fetch(t0);
    put(0);
    fetch(t0 + 1);
    __syncthreads();
    int buf = 0;
    const int half = lane >> 5, ca = (wm * 64 + (lane & 31)) ^ (32 * half), cb = (wn * 64 + (lane & 31)) ^ (32 * half);
    for (int t = t0; t < t1; ++t, buf ^= 1) {
      const float* sa = smem + buf * 2 * TILE + half * BT;
      const float* sb = sa + TILE;
      float fa[2][2], fb[2][2];
      auto read = [&](int kk, int at) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fa[at][i] = sa[kk * 2 * BT + (ca ^ (32 * i))];
          fb[at][i] = sb[kk * 2 * BT + (cb ^ (32 * i))];
        }
      };
      read(0, 0);
#pragma unroll
      for (int kk = 0; kk < BK / 2; ++kk) {
        if (kk + 1 < BK / 2) read(kk + 1, (kk + 1) & 1);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = mfma32_f32(fb[kk & 1][j], fa[kk & 1][i], acc[i][j]);
        if (kk == 7) put(buf ^ 1);
        if (kk == 8) fetch(t + 2);
      }
      if ((t - t0) % (LONG / BK) == LONG / BK - 1) settle();
      __syncthreads();
    }
    settle();
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(smem + (wm * 64 + i * 32 + (lane & 31)) * CP + wn * 64 + j * 32 + 8 * g + 4 * (lane >> 5)) =
            make_float4(sum[i][j][4 * g], sum[i][j][4 * g + 1], sum[i][j][4 * g + 2], sum[i][j][4 * g + 3]);
  __syncthreads();
  f32_epilogue<BT, CP, E>(a, p, smem, M, N, m0, n0, tile, split, splits, tiles);
}

// 32 x 32 tiles for small products, where what counts is the latency of one chain on many CUs: fragments go from memory straight
// to registers, the four waves take every fourth eight of k and are added up in LDS in their order.  Lane l
// holds row l % 32; half l / 32 feeds k0 + 4 (l / 32) + j to the j-th MFMA, the same in both operands.
template <bool KA, bool KB, Prod E>
__device__ __forceinline__ void f32_small(const VocabArgs& a, const F32Product& p, int wg) {
  constexpr int BT = 32, CP = BT + 4, PF = 4, LONG = 1024;
  __shared__ __attribute__((aligned(16))) float red[4][BT * CP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  const int cnt = piece_rows(a);
  const int M = E == Prod::Dw ? p.M : cnt, N = p.N;
  const int tn = (N + BT - 1) / BT, tiles = (M + BT - 1) / BT * tn;
  const int Kall = E == Prod::Dw ? cnt : p.K;
  const int splits = (E == Prod::Dh || E == Prod::Dw) && tiles ? f32_splits(BT, tiles, Kall) : 1;
  if (wg >= tiles * splits) return;
  const int split = wg / tiles, tile = wg - split * tiles;
  const int m0 = tile / tn * BT, n0 = tile % tn * BT;
  const int n8 = (Kall + 7) / 8;
  const int kb = (int)((long)n8 * split / splits) * 8, K = min(Kall, (int)((long)n8 * (split + 1) / splits) * 8);
  f32x16 acc, sum;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = sum[r] = 0.f;
  auto load = [&](auto KM, const float* X, long ld, int r0, int rows, int k, float (&v)[4]) {
    const int r = r0 + l32;
    if constexpr (decltype(KM)::value) {
      const float* q = X + (long)min(r, rows - 1) * ld + k;
      if (k + 4 <= K) {
        *reinterpret_cast<f32x4*>(v) = *reinterpret_cast<const f32x4_a4*>(q);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = k + i < K ? q[i] : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = k + i < K ? X[(long)(k + i) * ld + min(r, rows - 1)] : 0.f;
    }
  };
  int done = 0;
  for (int k0 = kb + wave * 8; k0 < K; k0 += 32 * PF) {
    float fa[PF][4], fb[PF][4];
#pragma unroll
    for (int q = 0; q < PF; ++q) {  // past K: zeros
      load(std::integral_constant<bool, KA>{}, p.A, p.lda, m0, M, k0 + q * 32 + half * 4, fa[q]);
      load(std::integral_constant<bool, KB>{}, p.B, p.ldb, n0, N, k0 + q * 32 + half * 4, fb[q]);
    }
#pragma unroll
    for (int q = 0; q < PF; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = mfma32_f32(fb[q][j], fa[q][j], acc);
    if ((done += 8 * PF) >= LONG) {
      done = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sum[r] += acc[r];
        acc[r] = 0.f;
      }
    }
  }
#pragma unroll
  for (int g = 0; g < 4; ++g)
    *reinterpret_cast<float4*>(red[wave] + l32 * CP + 8 * g + 4 * half) =
        make_float4(sum[4 * g] + acc[4 * g], sum[4 * g + 1] + acc[4 * g + 1], sum[4 * g + 2] + acc[4 * g + 2], sum[4 * g + 3] + acc[4 * g + 3]);
  __syncthreads();
  for (int i = tid; i < BT * BT; i += 256) {
    const int at = i / BT * CP + i % BT;
    red[0][at] = ((red[0][at] + red[1][at]) + red[2][at]) + red[3][at];
  }
  __syncthreads();
  f32_epilogue<BT, CP, E>(a, p, red[0], M, N, m0, n0, tile, split, splits, tiles);
}
template <bool KA, bool KB, Prod E>
__global__ __launch_bounds__(256) void vocab_f32_small_k(VocabArgs a, F32Product p) {
  f32_small<KA, KB, E>(a, p, blockIdx.x);
}
// both gradients in one launch, dh by the first n_dh workgroups
__global__ __launch_bounds__(256) void vocab_f32_small_grads_k(VocabArgs a, F32Product dh, F32Product dw, int n_dh) {
  if ((int)blockIdx.x < n_dh) f32_small<true, false, Prod::Dh>(a, dh, blockIdx.x);
  else f32_small<false, false, Prod::Dw>(a, dw, blockIdx.x - n_dh);
}

// dh or dw of a piece from its shares.  G threads take every G-th share of a column each, and are added up in their order.
template <Prod E, int G>
__global__ __launch_bounds__(256) void vocab_f32_shares_k(VocabArgs a, F32Product p, int bt) {
  __shared__ float red[256];
  const int cnt = piece_rows(a), M = E == Prod::Dw ? p.M : cnt, K = E == Prod::Dw ? cnt : p.K;
  const int m = blockIdx.x, lane = threadIdx.x % (256 / G), g = threadIdx.x / (256 / G), n = blockIdx.y * (256 / G) + lane;
  if (m >= M) return;
  const int tn = (p.N + bt - 1) / bt, tiles = (M + bt - 1) / bt * tn, splits = f32_splits(bt, tiles, K);
  if (splits == 1) return;
  float v = 0.f;
  if (n < p.N) {
    const float* q = a.shares + (long)(m / bt * tn + n / bt) * bt * bt + (m % bt) * bt + n % bt;
#pragma unroll 8
    for (int s = g; s < splits; s += G) v += q[(long)s * tiles * bt * bt];
  }
  if constexpr (G > 1) {
    red[threadIdx.x] = v;
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int o = 1; o < G; ++o) v += red[o * (256 / G) + lane];
  }
  if (n < p.N) f32_gradient<E>(a, m, n, v);
}

// ---------------------------------------------------------------- rows
// a row's tiles joined by the lanes of a wave
__device__ __forceinline__ Peak join_wave(Peak p) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) p = join(p, Peak{__shfl_xor(p.m, o), __shfl_xor(p.l, o), __shfl_xor(p.at, o)});
  return p;
}

// ... and by those of a workgroup; red: one of each wave
__device__ __forceinline__ Peak join_row(const VocabArgs& a, int m, Peak* red) {
  Peak p{-INFINITY, 0.f, INT32_MAX};
  for (int t = threadIdx.x; t < a.tiles; t += 256) {
    const float2 q = a.part[(long)m * a.tiles + t];
    p = join(p, Peak{q.x, q.y, a.part_at ? a.part_at[(long)m * a.tiles + t] : 0});
  }
  p = join_wave(p);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = p;
  __syncthreads();
  return join(join(red[0], red[1]), join(red[2], red[3]));
}

// A workgroup per row: loss and lse, or the token and its log-probability.
__global__ __launch_bounds__(256) void vocab_rows_k(VocabArgs a) {
  __shared__ Peak red[4];
  const int m = blockIdx.x;
  if (m >= piece_rows(a)) return;
  const Peak p = join_row(a, m, red);
  if (threadIdx.x) return;
  if (a.few && a.labels && !counts(a, a.labels[m])) {
    a.loss[m] = a.lse[m] = 0.f;
    return;
  }
  const float log_l = logf(p.l);
  if (a.token) {
    a.token[a.row0 + m] = p.at;
    a.logprob[a.row0 + m] = -log_l;
    return;
  }
  const int row = a.few ? m : a.idx[a.row0 + m];
  a.loss[row] = (p.m - a.target[a.row0 + m]) + log_l;  // not lse - s: of a row that is sure of its label little is left
  a.lse[row] = p.m + log_l;
}

// Loss and lse of a row, and its P in the place of the logits, rounded once to the storage type (few rows: in two parts); zeros past V and in the rows
// up to a multiple of 64; with bf16 tensors what the stored P falls short of a sum of zero (row_left).  A workgroup takes 16384 columns of one row and joins the row's tiles by itself.
// With bf16 tensors the logits come in fp16, as s - (the largest of their tile, which is in part): off by 2^-11 of that difference
// at most, so P by 2^-11 (m - s) of itself.  What is large of P has s near m and keeps its digits; P a thousandth of its tile's
// largest is off by 2^-8.2 at most, its own rounding to bf16 by 2^-8; the label's entry comes from the loss, in fp32.  Half the bytes of fp32 logits:
// 2048 x 32000 took 50 to 54 us here instead of 78 (53 to 58 with the sums of what is stored), and 16 less to store.
constexpr int P_COLS = 16384;
template <typename T>
__global__ __launch_bounds__(256) void vocab_p_k(VocabArgs a) {
  __shared__ Peak red[4];
  __shared__ float short_of[4];
  const int m = blockIdx.x, cnt = piece_rows(a), tid = threadIdx.x, first = blockIdx.y * P_COLS + tid * 8;
  const int last = min((int)(blockIdx.y + 1) * P_COLS, a.Vp);
  if (m >= ((cnt + 63) & ~63)) return;
  const long at = (long)m * a.Vp;
  T* p = static_cast<T*>(a.logits) + at;
  float left = 0.f;  // minus the sum of what is stored
  auto store = [&](int v, const float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
      const bf16x8 hi = pack_frag(x);
      *reinterpret_cast<bf16x8*>(p + v) = hi;
      float y[8];
      unpack_frag(hi, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) left -= y[e];
      if (two_parts(cnt)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] - y[e];
        const bf16x8 lo = pack_frag(y);
        *reinterpret_cast<bf16x8*>(p + (long)TWO_PARTS * a.Vp + v) = lo;
        unpack_frag(lo, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) left -= y[e];
      }
    } else {
      St<T>::st4(p, v, x);
      St<T>::st4(p, v + 4, x + 4);
    }
  };
  if (m >= cnt) {
    const float zero[8] = {};
    for (int v0 = first; v0 < last; v0 += 2048) store(v0, zero);
    return;
  }
  const Peak q = join_row(a, m, red);
  const float log_l = logf(q.l), lse = q.m + log_l;  // P does not take lse, whose rounding would be in a whole row but its label
  const float loss = (q.m - a.target[a.row0 + m]) + log_l;  // not lse - s: of a row that is sure of its label little is left
  float g = a.g_c[a.row0 + m];
  if constexpr (sizeof(T) == 2) g /= dloss_unit(a);
  const int lab = a.lab_c[a.row0 + m];
  if (blockIdx.y == 0 && tid == 0) {
    const int row = a.idx[a.row0 + m];
    a.loss[row] = loss;
    a.lse[row] = lse;
  }
#pragma unroll 4
  for (int v0 = first; v0 < last; v0 += 2048) {
    float x[8];
    if constexpr (sizeof(T) == 2) {
      const half8 h = *reinterpret_cast<const half8*>(static_cast<const _Float16*>(a.logits) + at + v0);
      const float top = a.part[(long)m * a.tiles + min(v0, a.V - 1) / a.bn].x - q.m - log_l;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)h[e] + top;
    } else {
      const float* s = static_cast<const float*>(a.logits) + at + v0;
      const float4 lo = *reinterpret_cast<const float4*>(s), hi = *reinterpret_cast<const float4*>(s + 4);
      x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w;
      x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] - q.m - log_l;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v0 + e < a.V ? g * exp_below(x[e]) : 0.f;
    if (lab >= v0 && lab < v0 + 8) {
      const float y = g * expm1f(-loss);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = v0 + e == lab ? y : x[e];
    }
    store(v0, x);
  }
  if constexpr (sizeof(T) == 2) {
    left = wave_sum(left);
    if ((tid & 63) == 0) short_of[tid >> 6] = left;
    __syncthreads();
    if (tid == 0) a.left[(long)m * a.left_n + blockIdx.y] = (short_of[0] + short_of[1]) + (short_of[2] + short_of[3]);
  }
}

// ---------------------------------------------------------------- launches
static long up(long x, long m) { return (x + m - 1) / m * m; }

static long f32_tiles(long rows, long cols, int bt) { return (up(rows, bt) / bt) * (up(cols, bt) / bt); }

// Whether the fp32 products take 32-wide tiles: where 128-wide ones, with the shares of their k, leave most CUs idle (dh of 2048 x 768, 5000
// classes: 321 us by 32, 159 + 6 by 128 in shares), where they would be half empty or less (32 x 30000, d 2048: logits 124 us and 163,
// dh 78 and 152; 20 x 40000, d 256: logits 18 and 47), or where a row of w is too short for them
static bool small_logits(const VocabArgs& a) { return a.d < 4 || a.n <= 64 || f32_tiles(a.n, a.V, 128) < 128; }
static bool small_grad(long rows, int d, int K) {
  const long tiles = f32_tiles(rows, d, 128);
  return d <= 64 || rows <= 64 || tiles * (tiles < 128 ? f32_splits(128, (int)tiles, K) : 1) < 128;
}
static bool small_dh(const VocabArgs& a) { return small_grad(a.n, a.d, a.V); }
static bool small_dw(const VocabArgs& a) { return small_grad(a.V, a.d, a.n); }
// workgroups that dh or dw may have, whichever rows count
static long f32_wgs(int bt, long tiles) {
  const long slots = bt == 128 && tiles > 256 ? 2 * F32_SLOTS : F32_SLOTS;
  return tiles > slots ? tiles : slots;
}
static size_t f32_share_bytes(const VocabArgs& a) {
  auto bytes = [](bool small, long rows, int d) {
    const int bt = small ? 32 : 128;
    return (size_t)(bt == 128 && f32_tiles(rows, d, bt) > 256 ? 2 * F32_SLOTS : F32_SLOTS) * bt * bt * 4;
  };
  const size_t h = bytes(small_dh(a), a.n, a.d), w = bytes(small_dw(a), a.V, a.d);
  return h > w ? h : w;
}

// The workspace: sizes, and the pointers into it where there is one
size_t vocab_layout(int dtype, VocabArgs& a, bool grads, bool next, void* ws) {
  const bool low = dtype == DT_BF16;
  const long es = low ? 2 : 4, np = up(a.n, 64);
  a.Vp = (int)up(a.V, 64);
  a.dp = (int)up(a.d, 64);
  a.bn = low ? vocab_mm_bn(a.n, a.d, a.V) : small_logits(a) ? 32 : 128;
  a.few = low && !grads && vocab_few(a.n, a.d);
  a.tiles = a.few ? vocab_few_wgs(a.n, a.d) : (a.V + a.bn - 1) / a.bn;
  // rows at a time: 2 GiB of logits, 2^24 partial sums; whole tiles of rows
  const long most = grads ? (low ? 1l << 30 : 1l << 29) / a.Vp : (1l << 24) / a.tiles;
  a.R = (int)(np <= most ? np : most / 256 * 256 > 256 ? most / 256 * 256 : 256);
  if (a.R > np) a.R = (int)np;
  if (a.few) a.R = a.n;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    void* p = ws ? static_cast<char*>(ws) + at : nullptr;
    at = (at + bytes + 255) & ~(size_t)255;
    return p;
  };
  a.hc = a.few ? nullptr : take((size_t)np * a.dp * es);
  a.part = static_cast<float2*>(take((size_t)a.R * a.tiles * 8));
  a.part_at = next ? static_cast<int*>(take((size_t)a.R * a.tiles * 4)) : nullptr;
  if (a.few) {
    a.target = next ? nullptr : static_cast<float*>(take((size_t)a.n * 4));
  } else if (!next) {
    a.n_counted = static_cast<int*>(take(4));
    a.block_count = a.n > PICK_DIRECT ? static_cast<int*>(take((size_t)(np / 1024 + 1) * 4)) : nullptr;
    a.idx = static_cast<int*>(take((size_t)a.n * 4));
    a.lab_c = static_cast<int*>(take((size_t)a.n * 4));
    a.target = static_cast<float*>(take((size_t)a.n * 4));
  }
  if (grads) {
    a.g_c = static_cast<float*>(take((size_t)a.n * 4));
    a.logits = take((size_t)(low && a.R < 2 * TWO_PARTS ? 2 * TWO_PARTS : a.R) * a.Vp * es);
    a.left_n = (a.Vp + P_COLS - 1) / P_COLS;
    a.left = low ? static_cast<float*>(take((size_t)a.R * a.left_n * 4)) : nullptr;
    a.shares = static_cast<float*>(take(low ? vocab_share_bytes(a.n, a.R, a.d, a.V) : f32_share_bytes(a)));
    if (low && a.n > a.R) a.dw_acc = static_cast<float*>(take((size_t)a.V * a.d * 4));
    a.ld_acc = a.d;
  }
  return at;
}

// sums of shares, where there may be any: dw's tiles are known here, dh's may be fewer
template <Prod E>
static void f32_shares(const VocabArgs& a, const F32Product& p, int bt, hipStream_t s) {
  const long rows = E == Prod::Dw ? p.M : a.rows;
  const int K = E == Prod::Dw ? a.rows : p.K;
  if (f32_splits(bt, E == Prod::Dw ? (int)f32_tiles(rows, p.N, bt) : 1, K) == 1) return;
  if (rows * p.N >= 262144) RG_LAUNCH((vocab_f32_shares_k<E, 1>), dim3((unsigned)rows, (p.N + 255) / 256), dim3(256), 0, s, a, p, bt);
  else RG_LAUNCH((vocab_f32_shares_k<E, 8>), dim3((unsigned)rows, (p.N + 31) / 32), dim3(256), 0, s, a, p, bt);
}

template <bool KA, bool KB, Prod E>
static void go_f32(const VocabArgs& a, const F32Product& p, bool small, hipStream_t s) {
  constexpr bool shared = E == Prod::Dh || E == Prod::Dw;
  const int bt = small ? 32 : 128;
  const long tiles = f32_tiles(E == Prod::Dw ? p.M : a.rows, p.N, bt);
  const unsigned wgs = (unsigned)(shared ? f32_wgs(bt, tiles) : tiles);
  if (small) RG_LAUNCH((vocab_f32_small_k<KA, KB, E>), dim3(wgs), dim3(256), 0, s, a, p);
  else RG_LAUNCH((vocab_f32_k<KA, KB, E>), dim3(wgs), dim3(256), 0, s, a, p);
  if constexpr (shared) f32_shares<E>(a, p, bt, s);
}

static void vocab_logits_f32(const VocabArgs& a, bool keep, hipStream_t s) {
  const float* H = static_cast<const float*>(a.hc) + (long)a.row0 * a.dp;
  const F32Product p{H, a.dp, static_cast<const float*>(a.w), a.ldw, 0, a.V, a.d};
  if (keep) go_f32<true, true, Prod::Logits>(a, p, a.bn == 32, s);
  else go_f32<true, true, Prod::Stats>(a, p, a.bn == 32, s);
}

static void vocab_grads_f32(const VocabArgs& a, hipStream_t s) {
  const float* H = static_cast<const float*>(a.hc) + (long)a.row0 * a.dp;
  const float* P = static_cast<const float*>(a.logits);
  const F32Product h{P, a.Vp, static_cast<const float*>(a.w), a.ldw, 0, a.d, a.V};
  const F32Product w{P, a.Vp, H, a.dp, a.V, a.d, 0};
  const bool sh = small_dh(a), sw = small_dw(a);
  // Small products are bound by their latency: both in one launch where neither has shares (128 x 512, d 128: 10.8 us, one after the other 7.2 and 4.9, and a launch less)
  const long th = f32_tiles(a.rows, a.d, 32), tw = f32_tiles(a.V, a.d, 32);
  if (a.dh && a.dw && sh && sw && f32_splits(32, 1, a.V) == 1 &&
      f32_splits(32, (int)tw, a.rows) == 1) {
    RG_LAUNCH(vocab_f32_small_grads_k, dim3((unsigned)(th + tw)), dim3(256), 0, s, a, h, w, (int)th);
    return;
  }
  if (a.dh) go_f32<true, false, Prod::Dh>(a, h, sh, s);
  if (a.dw) go_f32<false, false, Prod::Dw>(a, w, sw, s);
}

template <typename T>
static hipError_t vocab_t(VocabArgs a, hipStream_t s) {
  constexpr bool low = sizeof(T) == 2;
  const bool grads = a.dh || a.dw;
  if (a.few) {
    a.rows = a.n;
    launch_vocab_few_bf16(a, s);
    RG_LAUNCH(vocab_rows_k, dim3(a.n), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (a.labels && a.block_count) RG_LAUNCH(vocab_count_k, dim3((a.n + 1023) / 1024), dim3(256), 0, s, a);
  const bool wide = (reinterpret_cast<uintptr_t>(a.h) & 15u) == 0 && a.ldh * sizeof(T) % 16 == 0 && a.d * sizeof(T) % 16 == 0;
  RG_LAUNCH(vocab_pick_k<T>, dim3((a.n + PICK_ROWS - 1) / PICK_ROWS), dim3(256), 0, s, a, wide);
  a.count = a.labels ? a.n_counted : nullptr;
  for (a.row0 = 0; a.row0 < a.n; a.row0 += a.R) {
    a.rows = a.n - a.row0 < a.R ? a.n - a.row0 : a.R;
    a.first = a.row0 == 0;
    a.last = a.row0 + a.R >= a.n;
    if constexpr (low) launch_vocab_logits_bf16(a, grads, s);
    else vocab_logits_f32(a, grads, s);
    if (!grads) {
      RG_LAUNCH(vocab_rows_k, dim3(a.rows), dim3(256), 0, s, a);
      continue;
    }
    RG_LAUNCH(vocab_p_k<T>, dim3((unsigned)up(a.rows, 64), a.left_n), dim3(256), 0, s, a);
    if constexpr (low) launch_vocab_grads_bf16(a, s);
    else vocab_grads_f32(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_vocab(int dtype, const VocabArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? vocab_t<bf16>(a, s) : vocab_t<float>(a, s);
}

}  // namespace rg
