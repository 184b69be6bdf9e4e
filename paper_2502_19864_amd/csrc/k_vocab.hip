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
// The logits of a piece of the rows are held in fp32 while they are needed.  Pieces of the vocabulary would need
// no more memory, but lse needs all columns before P has any: the product h w^T would run twice, 8 n V d
// operations instead of 6.
#include "common.h"
#include "kernels.h"
#include "vocab_peak.h"

namespace rg {

// ---------------------------------------------------------------- rows that count
// One workgroup: a stable compaction of the labels, 1024 at a time.
__global__ __launch_bounds__(1024) void vocab_scan_k(VocabArgs a) {
  __shared__ int wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base = 0;
  for (int n0 = 0; n0 < a.n; n0 += 1024) {
    const int n = n0 + tid;
    const int lab = n < a.n ? a.labels[n] : -1;
    const bool in = lab >= 0 && lab < a.V;
    const uint64_t vote = __ballot(in);
    if (lane == 0) wsum[wave] = __popcll(vote);
    __syncthreads();
    int before = base, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? wsum[w] : 0;
      all += wsum[w];
    }
    if (in) {
      const int at = before + __popcll(vote & ((1ull << lane) - 1));
      a.idx[at] = n;
      a.lab_c[at] = lab;
      if (a.dloss) a.g_c[at] = a.dloss[n];
    } else if (n < a.n) {
      a.loss[n] = 0.f;
      a.lse[n] = 0.f;
    }
    base += all;
    __syncthreads();
  }
  if (tid == 0) *a.n_counted = base;
}

// hc[i] = h[idx[i]], zeros past d and past the rows that count up to a multiple of 64; the gradient's rows that do
// not count are zeros.  One workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void vocab_gather_k(VocabArgs a) {
  const int i = blockIdx.x, cnt = a.labels ? *a.n_counted : a.n;
  if (i < ((cnt + 63) & ~63)) {
    const T* src = static_cast<const T*>(a.h) + (i < cnt ? (long)(a.labels ? a.idx[i] : i) : 0) * a.ldh;
    T* dst = static_cast<T*>(a.hc) + (long)i * a.dp;
    for (int k = threadIdx.x; k < a.dp; k += 256) dst[k] = i < cnt && k < a.d ? src[k] : T(0);
  }
  if (a.dh && i < a.n) {
    const int lab = a.labels[i];
    if (lab < 0 || lab >= a.V) {
      T* dst = static_cast<T*>(a.dh) + (long)i * a.lddh;
      for (int k = threadIdx.x; k < a.d; k += 256) dst[k] = T(0);
    }
  }
}

// ---------------------------------------------------------------- products in fp32
// C[m][n] = sum_k A(m, k) B(n, k) on 128 x 128 tiles: registers -> LDS [k][m], MFMA 32x32x2 f32, four waves of 64 x 64.
// KA: A is [M][K], else [K][M]; KB likewise.
__device__ __forceinline__ void ld8_any(const float* p, int valid, float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < valid ? p[i] : 0.f;
}

template <bool KA, bool KB, Prod E>
__global__ __launch_bounds__(256) void vocab_f32_k(VocabArgs a, const float* A, long lda, const float* B, long ldb, int M0,
                                                   int N, int K0) {
  constexpr int BT = 128, BK = 16, PITCH = 160, CP = BT + 4;
  __shared__ __attribute__((aligned(16))) float smem[BT * CP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int cnt = piece_rows(a);
  const int M = E == Prod::Dw ? M0 : cnt, K = E == Prod::Dw ? cnt : K0;
  const int tn = (N + BT - 1) / BT, m0 = (int)(blockIdx.x / tn) * BT, n0 = (int)(blockIdx.x % tn) * BT;
  if (m0 >= M) return;
  float* sa = smem;
  float* sb = smem + BK * PITCH;
  // Sums over a vocabulary are long, and the matrix unit's additions lean to one side: 300,000 terms in one chain were off by
  // 1e-3 of a gradient beside a label's large term.  So a chain ends after LONG, and the chains are added up.
  constexpr int LONG = 1024;
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
  float ra[8], rb[8];
  auto fetch = [&](int k0) {
    if constexpr (KA) {
      const int m = m0 + (tid >> 1), k = k0 + (tid & 1) * 8;
      ld8_any(A + (long)min(m, M - 1) * lda + k, m < M ? K - k : 0, ra);
    } else {
      const int k = k0 + (tid >> 4), m = m0 + (tid & 15) * 8;
      ld8_any(A + (long)min(k, K - 1) * lda + m, k < K ? M - m : 0, ra);
    }
    if constexpr (KB) {
      const int n = n0 + (tid >> 1), k = k0 + (tid & 1) * 8;
      ld8_any(B + (long)min(n, N - 1) * ldb + k, n < N ? K - k : 0, rb);
    } else {
      const int k = k0 + (tid >> 4), n = n0 + (tid & 15) * 8;
      ld8_any(B + (long)min(k, K - 1) * ldb + n, k < K ? N - n : 0, rb);
    }
  };
  if (K > 0) fetch(0);
  for (int k0 = 0; k0 < K; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (KA) sa[((tid & 1) * 8 + i) * PITCH + (tid >> 1)] = ra[i];
      else sa[(tid >> 4) * PITCH + (tid & 15) * 8 + i] = ra[i];
      if constexpr (KB) sb[((tid & 1) * 8 + i) * PITCH + (tid >> 1)] = rb[i];
      else sb[(tid >> 4) * PITCH + (tid & 15) * 8 + i] = rb[i];
    }
    __syncthreads();
    if (k0 + BK < K) fetch(k0 + BK);
#pragma unroll
    for (int k = 0; k < BK; k += 2) {
      float fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = sa[(k + (lane >> 5)) * PITCH + wm * 64 + i * 32 + (lane & 31)];
        fb[i] = sb[(k + (lane >> 5)) * PITCH + wn * 64 + i * 32 + (lane & 31)];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mfma32_f32(fb[j], fa[i], acc[i][j]);
    }
    if ((k0 + BK) % LONG == 0) settle();
  }
  settle();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        smem[(wm * 64 + i * 32 + (lane & 31)) * CP + wn * 64 + j * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4] = sum[i][j][r];
  __syncthreads();
  if constexpr (E == Prod::Stats || E == Prod::Logits) {
    // two threads per row, 64 columns each
    const int row = tid >> 1, m = m0 + row, c0 = (tid & 1) * 64;
    const int lab = a.lab_c && m < M ? a.lab_c[a.row0 + m] : -1;
    Peak p{-INFINITY, 0.f, n0 + c0 < N ? n0 + c0 : n0};
    for (int c = c0; c < c0 + 64 && n0 + c < N; ++c) {
      const float s = smem[row * CP + c];
      if (s > p.m) {
        p.m = s;
        p.at = n0 + c;
      }
    }
    const float z = p.m == -INFINITY ? 0.f : p.m;
    for (int c = c0; c < c0 + 64 && n0 + c < N; ++c) {
      const float s = smem[row * CP + c];
      p.l += exp_below(s - z);
      if (n0 + c == lab) a.target[a.row0 + m] = s;
    }
    const Peak q{__shfl_xor(p.m, 1), __shfl_xor(p.l, 1), __shfl_xor(p.at, 1)};
    p = join(p, q);
    if (m < M && (tid & 1) == 0) {
      a.part[(long)m * a.tiles + n0 / BT] = make_float2(p.m, p.l);
      if (a.part_at) a.part_at[(long)m * a.tiles + n0 / BT] = p.at;
    }
    if constexpr (E == Prod::Logits)
      for (int i = tid; i < BT * BT; i += 256) {
        const int r = i / BT, c = i % BT;
        if (m0 + r < M && n0 + c < N) a.logits[(long)(m0 + r) * a.Vp + n0 + c] = smem[r * CP + c];
      }
  } else {
    for (int i = tid; i < BT * BT; i += 256) {
      const int r = i / BT, c = i % BT, m = m0 + r, n = n0 + c;
      if (m >= M || n >= N) continue;
      const float v = smem[r * CP + c];
      if constexpr (E == Prod::Dh) {
        static_cast<float*>(a.dh)[(long)a.idx[a.row0 + m] * a.lddh + n] = v;
      } else {
        float* o = static_cast<float*>(a.dw) + (long)m * a.lddw + n;
        *o = a.first ? v : *o + v;
      }
    }
  }
}

// ---------------------------------------------------------------- rows
// One wave per row: its tiles' (maximum, sum) joined; loss and lse, or the token and its log-probability.
__global__ __launch_bounds__(256) void vocab_rows_k(VocabArgs a) {
  const int m = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (m >= piece_rows(a)) return;
  Peak p{-INFINITY, 0.f, INT32_MAX};
  for (int t = lane; t < a.tiles; t += 64) {
    const float2 q = a.part[(long)m * a.tiles + t];
    p = join(p, Peak{q.x, q.y, a.part_at ? a.part_at[(long)m * a.tiles + t] : 0});
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) p = join(p, Peak{__shfl_xor(p.m, o), __shfl_xor(p.l, o), __shfl_xor(p.at, o)});
  if (lane) return;
  const float log_l = logf(p.l);
  if (a.token) {
    a.token[a.row0 + m] = p.at;
    a.logprob[a.row0 + m] = -log_l;
    return;
  }
  const int row = a.idx[a.row0 + m];
  const float t = a.target[a.row0 + m], lse = p.m + log_l;
  a.loss[row] = (p.m - t) + log_l;  // not lse - t: of a row that is sure of its label little is left
  a.lse[row] = lse;
  a.stat[m] = make_float2(lse, (p.m - t) + log_l);
}

// P of a piece from its logits, rounded once to the storage type; zeros past V and in the rows up to a multiple of 64
template <typename T>
__global__ __launch_bounds__(256) void vocab_p_k(VocabArgs a) {
  const int m = blockIdx.x, cnt = piece_rows(a);
  if (m >= ((cnt + 63) & ~63)) return;
  const bool in = m < cnt;
  const float2 st = in ? a.stat[m] : make_float2(0.f, 0.f);
  const float g = in ? a.g_c[a.row0 + m] : 0.f;
  const int lab = in ? a.lab_c[a.row0 + m] : -1;
  const float* s = a.logits + (long)m * a.Vp;
  T* p = static_cast<T*>(a.P) + (long)m * a.Vp;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int v = blockIdx.y * 1024 + i * 256 + threadIdx.x;
    if (v >= a.Vp) break;
    const float x = in && v < a.V ? g * (v == lab ? expm1f(-st.y) : exp_below(s[v] - st.x)) : 0.f;
    St<T>::st(p, v, x);
  }
}

// ---------------------------------------------------------------- launches
constexpr int F32_TILE = 128;

static long up(long x, long m) { return (x + m - 1) / m * m; }

// The workspace: sizes, and the pointers into it where there is one
size_t vocab_layout(int dtype, VocabArgs& a, bool grads, bool next, void* ws) {
  const long es = dtype == DT_BF16 ? 2 : 4, np = up(a.n, 64);
  a.Vp = (int)up(a.V, 64);
  a.dp = (int)up(a.d, 64);
  a.bn = dtype == DT_BF16 ? vocab_mm_bn(a.n, a.V) : F32_TILE;
  a.tiles = (a.V + a.bn - 1) / a.bn;
  // rows at a time: 2^29 logits (2 GiB), 2^24 partial sums; whole tiles of rows
  const long most = grads ? (1l << 29) / a.Vp : (1l << 24) / a.tiles;
  a.R = (int)(np <= most ? np : most / 256 * 256 > 256 ? most / 256 * 256 : 256);
  if (a.R > np) a.R = (int)np;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    void* p = ws ? static_cast<char*>(ws) + at : nullptr;
    at = (at + bytes + 255) & ~(size_t)255;
    return p;
  };
  a.hc = take((size_t)np * a.dp * es);
  a.part = static_cast<float2*>(take((size_t)a.R * a.tiles * 8));
  a.part_at = next ? static_cast<int*>(take((size_t)a.R * a.tiles * 4)) : nullptr;
  if (!next) {
    a.n_counted = static_cast<int*>(take(4));
    a.idx = static_cast<int*>(take((size_t)a.n * 4));
    a.lab_c = static_cast<int*>(take((size_t)a.n * 4));
    a.target = static_cast<float*>(take((size_t)a.n * 4));
    a.stat = static_cast<float2*>(take((size_t)a.R * 8));
  }
  if (grads) {
    a.g_c = static_cast<float*>(take((size_t)a.n * 4));
    a.logits = static_cast<float*>(take((size_t)a.R * a.Vp * 4));
    if (dtype == DT_BF16) {
      a.P = take((size_t)a.R * a.Vp * 2);
      a.dh_splits = vocab_dh_splits(a.R, a.d, a.V);
      a.dh_part = a.dh_splits > 1 ? static_cast<float*>(take((size_t)a.dh_splits * a.R * a.d * 4)) : nullptr;
      if (a.n > a.R) a.dw_acc = static_cast<float*>(take((size_t)a.V * a.d * 4));
      a.ld_acc = a.d;
    } else {
      a.P = a.logits;
    }
  }
  return at;
}

template <bool KA, bool KB, Prod E>
static void go_f32(const VocabArgs& a, const void* A, long lda, const void* B, long ldb, int M, int N, int K, hipStream_t s) {
  const unsigned wgs = ((M + F32_TILE - 1) / F32_TILE) * ((N + F32_TILE - 1) / F32_TILE);
  RG_LAUNCH((vocab_f32_k<KA, KB, E>), dim3(wgs), dim3(256), 0, s, a, static_cast<const float*>(A), lda,
            static_cast<const float*>(B), ldb, M, N, K);
}

template <typename T>
static hipError_t vocab_t(VocabArgs a, hipStream_t s) {
  constexpr bool low = sizeof(T) == 2;
  const bool grads = a.dh || a.dw;
  if (a.labels) RG_LAUNCH(vocab_scan_k, dim3(1), dim3(1024), 0, s, a);
  RG_LAUNCH(vocab_gather_k<T>, dim3((unsigned)up(a.n, 64)), dim3(256), 0, s, a);
  a.count = a.labels ? a.n_counted : nullptr;
  for (a.row0 = 0; a.row0 < a.n; a.row0 += a.R) {
    a.rows = a.n - a.row0 < a.R ? a.n - a.row0 : a.R;
    a.first = a.row0 == 0;
    a.last = a.row0 + a.R >= a.n;
    const T* H = static_cast<const T*>(a.hc) + (long)a.row0 * a.dp;
    if constexpr (low) launch_vocab_logits_bf16(a, grads, s);
    else if (grads) go_f32<true, true, Prod::Logits>(a, H, a.dp, a.w, a.ldw, a.rows, a.V, a.d, s);
    else go_f32<true, true, Prod::Stats>(a, H, a.dp, a.w, a.ldw, a.rows, a.V, a.d, s);
    RG_LAUNCH(vocab_rows_k, dim3((a.rows + 3) / 4), dim3(256), 0, s, a);
    if (!grads) continue;
    RG_LAUNCH(vocab_p_k<T>, dim3((unsigned)up(a.rows, 64), (a.Vp + 1023) / 1024), dim3(256), 0, s, a);
    if (a.dh) {
      if constexpr (low) launch_vocab_dh_bf16(a, s);
      else go_f32<true, false, Prod::Dh>(a, a.P, a.Vp, a.w, a.ldw, a.rows, a.d, a.V, s);
    }
    if (a.dw) {
      if constexpr (low) launch_vocab_dw_bf16(a, s);
      else go_f32<false, false, Prod::Dw>(a, a.P, a.Vp, H, a.dp, a.V, a.d, 0, s);
    }
  }
  return hipGetLastError();
}

hipError_t launch_vocab(int dtype, const VocabArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? vocab_t<bf16>(a, s) : vocab_t<float>(a, s);
}

}  // namespace rg
