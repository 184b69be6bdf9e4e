// LayerNorm and RMSNorm of rows, a residual added before, with the gradients of x, gain and shift.
//
//   s = x + res (as stored)      u = (s - mean) rstd      y = u gain + shift
//   rstd = 1 / sqrt(mean((s - mean)^2) + eps); RMSNorm: mean = 0
//   a = dy gain;  ds = rstd (a - mean(a) - u mean(a u)) + dskip (RMSNorm: without mean(a))
//   dgain += sum over rows of dy u;  dshift += sum over rows of dy
//
// Bound by memory.  A row stays in the registers of the threads that read it, so the mean, the
// squares around it (not the difference of two sums) and the result take one read of it.  The backward's
// workgroups run over many rows each and keep their columns' sums in registers; a second kernel adds
// the workgroups' sums in a fixed order.  16384 x 4096 in bf16: forward with residual 87 us, backward with dskip 114 us and 5 for the
// sums, 6.1 and 4.7 TB/s, more than a copy's 5.2 in the first as the passes leave some of the bytes in cache.
#include "common.h"
#include "kernels.h"

namespace rg {

// 16-byte pieces of a row: VE elements
template <typename T> constexpr int VE = 16 / sizeof(T);

// Column of element i of thread t's piece c, TPR threads to a row: 16 bytes side by side in rows that allow it (WIDE), else
// elements TPR apart, so that a wave's loads of single elements lie side by side too (2038 x 2382 in bf16: forward 14.7 us, side by side 25; backward 17.6 and 29).
template <bool WIDE, typename T, int TPR>
__device__ __forceinline__ int col_of(int c, int t, int i) {
  return WIDE ? (c * TPR + t) * VE<T> + i : (c * VE<T> + i) * TPR + t;
}
template <bool WIDE, int TPR, typename T>
__device__ __forceinline__ void ld_piece(const T* row, int c, int t, int d, float v[VE<T>]) {
  if constexpr (WIDE) {
    const T* p = row + col_of<WIDE, T, TPR>(c, t, 0);
    if constexpr (sizeof(T) == 2) unpack_frag(*reinterpret_cast<const bf16x8*>(p), v);
    else St<T>::ld4(p, 0, v);
  } else {
#pragma unroll
    for (int i = 0; i < VE<T>; ++i) {  // no branch: what is past the row is read as its last element and left out
      const int at = col_of<WIDE, T, TPR>(c, t, i);
      const float x = St<T>::ld(row, min(at, d - 1));
      v[i] = at < d ? x : 0.f;
    }
  }
}
template <bool WIDE, int TPR, typename T>
__device__ __forceinline__ void st_piece(T* row, int c, int t, int d, const float v[VE<T>]) {
  if constexpr (WIDE) {
    T* p = row + col_of<WIDE, T, TPR>(c, t, 0);
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x8*>(p) = pack_frag(v);
    else St<T>::st4(p, 0, v);
  } else {
#pragma unroll
    for (int i = 0; i < VE<T>; ++i) {
      const int at = col_of<WIDE, T, TPR>(c, t, i);
      if (at < d) St<T>::st(row, at, v[i]);
    }
  }
}
// what storing and loading again makes of v
template <typename T>
__device__ __forceinline__ float stored(float v) {
  if constexpr (sizeof(T) == 2) return bf2f(f2bf(v));
  return v;
}

// sum over the TPR threads of a row, in every one of them; red: one float per wave, free again after the next barrier
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += red[w];
  }
  return v;
}

// TPR threads per row, CH pieces per thread
template <typename T, int TPR, int CH, bool WIDE>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_fwd_k(NormArgs a) {
  constexpr int E = VE<T>, NT = TPR > 256 ? TPR : 256, RPW = NT / TPR;
  __shared__ float red[16];
  const int t = threadIdx.x % TPR;
  const long row = ((long)blockIdx.y * gridDim.x + blockIdx.x) * RPW + threadIdx.x / TPR;
  if (row >= a.rows) return;  // whole waves, or the workgroup
  const T* x = static_cast<const T*>(a.x.p) + row * a.x.t;
  const T* res = a.res.p ? static_cast<const T*>(a.res.p) + row * a.res.t : nullptr;
  float v[CH][E];
  float sum = 0.f;
  auto some = [&](int c) { return col_of<WIDE, T, TPR>(c, t, 0) < a.d; };  // of the piece is in the row
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[c][i] = 0.f;
    if (!some(c)) continue;
    ld_piece<WIDE, TPR>(x, c, t, a.d, v[c]);
    if (res) {
      float r[E];
      ld_piece<WIDE, TPR>(res, c, t, a.d, r);
#pragma unroll
      for (int i = 0; i < E; ++i) v[c][i] = stored<T>(v[c][i] + r[i]);
      st_piece<WIDE, TPR>(static_cast<T*>(a.s.p) + row * a.s.t, c, t, a.d, v[c]);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) sum += v[c][i];
  }
  const float mean = a.rms ? 0.f : row_sum<TPR>(sum, red) / a.d;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float w = col_of<WIDE, T, TPR>(c, t, i) < a.d ? v[c][i] - mean : 0.f;
      sq += w * w;
    }
  const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, red) / a.d + a.eps);
  if (a.stats && t == 0) a.stats[row] = make_float2(mean, rstd);
  const T* gain = static_cast<const T*>(a.gain);
  const T* shift = static_cast<const T*>(a.shift);
  T* y = static_cast<T*>(a.y.p) + row * a.y.t;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (!some(c)) continue;
    float g[E], b[E];
    ld_piece<WIDE, TPR>(gain, c, t, a.d, g);
    if (shift) ld_piece<WIDE, TPR>(shift, c, t, a.d, b);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float u = (v[c][i] - mean) * rstd * g[i];
      v[c][i] = shift ? u + b[i] : u;
    }
    st_piece<WIDE, TPR>(y, c, t, a.d, v[c]);
  }
}

// a piece as it lies in memory
template <bool WIDE, int TPR, typename T>
__device__ __forceinline__ uint4 ld_raw(const T* row, int c, int t, int d) {
  if constexpr (WIDE) return *reinterpret_cast<const uint4*>(row + col_of<WIDE, T, TPR>(c, t, 0));
  typedef T V __attribute__((ext_vector_type(VE<T>)));
  V v;
#pragma unroll
  for (int i = 0; i < VE<T>; ++i) {
    const int at = col_of<WIDE, T, TPR>(c, t, i);
    const T x = row[min(at, d - 1)];
    v[i] = at < d ? x : T(0);
  }
  return __builtin_bit_cast(uint4, v);
}
template <typename T>
__device__ __forceinline__ void unpack_raw(const uint4& q, float v[VE<T>]) {
  if constexpr (sizeof(T) == 2) {
    unpack_frag(__builtin_bit_cast(bf16x8, q), v);
  } else {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y);
    v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
}

// The next row of a workgroup is on its way while one is worked on (AHEAD; not in the widest rows, whose registers are full).  Rows
// stay as they lie in memory, and are unpacked for the sums and again for the result.
template <typename T, int TPR, int CH, bool AHEAD, bool WIDE>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_bwd_k(NormArgs a) {
  constexpr int E = VE<T>, NT = TPR > 256 ? TPR : 256, RPW = NT / TPR;
  __shared__ float red[32];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  auto some = [&](int c) { return col_of<WIDE, T, TPR>(c, t, 0) < a.d; };
  uint4 g[CH];
  float dg[CH][E], db[CH][E];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < E; ++i) dg[c][i] = db[c][i] = 0.f;
    g[c] = some(c) ? ld_raw<WIDE, TPR>(static_cast<const T*>(a.gain), c, t, a.d) : make_uint4(0, 0, 0, 0);
  }
  const float inv_d = 1.f / a.d;
  const long stride = (long)gridDim.x * RPW;
  struct Row {
    uint4 x[CH], y[CH], k[CH];
    float2 st;
  };
  auto load = [&](long row, Row& r) {
    const T* x = static_cast<const T*>(a.s.p) + row * a.s.t;
    const T* dy = static_cast<const T*>(a.dy.p) + row * a.dy.t;
    const T* k = static_cast<const T*>(a.dskip.p) + row * a.dskip.t;
    r.st = a.stats[row];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      r.x[c] = r.y[c] = r.k[c] = make_uint4(0, 0, 0, 0);
      if (!some(c)) continue;
      r.x[c] = ld_raw<WIDE, TPR>(x, c, t, a.d);
      r.y[c] = ld_raw<WIDE, TPR>(dy, c, t, a.d);
      if (a.dskip.p) r.k[c] = ld_raw<WIDE, TPR>(k, c, t, a.d);
    }
  };
  // rows group, group + groups, ..; every row of a workgroup's loop has all its threads
  long row = (long)blockIdx.x * RPW + sub;
  Row now, next;
  if (row < a.rows) load(row, now);
  for (; row < a.rows; row += stride) {
    if constexpr (AHEAD)
      if (row + stride < a.rows) load(row + stride, next);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float u[E], w[E], gf[E];
      unpack_raw<T>(now.x[c], u);
      unpack_raw<T>(now.y[c], w);
      unpack_raw<T>(g[c], gf);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        u[i] = col_of<WIDE, T, TPR>(c, t, i) < a.d ? (u[i] - now.st.x) * now.st.y : 0.f;
        dg[c][i] += w[i] * u[i];
        db[c][i] += w[i];
        w[i] *= gf[i];
        s1 += w[i];
        s2 += w[i] * u[i];
      }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6;
      __syncthreads();
      if ((threadIdx.x & 63) == 0) {
        red[wave] = s1;
        red[16 + wave] = s2;
      }
      __syncthreads();
      s1 = s2 = 0.f;
#pragma unroll
      for (int v = 0; v < TPR / 64; ++v) {
        s1 += red[v];
        s2 += red[16 + v];
      }
    }
    s1 = a.rms ? 0.f : s1 * inv_d;
    s2 *= inv_d;
    T* dx = static_cast<T*>(a.dx.p) + row * a.dx.t;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!some(c)) continue;
      float u[E], w[E], gf[E], k[E];
      unpack_raw<T>(now.x[c], u);
      unpack_raw<T>(now.y[c], w);
      unpack_raw<T>(g[c], gf);
      unpack_raw<T>(now.k[c], k);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float v = now.st.y * (w[i] * gf[i] - s1 - (u[i] - now.st.x) * now.st.y * s2);
        w[i] = a.dskip.p ? v + k[i] : v;
      }
      st_piece<WIDE, TPR>(dx, c, t, a.d, w);
    }
    if constexpr (AHEAD) now = next;
    else if (row + stride < a.rows) load(row + stride, now);
  }
  if (!a.part) return;
  // the row groups of a workgroup, then its sums: part[group][0: dgain, 1: dshift][d]
  __shared__ float acc[RPW > 1 ? (RPW - 1) * TPR * E * CH : 1];
  for (int which = 0; which < 2; ++which) {
    float* dst = which ? a.dshift : a.dgain;
    if (!dst) continue;
    float* out = a.part + ((long)blockIdx.x * 2 + which) * a.d;
    if constexpr (RPW > 1) {
      __syncthreads();
      if (sub)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < E; ++i) acc[(((sub - 1) * CH + c) * E + i) * TPR + t] = which ? db[c][i] : dg[c][i];
      __syncthreads();
      if (sub) continue;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int at = col_of<WIDE, T, TPR>(c, t, i);
        float v = which ? db[c][i] : dg[c][i];
        if constexpr (RPW > 1)
#pragma unroll
          for (int r = 1; r < RPW; ++r) v += acc[(((r - 1) * CH + c) * E + i) * TPR + t];
        if (at < a.d) out[at] = v;
      }
  }
}

// dgain += the workgroups' sums, dshift likewise (blockIdx.y 1): 32 columns and 32 shares of the groups per workgroup
__global__ __launch_bounds__(1024) void norm_sums_k(NormArgs a) {
  __shared__ float red[32][33];
  float* dst = blockIdx.y ? a.dshift : a.dgain;
  if (!dst) return;
  const int col = threadIdx.x & 31, share = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
  float v = 0.f;
  if (c < a.d) {
    const float* p = a.part + (long)blockIdx.y * a.d + c;
#pragma unroll 8
    for (int g = share; g < a.groups; g += 32) v += p[(long)g * 2 * a.d];
  }
  red[share][col] = v;
  __syncthreads();
  if (share || c >= a.d) return;
  v = 0.f;
#pragma unroll
  for (int s = 0; s < 32; ++s) v += red[s][col];
  dst[c] += v;
}

// threads per row and pieces per thread
struct NormShape {
  int tpr, ch;
};
static NormShape norm_shape(int dtype, int d, bool back) {
  const int pieces = (d + (dtype == DT_BF16 ? 7 : 3)) / (dtype == DT_BF16 ? 8 : 4);
  // up to four pieces to a lane in the forward, two in the backward, which holds three rows and the columns' sums
  for (int tpr : {64, 256, 1024})
    for (int ch : {1, 2, 4})
      if (tpr * ch >= pieces && (!back || ch < 4 || tpr == 1024)) return {tpr, ch};
  return {0, 0};
}

int norm_groups(int dtype, long rows, int d) {
  const NormShape f = norm_shape(dtype, d, true);
  const int rpw = f.tpr >= 256 ? 1 : 256 / f.tpr;
  const long wgs = (rows + rpw - 1) / rpw;
  return (int)(wgs < 512 ? wgs : 512);  // 16384 x 4096: 256 and 1024 were slower
}

static bool rows_wide(const NormRows& r, int es) {
  return r.p == nullptr || ((reinterpret_cast<uintptr_t>(r.p) & 15u) == 0 && (r.t * es & 15) == 0);
}

template <typename T, int TPR, int CH, bool WIDE>
static hipError_t norm_go(const NormArgs& a, bool back, hipStream_t s) {
  constexpr int NT = TPR > 256 ? TPR : 256, RPW = NT / TPR;
  if (back) {
    constexpr bool ahead = WIDE && CH * VE<T> <= 16 && (TPR < 1024 || CH == 1);
    if constexpr (CH < 4 || TPR == 1024) RG_LAUNCH((norm_bwd_k<T, TPR, CH, ahead, WIDE>), dim3(a.groups), dim3(NT), 0, s, a);
    else return hipErrorInvalidValue;
    if (a.part) RG_LAUNCH(norm_sums_k, dim3((a.d + 31) / 32, 2), dim3(1024), 0, s, a);
  } else if constexpr (CH > 1 || TPR == 64) {
    // HIP takes fewer than 2^32 threads in a dimension of a launch
    const long wgs = (a.rows + RPW - 1) / RPW, y = (wgs + (1l << 21) - 1) >> 21;
    RG_LAUNCH((norm_fwd_k<T, TPR, CH, WIDE>), dim3((unsigned)((wgs + y - 1) / y), (unsigned)y), dim3(NT), 0, s, a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T, bool WIDE>
static hipError_t norm_shapes(const NormShape& f, const NormArgs& a, bool back, hipStream_t s) {
  switch (f.tpr * 8 + f.ch) {
    case 64 * 8 + 1: return norm_go<T, 64, 1, WIDE>(a, back, s);
    case 64 * 8 + 2: return norm_go<T, 64, 2, WIDE>(a, back, s);
    case 64 * 8 + 4: return norm_go<T, 64, 4, WIDE>(a, back, s);
    case 256 * 8 + 1: return norm_go<T, 256, 1, WIDE>(a, back, s);
    case 256 * 8 + 2: return norm_go<T, 256, 2, WIDE>(a, back, s);
    case 256 * 8 + 4: return norm_go<T, 256, 4, WIDE>(a, back, s);
    case 1024 * 8 + 1: return norm_go<T, 1024, 1, WIDE>(a, back, s);
    case 1024 * 8 + 2: return norm_go<T, 1024, 2, WIDE>(a, back, s);
    case 1024 * 8 + 4:  // fp32 alone has rows of as many pieces
      if constexpr (sizeof(T) == 4) return norm_go<T, 1024, 4, WIDE>(a, back, s);
  }
  return hipErrorInvalidValue;
}

template <typename T>
static hipError_t norm_t(int dtype, const NormArgs& a, bool back, hipStream_t s) {
  const int es = sizeof(T);
  const auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
  const bool wide = a.d % VE<T> == 0 && rows_wide(a.x, es) && rows_wide(a.res, es) && rows_wide(a.s, es) &&
                    rows_wide(a.y, es) && rows_wide(a.dy, es) && rows_wide(a.dskip, es) && rows_wide(a.dx, es) &&
                    al(a.gain) && al(a.shift);
  const NormShape f = norm_shape(dtype, a.d, back);
  return wide ? norm_shapes<T, true>(f, a, back, s) : norm_shapes<T, false>(f, a, back, s);
}

hipError_t launch_norm_fwd(int dtype, const NormArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? norm_t<bf16>(dtype, a, false, s) : norm_t<float>(dtype, a, false, s);
}
hipError_t launch_norm_bwd(int dtype, const NormArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? norm_t<bf16>(dtype, a, true, s) : norm_t<float>(dtype, a, true, s);
}

}  // namespace rg
