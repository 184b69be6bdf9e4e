// Rotary embedding: pair (i, i + P) of a head, i < P, turns by angle pos[axis of i] * freq[i]:
//
//   o_i = x_i cos - x_{i+P} sin,   o_{i+P} = x_{i+P} cos + x_i sin
//
// and by the opposite angle for the inverse, which is the backward.  Dimensions from 2 P on
// are copied.
//
// Angles of far positions need more than 32 bits: a position of 10^6 has turned some
// 10^5 times, which leaves fp32 no digit of the angle's place in the turn.  The turns are counted in 64 bits,
// the whole ones dropped, and only the rest rounded.  That costs a few 64-bit operations per row and pair, shared by all
// heads: a workgroup forms its rows' (cos, sin) once, in LDS.
//
// Bound by memory: 2 x 4097 rows of 16 + 16 heads of 128 in bf16 take 26 us each way, 5.1 TB/s.
#include "common.h"
#include "kernels.h"

namespace rg {

template <typename T, int VE>
__device__ __forceinline__ void ld_n(const T* p, float v[VE]) {
  if constexpr (VE == 8) {
    unpack_frag(*reinterpret_cast<const bf16x8*>(p), v);
  } else if constexpr (VE == 4) {
    St<T>::ld4(p, 0, v);
  } else {
    v[0] = St<T>::ld(p, 0);
  }
}
template <typename T, int VE>
__device__ __forceinline__ void st_n(T* p, const float v[VE]) {
  if constexpr (VE == 8) {
    *reinterpret_cast<bf16x8*>(p) = pack_frag(v);
  } else if constexpr (VE == 4) {
    St<T>::st4(p, 0, v);
  } else {
    St<T>::st(p, 0, v[0]);
  }
}

// VE elements at a time (16 bytes, or one); rows_wg rows per workgroup, its heads dealt over gridDim.y
template <typename T, int VE>
__global__ __launch_bounds__(256) void rotary_k(RotaryArgs a, int rows_wg) {
  __shared__ float2 cs[ROTARY_MAX_PAIRS];
  const long n_rows = (long)a.B * a.S, row0 = (long)blockIdx.x * rows_wg;
  const int rows = (int)(n_rows - row0 < rows_wg ? n_rows - row0 : rows_wg);
  for (int i = threadIdx.x; i < rows * a.pairs; i += 256) {
    const int r = i / a.pairs, j = i % a.pairs;
    int axis = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e) axis += e + 1 < a.axes && j >= a.end[e] ? 1 : 0;
    const double turns = (double)a.pos[axis * n_rows + row0 + r] * (a.freq[j] * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();
  const int pc = a.pairs / VE, rc = (a.dh - 2 * a.pairs) / VE, per_head = pc + rc, heads = a.H + a.Hkv;
  const int h0 = (int)((long)heads * blockIdx.y / gridDim.y), h1 = (int)((long)heads * (blockIdx.y + 1) / gridDim.y);
  for (int i = threadIdx.x; i < rows * (h1 - h0) * per_head; i += 256) {
    const int c = i % per_head, h = h0 + i / per_head % (h1 - h0), r = i / per_head / (h1 - h0);
    const long row = row0 + r, b = row / a.S, t = row % a.S;
    const bool isk = h >= a.H;
    const View& in = isk ? a.k : a.q;
    const View& out = isk ? a.ok : a.oq;
    const int hh = isk ? h - a.H : h;
    const T* x = static_cast<const T*>(in.p) + b * in.b + t * in.t + hh * in.h;
    T* o = static_cast<T*>(out.p) + b * out.b + t * out.t + hh * out.h;
    float u[VE], v[VE];
    if (c < pc) {
      ld_n<T, VE>(x + c * VE, u);
      ld_n<T, VE>(x + a.pairs + c * VE, v);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 z = cs[r * a.pairs + c * VE + e];
        const float p = u[e], q = v[e];
        u[e] = p * z.x - q * z.y;
        v[e] = q * z.x + p * z.y;
      }
      st_n<T, VE>(o + c * VE, u);
      st_n<T, VE>(o + a.pairs + c * VE, v);
    } else {
      const int at = 2 * a.pairs + (c - pc) * VE;
      ld_n<T, VE>(x + at, u);
      st_n<T, VE>(o + at, u);
    }
  }
}

static bool wide_ok(const View& v, int es) {
  return v.p == nullptr || ((reinterpret_cast<uintptr_t>(v.p) & 15u) == 0 && ((v.b | v.t | v.h) * es & 15) == 0);
}

template <typename T, int VE>
static hipError_t rotary_t(const RotaryArgs& a, hipStream_t s) {
  const long rows = (long)a.B * a.S;
  // angles for every thread where rows are many; few rows are spread over their heads
  int rows_wg = rows >= 1024 ? 256 / a.pairs : 1;
  if (rows_wg < 1) rows_wg = 1;
  const long wgs = (rows + rows_wg - 1) / rows_wg;
  const int heads = a.H + a.Hkv, split = wgs >= 256 ? 1 : heads < 8 ? heads : 8;
  const bool wide = VE > 1 && a.pairs % VE == 0 && a.dh % VE == 0 && wide_ok(a.q, sizeof(T)) && wide_ok(a.k, sizeof(T)) &&
                    wide_ok(a.oq, sizeof(T)) && wide_ok(a.ok, sizeof(T));
  if (wide) RG_LAUNCH((rotary_k<T, VE>), dim3((unsigned)wgs, split), dim3(256), 0, s, a, rows_wg);
  else RG_LAUNCH((rotary_k<T, 1>), dim3((unsigned)wgs, split), dim3(256), 0, s, a, rows_wg);
  return hipGetLastError();
}

hipError_t launch_rotary(int dtype, const RotaryArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? rotary_t<bf16, 8>(a, s) : rotary_t<float, 4>(a, s);
}

}  // namespace rg
