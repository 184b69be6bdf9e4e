// Dropout from a counter-based generator: y = [res +] keep / (1 - p) x, the mask formed
// from (seed, offset, site, element) wherever it is needed and never stored, so the backward is
// the same kernel on dY.
//
// Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011): ten rounds of two 32 x 32 -> 64 bit products turn a 128-bit
// counter and a 64-bit key into four words.  One evaluation serves the eight elements of a
// chunk, 16 bits each (16 B of bf16), so p comes in steps of 2^-16 and the twenty
// products are spread over eight elements; the factor is 1 / (1 - p) for that p.
//
// Bound by memory: one chunk per thread, 67 M bf16 elements with a residual 73 us (5.5 TB/s),
// 3.1 M 5.5 us, which is the launch.
#include "common.h"
#include "kernels.h"

namespace rg {

struct Philox {
  uint32_t w[4];
};
__device__ __forceinline__ Philox philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                                uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint32_t h0 = __umulhi(c0, 0xD2511F53u), l0 = c0 * 0xD2511F53u;
    const uint32_t h1 = __umulhi(c2, 0xCD9E8D57u), l1 = c2 * 0xCD9E8D57u;
    c0 = h1 ^ c1 ^ k0;
    c1 = l1;
    c2 = h0 ^ c3 ^ k1;
    c3 = l0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_k(const T* x, const T* res, T* y, long n, uint32_t thr, float f,
                                                 const uint64_t* rng, uint32_t site, bool wide) {
  const long c = ((long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  if (c * 8 >= n) return;
  const uint64_t seed = rng[0], off = rng[1];
  const Philox u = philox4x32_10((uint32_t)c, site, (uint32_t)off, (uint32_t)(off >> 32), (uint32_t)seed,
                                 (uint32_t)(seed >> 32));
  float v[8], r[8];
  const bool whole = wide && c * 8 + 8 <= n;
  if (whole) {
    St<T>::ld4(x, c * 8, v);
    St<T>::ld4(x, c * 8 + 4, v + 4);
    if (RES) {
      St<T>::ld4(res, c * 8, r);
      St<T>::ld4(res, c * 8 + 4, r + 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long at = c * 8 + i;
      v[i] = at < n ? St<T>::ld(x, at) : 0.f;
      if (RES) r[i] = at < n ? St<T>::ld(res, at) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t h = (u.w[i >> 1] >> (16 * (i & 1))) & 0xffffu;
    v[i] = h >= thr ? v[i] * f : 0.f;
    if (RES) v[i] += r[i];
  }
  if (whole) {
    St<T>::st4(y, c * 8, v);
    St<T>::st4(y, c * 8 + 4, v + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c * 8 + i < n) St<T>::st(y, c * 8 + i, v[i]);
  }
}

template <typename T>
static hipError_t dropout_t(const void* x, const void* res, void* y, long n, uint32_t thr, const uint64_t* rng,
                            uint32_t site, hipStream_t s) {
  const float f = 65536.f / (65536.f - (float)thr);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(res)) & 15u) == 0;
  // HIP takes fewer than 2^32 threads in a dimension of a launch: from 2^34 elements on, more than one row of them
  const long wgs = (n + 2047) / 2048, rows = (wgs + (1l << 23) - 1) >> 23;
  const dim3 grid((unsigned)((wgs + rows - 1) / rows), (unsigned)rows), block(256);
  if (res)
    RG_LAUNCH((dropout_k<T, true>), grid, block, 0, s, static_cast<const T*>(x), static_cast<const T*>(res),
              static_cast<T*>(y), n, thr, f, rng, site, wide);
  else
    RG_LAUNCH((dropout_k<T, false>), grid, block, 0, s, static_cast<const T*>(x), static_cast<const T*>(nullptr),
              static_cast<T*>(y), n, thr, f, rng, site, wide);
  return hipGetLastError();
}

hipError_t launch_dropout(int dtype, const void* x, const void* res, void* y, long n, uint32_t thr,
                          const uint64_t* rng, uint32_t site, hipStream_t s) {
  return dtype == DT_BF16 ? dropout_t<bf16>(x, res, y, n, thr, rng, site, s)
                          : dropout_t<float>(x, res, y, n, thr, rng, site, s);
}

}  // namespace rg
