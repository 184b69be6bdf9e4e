// The block operators behind the C ABI: attention with a window, sinks and a relative
// position bias, and dropout.  Argument checks and the kernels' argument
// structs; nothing here allocates or keeps anything.
#include <math.h>

#include <utility>

#include "kernels.h"
#include "ringada.h"
#include "status.h"

using namespace rg;

static MaskedAttnArgs attn_sizes(const ringada_attn_desc& D) {
  MaskedAttnArgs a{};
  a.B = D.batch; a.H = D.n_heads; a.Hkv = D.n_kv_heads; a.dh = D.d_head; a.Sq = D.seq_q; a.Sk = D.seq_k;
  a.causal = D.causal != 0;
  // no two rows are seq_q + seq_k apart: such a window hides nothing
  a.window = D.window >= D.seq_q + D.seq_k ? 0 : D.window;
  a.sinks = D.sinks < D.seq_k ? D.sinks : D.seq_k;
  a.scale = D.scale;
  a.R = D.n_buckets ? D.max_distance : 0;
  a.nb = D.n_buckets;
  return a;
}

static ringada_status check_attn(const ringada_attn_desc* D) {
  if (!D) return fail(RINGADA_E_INVALID, "desc is NULL");
  if (D->dtype != RINGADA_F32 && D->dtype != RINGADA_BF16) return fail(RINGADA_E_INVALID, "unknown dtype %d", D->dtype);
  if (D->batch < 1 || D->n_heads < 1 || D->n_kv_heads < 1 || D->d_head < 1 || D->seq_q < 1 || D->seq_k < 1)
    return fail(RINGADA_E_INVALID, "sizes must be positive");
  if (D->n_heads % D->n_kv_heads) return fail(RINGADA_E_INVALID, "n_heads %% n_kv_heads != 0");
  if (D->window < 0 || D->sinks < 0) return fail(RINGADA_E_INVALID, "window and sinks must be >= 0");
  if (!(D->scale > 0.f) || !isfinite(D->scale)) return fail(RINGADA_E_INVALID, "scale must be positive and finite");
  if (D->n_buckets < 0 || D->n_buckets > 65535 || D->max_distance < 0)
    return fail(RINGADA_E_INVALID, "n_buckets must be in [0, 65535] and max_distance >= 0");
  if (D->max_distance > ATTN_MAX_DISTANCE) return fail(RINGADA_E_UNSUPPORTED, "max_distance above %d", ATTN_MAX_DISTANCE);
  if (D->dtype == RINGADA_BF16 && D->d_head != 64 && D->d_head != 128)
    return fail(RINGADA_E_UNSUPPORTED, "bf16 path: d_head must be 64 or 128 (got %d)", D->d_head);
  if (D->d_head > 128) return fail(RINGADA_E_UNSUPPORTED, "f32 path: d_head must be at most 128 (got %d)", D->d_head);
  if (D->seq_q > (1 << 24) || D->seq_k > (1 << 24)) return fail(RINGADA_E_UNSUPPORTED, "sequences above 2^24 rows");
  const int64_t rows = D->seq_q > D->seq_k ? D->seq_q : D->seq_k;
  if ((int64_t)D->batch * D->n_heads * ((rows + 31) / 32) >= (1ll << 31) || D->n_heads > 65535 ||
      !masked_attn_fits(D->dtype, attn_sizes(*D)))
    return fail(RINGADA_E_UNSUPPORTED, "too many rows for one launch");
  return RINGADA_OK;
}

// writes: no two elements of the view may share an address
static ringada_status check_view(const ringada_attn_desc& D, const char* name, const ringada_view& v, int64_t rows,
                                 int64_t heads, bool writes, View& out) {
  if (!v.data) return fail(RINGADA_E_INVALID, "%s is NULL", name);
  const uintptr_t p = reinterpret_cast<uintptr_t>(v.data);
  int64_t stride[3] = {v.batch, v.row, v.head}, n[3] = {D.batch, rows, heads};
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) stride[i] = 0;  // whatever it is, it leads nowhere
    if (stride[i] < 0 || stride[i] >= (1ll << 40) || (n[i] > 1 && stride[i] > (1ll << 46) / (n[i] - 1)))
      return fail(RINGADA_E_INVALID, "%s: stride out of range", name);  // 2^46 elements: no address space holds more
  }
  out = View{v.data, (long)stride[0], (long)stride[1], (long)stride[2]};
  if (D.dtype == RINGADA_BF16 ? ((p & 15u) || ((stride[0] | stride[1] | stride[2]) & 7)) : (p & 3u))
    return fail(RINGADA_E_INVALID, "%s: bf16 views need 16-byte aligned data and strides that are multiples of 8, "
                                   "f32 views 4-byte aligned data", name);
  if (stride[1] >= (1 << 24)) return fail(RINGADA_E_UNSUPPORTED, "%s: row stride above 2^24 elements", name);
  if (writes) {
    for (int i = 0; i < 2; ++i)  // by stride, smallest first
      for (int j = 0; j < 2 - i; ++j)
        if (stride[j] > stride[j + 1]) {
          std::swap(stride[j], stride[j + 1]);
          std::swap(n[j], n[j + 1]);
        }
    int64_t extent = D.d_head;
    for (int i = 0; i < 3; ++i) {
      if (n[i] == 1) continue;
      if (stride[i] < extent) return fail(RINGADA_E_INVALID, "%s: rows of an output overlap", name);
      extent = stride[i] * (n[i] - 1) + extent;
    }
  }
  return RINGADA_OK;
}

// What a tensor takes in memory: runs of len bytes, n[i] of them every stride[i] bytes.
struct Region {
  const char* name;
  uintptr_t p;
  int64_t len, stride[3], n[3];
};
static Region flat(const char* name, const void* p, size_t bytes) {
  return {name, reinterpret_cast<uintptr_t>(p), (int64_t)bytes, {0, 0, 0}, {1, 1, 1}};
}
static Region region(const char* name, const ringada_attn_desc& D, const View& v, int64_t rows, int64_t heads) {
  const int64_t es = D.dtype == RINGADA_BF16 ? 2 : 4;
  return {name, reinterpret_cast<uintptr_t>(v.p), D.d_head * es, {v.b * es, v.t * es, v.h * es}, {D.batch, rows, heads}};
}
// Whether d + sum of c_k s_k, lo_k <= c_k <= hi_k, falls between -below and above: strides in falling order, each
// coefficient tried where the smaller ones can still reach.  In tensors of one buffer, whose strides are
// the same, that is two or three values a stride.
struct Search {
  int64_t s[6], lo[6], hi[6], rest_lo[7], rest_hi[7], below, above;
  int n = 0, left = 1 << 16;
  bool hit(int k, int64_t d) {
    if (k == n) return -below < d && d < above;
    auto floor_div = [](int64_t a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
    const int64_t c0 = -floor_div(d + rest_hi[k + 1] + below - 1, s[k]);
    const int64_t c1 = floor_div(above - 1 - d - rest_lo[k + 1], s[k]);
    for (int64_t c = c0 > lo[k] ? c0 : lo[k]; c <= c1 && c <= hi[k] && left-- > 0; ++c)
      if (hit(k + 1, d + c * s[k])) return true;
    return false;
  }
};
// Exact, but for tensors of different strides woven into each other beyond the search's limit
static bool overlap(const Region& a, const Region& b) {
  if (!a.p || !b.p || !a.len || !b.len) return false;
  int64_t ea = a.len, eb = b.len;
  for (int i = 0; i < 3; ++i) {
    ea += a.stride[i] * (a.n[i] - 1);
    eb += b.stride[i] * (b.n[i] - 1);
  }
  if (a.p + ea <= b.p || b.p + eb <= a.p) return false;
  Search f;
  f.below = b.len;
  f.above = a.len;
  for (int i = 0; i < 6; ++i) {  // from a's run to b's: b's strides forwards, a's back
    const Region& r = i < 3 ? a : b;
    const int64_t s = r.stride[i % 3], m = r.n[i % 3] - 1;
    if (!s || !m) continue;
    int at = 0;
    while (at < f.n && f.s[at] > s) ++at;
    if (at == f.n || f.s[at] != s) {
      for (int k = f.n++; k > at; --k) {
        f.s[k] = f.s[k - 1];
        f.lo[k] = f.lo[k - 1];
        f.hi[k] = f.hi[k - 1];
      }
      f.s[at] = s;
      f.lo[at] = f.hi[at] = 0;
    }
    (i < 3 ? f.lo[at] : f.hi[at]) += i < 3 ? -m : m;
  }
  f.rest_lo[f.n] = f.rest_hi[f.n] = 0;
  for (int k = f.n - 1; k >= 0; --k) {
    f.rest_lo[k] = f.rest_lo[k + 1] + f.lo[k] * f.s[k];
    f.rest_hi[k] = f.rest_hi[k + 1] + f.hi[k] * f.s[k];
  }
  return f.hit(0, (int64_t)(b.p - a.p));
}
// none of all[n_in .. n - 1], the outputs, may overlap an input (those before) or another output
static ringada_status check_apart(const Region* all, int n_in, int n) {
  for (int i = n_in; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(all[i], all[j])) return fail(RINGADA_E_INVALID, "%s overlaps %s", all[i].name, all[j].name);
  return RINGADA_OK;
}

static ringada_status fill_tensors(const ringada_attn_desc& D, const ringada_attn_tensors* t, MaskedAttnArgs& a) {
  if (!t) return fail(RINGADA_E_INVALID, "tensors is NULL");
  RG_TRY(check_view(D, "q", t->q, D.seq_q, D.n_heads, false, a.q));
  RG_TRY(check_view(D, "k", t->k, D.seq_k, D.n_kv_heads, false, a.k));
  RG_TRY(check_view(D, "v", t->v, D.seq_k, D.n_kv_heads, false, a.v));
  RG_TRY(check_view(D, "o", t->o, D.seq_q, D.n_heads, true, a.o));
  if ((t->table != nullptr) != (D.n_buckets > 0) || (t->table && !t->bucket))
    return fail(RINGADA_E_INVALID, "table and bucket must be given exactly when n_buckets > 0");
  a.lse = t->lse;
  a.len_q = t->len_q;
  a.len_k = t->len_k;
  a.table = t->table;
  a.bucket = t->bucket;
  return RINGADA_OK;
}
// what both passes read; returns how many
static int read_regions(const ringada_attn_desc& D, const MaskedAttnArgs& a, Region* in) {
  in[0] = region("q", D, a.q, D.seq_q, D.n_heads);
  in[1] = region("k", D, a.k, D.seq_k, D.n_kv_heads);
  in[2] = region("v", D, a.v, D.seq_k, D.n_kv_heads);
  in[3] = flat("len_q", a.len_q, (size_t)D.batch * 4);
  in[4] = flat("len_k", a.len_k, (size_t)D.batch * 4);
  in[5] = flat("table", a.table, (size_t)D.n_buckets * D.n_heads * 4);
  in[6] = flat("bucket", a.table ? a.bucket : nullptr, ((size_t)D.max_distance * 2 + 1) * 4);
  return 7;
}

static ringada_status check_workspace(const void* ws, size_t have, size_t need, const Region* all, int n) {
  if (have < need || (need && !ws))
    return fail(RINGADA_E_WORKSPACE, "workspace of %zu bytes, the call needs %zu", ws ? have : (size_t)0, need);
  if (need && (reinterpret_cast<uintptr_t>(ws) & 255u)) return fail(RINGADA_E_INVALID, "workspace must be 256-byte aligned");
  const Region w = flat("workspace", ws, need);
  for (int i = 0; i < n; ++i)
    if (overlap(w, all[i])) return fail(RINGADA_E_INVALID, "the workspace overlaps %s", all[i].name);
  return RINGADA_OK;
}

extern "C" ringada_status ringada_attn_plan(const ringada_attn_desc* desc, int32_t with_dtable, size_t* forward_bytes,
                                            size_t* backward_bytes) {
  RG_TRY(check_attn(desc));
  size_t f, b;
  masked_attn_bytes(desc->dtype, attn_sizes(*desc), with_dtable && desc->n_buckets, &f, &b);
  if (forward_bytes) *forward_bytes = f;
  if (backward_bytes) *backward_bytes = b;
  return RINGADA_OK;
}

extern "C" ringada_status ringada_attn_forward(void* stream, const ringada_attn_desc* desc,
                                               const ringada_attn_tensors* t, void* workspace,
                                               size_t workspace_bytes) {
  RG_TRY(check_attn(desc));
  MaskedAttnArgs a = attn_sizes(*desc);
  RG_TRY(fill_tensors(*desc, t, a));
  Region all[9];
  const int n_in = read_regions(*desc, a, all);
  all[n_in] = region("o", *desc, a.o, desc->seq_q, desc->n_heads);
  all[n_in + 1] = flat("lse", t->lse, (size_t)desc->batch * desc->n_heads * desc->seq_q * 4);
  RG_TRY(check_apart(all, n_in, n_in + 2));
  size_t need, unused;
  masked_attn_bytes(desc->dtype, a, false, &need, &unused);
  RG_TRY(check_workspace(workspace, workspace_bytes, need, all, n_in + 2));
  a.part = static_cast<float*>(workspace);
  RG_HIP(launch_masked_attn_fwd(desc->dtype, a, static_cast<hipStream_t>(stream)));
  return RINGADA_OK;
}

extern "C" ringada_status ringada_attn_backward(void* stream, const ringada_attn_desc* desc,
                                                const ringada_attn_tensors* t, const ringada_attn_grads* g,
                                                void* workspace, size_t workspace_bytes) {
  RG_TRY(check_attn(desc));
  MaskedAttnArgs a = attn_sizes(*desc);
  RG_TRY(fill_tensors(*desc, t, a));
  if (!g) return fail(RINGADA_E_INVALID, "grads is NULL");
  if (!t->lse) return fail(RINGADA_E_INVALID, "the backward needs the forward's lse");
  RG_TRY(check_view(*desc, "dout", g->dout, desc->seq_q, desc->n_heads, false, a.dout));
  RG_TRY(check_view(*desc, "dq", g->dq, desc->seq_q, desc->n_heads, true, a.dq));
  RG_TRY(check_view(*desc, "dk", g->dk, desc->seq_k, desc->n_kv_heads, true, a.dk));
  RG_TRY(check_view(*desc, "dv", g->dv, desc->seq_k, desc->n_kv_heads, true, a.dv));
  if (g->dtable && !desc->n_buckets) return fail(RINGADA_E_INVALID, "dtable without a table");
  a.dtable = g->dtable;
  const int64_t H = desc->n_heads, Hkv = desc->n_kv_heads;
  Region all[14];
  int n_in = read_regions(*desc, a, all);
  all[n_in++] = region("o", *desc, a.o, desc->seq_q, H);
  all[n_in++] = region("dout", *desc, a.dout, desc->seq_q, H);
  all[n_in++] = flat("lse", t->lse, (size_t)desc->batch * H * desc->seq_q * 4);
  all[n_in] = region("dq", *desc, a.dq, desc->seq_q, H);
  all[n_in + 1] = region("dk", *desc, a.dk, desc->seq_k, Hkv);
  all[n_in + 2] = region("dv", *desc, a.dv, desc->seq_k, Hkv);
  all[n_in + 3] = flat("dtable", g->dtable, (size_t)desc->n_buckets * H * 4);
  RG_TRY(check_apart(all, n_in, n_in + 4));
  size_t need, unused;
  masked_attn_bytes(desc->dtype, a, g->dtable != nullptr, &unused, &need);
  RG_TRY(check_workspace(workspace, workspace_bytes, need, all, n_in + 4));
  masked_attn_workspace(desc->dtype, a, workspace);
  RG_HIP(launch_masked_attn_bwd(desc->dtype, a, static_cast<hipStream_t>(stream)));
  return RINGADA_OK;
}

// A whole number of up to 328 32-bit words: 1024^1024 and 16 words to spare.
struct Whole {
  int n = 1;
  uint32_t w[328] = {1};
  void times(uint32_t f, int power) {
    for (; power > 0; --power) {
      uint64_t carry = 0;
      for (int i = 0; i < n; ++i) {
        carry += (uint64_t)w[i] * f;
        w[i] = (uint32_t)carry;
        carry >>= 32;
      }
      if (carry) w[n++] = (uint32_t)carry;
    }
  }
  bool operator>=(const Whole& o) const {
    if (n != o.n) return n > o.n;
    for (int i = n - 1; i >= 0; --i)
      if (w[i] != o.w[i]) return w[i] > o.w[i];
    return true;
  }
};
// d >= one (dist / one)^(k / m), 1 <= k <= m <= 1024, all of them at most 1024.  The power is off by some 1e-16 of
// it; a distance nearer than that allows is compared in whole numbers, d^m with dist^k one^(m - k): some
// reach the power exactly, others lie within 1e-10 of it without reaching it.
static bool reaches(int d, int one, int dist, int k, int m) {
  const long double power = one * powl((long double)dist / one, k / (long double)m);
  if (fabsl(d - power) > 1e-12L * power) return d > power;
  Whole a, b;
  a.times(d, m);
  b.times(dist, k);
  b.times(one, m - k);
  return a >= b;
}

extern "C" ringada_status ringada_relpos_buckets(int32_t n_buckets, int32_t max_distance, int32_t bidirectional,
                                                 int32_t* map) {
  if (!map) return fail(RINGADA_E_INVALID, "map is NULL");
  const int n = bidirectional ? n_buckets / 2 : n_buckets, one = n / 2;
  if (n_buckets < 2 || (bidirectional && n_buckets % 2) || one < 1)
    return fail(RINGADA_E_INVALID, "n_buckets must be at least 2, or a multiple of 2 from 4 when bidirectional");
  if (max_distance <= one || max_distance > ATTN_MAX_DISTANCE)
    return fail(RINGADA_E_INVALID, "max_distance must be in (%d, %d]", one, ATTN_MAX_DISTANCE);
  for (int r = -max_distance; r <= max_distance; ++r) {
    const int d = bidirectional ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
    int t = d;
    if (d >= one) {
      // one + k for the largest k with d >= one (max_distance / one)^(k / (n - one))
      int k = 0;
      while (k < n - one && reaches(d, one, max_distance, k + 1, n - one)) ++k;
      t = one + k < n ? one + k : n - 1;
    }
    map[r + max_distance] = t + (bidirectional && r > 0 ? n : 0);
  }
  return RINGADA_OK;
}

// ================================================================ dropout
static bool same_or_apart(const void* a, const void* b, size_t n) {
  const char* x = static_cast<const char*>(a);
  const char* y = static_cast<const char*>(b);
  return x == y || x + n <= y || y + n <= x;
}

extern "C" ringada_status ringada_dropout(void* stream, int32_t dtype, const void* x, const void* res, void* y,
                                          int64_t n, float p, const uint64_t* rng, uint32_t site) {
  if (dtype != RINGADA_F32 && dtype != RINGADA_BF16) return fail(RINGADA_E_INVALID, "unknown dtype");
  if (!x || !y || !rng || n <= 0 || n > (1ll << 35)) return fail(RINGADA_E_INVALID, "bad argument");
  if (!(p >= 0.f && p < 1.f)) return fail(RINGADA_E_INVALID, "p must be in [0, 1)");
  const uint32_t thr = dropout_threshold(p);
  if (thr > 65535) return fail(RINGADA_E_INVALID, "p rounds to 1 in steps of 2^-16");
  const size_t es = dtype == RINGADA_BF16 ? 2 : 4, bytes = (size_t)n * es;
  const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(res) | reinterpret_cast<uintptr_t>(y);
  if ((all & (es - 1)) || (reinterpret_cast<uintptr_t>(rng) & 7u)) return fail(RINGADA_E_INVALID, "misaligned tensor");
  if (!same_or_apart(x, y, bytes) || (res && !same_or_apart(res, y, bytes)))
    return fail(RINGADA_E_INVALID, "y overlaps x or res without being the same tensor");
  RG_HIP(launch_dropout(dtype, x, res, y, n, thr, rng, site, static_cast<hipStream_t>(stream)));
  return RINGADA_OK;
}
