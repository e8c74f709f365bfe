// Paged cache: argument checks, rotary frequencies and dispatch of the C entry points.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "aatc.h"
#include "aatc_internal.h"
#include "paged.h"

namespace {

using namespace aatc;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// log2 of the page size, or -1 for a descriptor that no entry point takes
int page_shift(const aatc_pages_t* d) {
  if (!d || (d->dtype != AATC_BF16 && d->dtype != AATC_F16) || d->n_kv_heads < 1 || d->n_kv_heads > 4096 ||
      d->n_pages < 1 || d->n_pages > (1 << 24))
    return -1;
  for (int s = 3; s <= 8; ++s)
    if (d->page_size == 1 << s)
      return (static_cast<uint64_t>(d->n_pages) * d->n_kv_heads * d->page_size) <= (1ull << 40) / (4 * D) ? s : -1;
  return -1;
}

size_t page_bytes(const aatc_pages_t* d) { return static_cast<size_t>(2) * d->n_kv_heads * d->page_size * D * 2; }

bool heads_ok(const aatc_heads_t* h) {
  return h && h->x && aligned16(h->x) && h->token_stride % 8 == 0 && h->head_stride % 8 == 0;
}

// Whether no two of the n_tokens x n_heads heads at these strides overlap, as the ones that a call writes must not (of a
// tensor that is broadcast, they all do; and where it is turned in place, some would be turned twice).
bool apart(int64_t token_stride, int64_t head_stride, int64_t n_tokens, int64_t n_heads) {
  using wide = __int128;
  const wide a = token_stride < 0 ? -static_cast<wide>(token_stride) : token_stride;
  const wide b = head_stride < 0 ? -static_cast<wide>(head_stride) : head_stride;
  if ((n_tokens > 1 && a < D) || (n_heads > 1 && b < D)) return false;
  if (n_tokens <= 1 || n_heads <= 1 || a >= (n_heads - 1) * b + D || b >= (n_tokens - 1) * a + D) return true;
  for (int64_t i = 1; i < n_heads; ++i) {            // neither within the other: the heads nearest to i heads on
    const wide j = i * b / a, off = i * b - j * a;
    if ((j < n_tokens && off < D) || (j + 1 < n_tokens && a - off < D)) return false;
  }
  return true;
}

paged::Heads heads(const aatc_heads_t* h) { return {h->x, h->token_stride, h->head_stride}; }

bool rope_ok(const aatc_rotary_t* r) {
  return r && r->turns && (reinterpret_cast<uintptr_t>(r->turns) & 7u) == 0 && r->rot_dim >= 16 && r->rot_dim <= D &&
         r->rot_dim % 16 == 0 && (r->interleaved == 0 || r->interleaved == 1) && std::isfinite(r->factor);
}

paged::Turn turn(const aatc_rotary_t* r, bool backward) {
  return {r->turns, r->rot_dim, r->interleaved, r->factor, backward ? -1.0f : 1.0f};
}

bool table_ok(const int32_t* table, int32_t n_rows, int32_t table_stride, int32_t max_pages) {
  return table && aligned4(table) && n_rows >= 1 && max_pages >= 1 && table_stride >= 0;
}

paged::Pool pool(const aatc_pages_t* d, void* pages, const int32_t* table, int32_t table_stride, int32_t max_pages,
                 int32_t* flags) {
  return {pages, table, table_stride, max_pages, d->n_pages, d->n_kv_heads, page_shift(d), flags};
}

// SMs of the current device (a property that cannot change: asked once per device and thread).
cudaError_t sm_count(int* sms) {
  static thread_local int known_dev = -1, known = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev != known_dev) {
    e = cudaDeviceGetAttribute(&known, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    known_dev = dev;
  }
  *sms = known;
  return cudaSuccess;
}

}  // namespace

extern "C" {

aatc_status_t aatc_pages_bytes(const aatc_pages_t* pages, size_t* bytes) {
  if (!bytes || page_shift(pages) < 0) return AATC_ERR_INVALID_ARG;
  *bytes = page_bytes(pages) * pages->n_pages;
  return AATC_OK;
}

aatc_status_t aatc_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double scale, int32_t original,
                                      double p0, double p1, double* freq_out, double* factor_out) {
  const bool plain = scaling == AATC_ROPE_PLAIN;
  const bool ranged = scaling == AATC_ROPE_RAMP || scaling == AATC_ROPE_BANDED;
  if (!freq_out || !factor_out || rot_dim < 16 || rot_dim > D || rot_dim % 16 != 0 || !std::isfinite(base) ||
      !(base > 1.0) || scaling < AATC_ROPE_PLAIN || scaling > AATC_ROPE_BANDED)
    return AATC_ERR_INVALID_ARG;
  if (!plain && (!std::isfinite(scale) || scale < 1.0)) return AATC_ERR_INVALID_ARG;
  if (ranged && (original < 1 || !std::isfinite(p0) || !std::isfinite(p1))) return AATC_ERR_INVALID_ARG;
  if (scaling == AATC_ROPE_RAMP && (p0 < p1 || p1 <= 0.0)) return AATC_ERR_INVALID_ARG;
  if (scaling == AATC_ROPE_BANDED && p1 <= p0) return AATC_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925286766559;
  if (scaling == AATC_ROPE_NTK) base *= std::pow(scale, rot_dim / (rot_dim - 2.0));
  double lo = 0.0, hi = 0.0;
  if (scaling == AATC_ROPE_RAMP) {
    const double per = rot_dim / (2.0 * std::log(base));
    lo = std::max(0.0, std::floor(per * std::log(original / (two_pi * p0))));
    hi = std::min(rot_dim - 1.0, std::ceil(per * std::log(original / (two_pi * p1))));
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double w = std::pow(base, -2.0 * i / rot_dim);
    double f = w;
    if (scaling == AATC_ROPE_LINEAR) f = w / scale;
    if (scaling == AATC_ROPE_RAMP) {
      const double t = std::min(1.0, std::max(0.0, (i - lo) / std::max(hi - lo, 1e-3)));
      f = w * (t / scale + (1.0 - t));
    }
    if (scaling == AATC_ROPE_BANDED) {
      const double u = std::min(1.0, std::max(0.0, (original * w / two_pi - p0) / (p1 - p0)));
      f = w * (u + (1.0 - u) / scale);
    }
    freq_out[i] = f;
  }
  *factor_out = scaling == AATC_ROPE_RAMP ? 0.1 * std::log(scale) + 1.0 : 1.0;
  return AATC_OK;
}

aatc_status_t aatc_rotary_turns(const double* freq, int32_t n, uint64_t* turns_out) {
  if (!freq || !turns_out || n < 1 || n > D / 2) return AATC_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(freq[i])) return AATC_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925286766559;
  for (int i = 0; i < n; ++i) {
    double t = std::fabs(freq[i]) / two_pi;                    // (1 - t of a small t would round)
    t -= std::floor(t);                                        // in [0, 1)
    // the upper and the lower 32 bits apart: each fits a double's 53 without rounding
    const double high = std::floor(std::ldexp(t, 32));
    const double low = std::ldexp(std::ldexp(t, 32) - high, 32);
    const uint64_t turns = (static_cast<uint64_t>(high) << 32) + static_cast<uint64_t>(std::nearbyint(low));
    turns_out[i] = freq[i] < 0.0 ? 0 - turns : turns;
  }
  return AATC_OK;
}

aatc_status_t aatc_rotate(const aatc_rotary_t* rope, int32_t dtype, const void* x, int64_t x_token_stride,
                          int64_t x_head_stride, const int32_t* positions, int32_t n_tokens, int32_t n_heads,
                          int32_t backward, void* out, int64_t out_token_stride, int64_t out_head_stride,
                          void* stream) {
  if (n_tokens == 0) return AATC_OK;
  const aatc_heads_t in = {x, x_token_stride, x_head_stride}, res = {out, out_token_stride, out_head_stride};
  if (!rope_ok(rope) || (dtype != AATC_BF16 && dtype != AATC_F16) || !heads_ok(&in) || !heads_ok(&res) || !positions ||
      !aligned4(positions) || n_tokens < 0 || n_heads < 1 || n_heads > 65536 ||
      !apart(out_token_stride, out_head_stride, n_tokens, n_heads) ||
      (x == out && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)))
    return AATC_ERR_INVALID_ARG;
  paged::AppendArgs a = {};
  a.turn = turn(rope, backward != 0);
  a.index = positions;
  a.n_tokens = n_tokens;
  a.n_q = n_heads;
  a.q = heads(&in);
  a.q_out = out;
  a.q_out_token_stride = out_token_stride;
  a.q_out_head_stride = out_head_stride;
  return status_from_cuda(paged::launch_append(dtype, a, static_cast<cudaStream_t>(stream)));
}

aatc_status_t aatc_paged_append(const aatc_pages_t* desc, void* pages, const int32_t* table, int32_t n_rows,
                                int32_t table_stride, int32_t max_pages, const int32_t* rows, const int32_t* index,
                                const int32_t* positions, int32_t n_tokens, const aatc_heads_t* k,
                                const aatc_heads_t* v, const aatc_rotary_t* rope, const aatc_heads_t* q,
                                int32_t n_q_heads, void* q_out, int32_t* dev_flags, void* stream) {
  if (page_shift(desc) < 0) return AATC_ERR_INVALID_ARG;
  if (n_tokens == 0) return AATC_OK;
  if (!pages || !aligned16(pages) || !table_ok(table, n_rows, table_stride, max_pages) || !index || !aligned4(index) ||
      !aligned4(rows) || !aligned4(positions) || !aligned4(dev_flags) || n_tokens < 0 || !heads_ok(k) || !heads_ok(v) ||
      (rope && !rope_ok(rope)) || (q != nullptr) != (q_out != nullptr))
    return AATC_ERR_INVALID_ARG;
  if (q && (!rope || !heads_ok(q) || !aligned16(q_out) || n_q_heads < 1 || n_q_heads > 65536 ||
            (q_out == q->x && !apart(q->token_stride, q->head_stride, n_tokens, n_q_heads))))
    return AATC_ERR_INVALID_ARG;
  paged::AppendArgs a = {};
  a.pool = pool(desc, pages, table, table_stride, max_pages, dev_flags);
  if (rope) a.turn = turn(rope, false);
  a.rows = rows;
  a.index = index;
  a.positions = positions;
  a.n_rows = n_rows;
  a.n_tokens = n_tokens;
  a.k = heads(k);
  a.v = heads(v);
  if (q) {
    a.n_q = n_q_heads;
    a.q = heads(q);
    a.q_out = q_out;
    a.q_out_token_stride = q_out == q->x ? q->token_stride : static_cast<int64_t>(n_q_heads) * D;
    a.q_out_head_stride = q_out == q->x ? q->head_stride : D;
  }
  return status_from_cuda(paged::launch_append(desc->dtype, a, static_cast<cudaStream_t>(stream)));
}

aatc_status_t aatc_paged_decode_workspace_bytes(const aatc_pages_t* desc, int32_t n_q_heads, size_t* bytes) {
  if (!bytes || page_shift(desc) < 0 || n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % desc->n_kv_heads)
    return AATC_ERR_INVALID_ARG;
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return status_from_cuda(e);
  *bytes = paged::decode_workspace(sms);
  return AATC_OK;
}

aatc_status_t aatc_paged_decode_attention(const aatc_pages_t* desc, const void* pages, const int32_t* table,
                                          int32_t table_stride, int32_t max_pages, const int32_t* lens, int32_t batch,
                                          const aatc_heads_t* q, int32_t n_q_heads, const aatc_paged_decode_t* how,
                                          float* out, float* lse, void* workspace, size_t workspace_bytes,
                                          int32_t* dev_flags, void* stream) {
  if (page_shift(desc) < 0 || !pages || !aligned16(pages) || !table_ok(table, batch, table_stride, max_pages) || !lens ||
      !aligned4(lens) || batch > 65535 || !heads_ok(q) || n_q_heads < 1 || n_q_heads > 65536 ||
      n_q_heads % desc->n_kv_heads || !how || !std::isfinite(how->scale) || !std::isfinite(how->cap) ||
      how->cap < 0.0f || how->window < 0 || (how->prior_out != nullptr) != (how->prior_lse != nullptr) ||
      !aligned16(how->prior_out) || !aligned4(how->prior_lse) || !aligned4(how->slopes) || !out || !aligned16(out) ||
      !aligned4(lse) || !aligned16(workspace) || !aligned4(dev_flags) ||
      static_cast<int64_t>(max_pages) * desc->page_size > INT32_MAX)
    return AATC_ERR_INVALID_ARG;
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return status_from_cuda(e);
  const size_t need = paged::decode_workspace(sms);
  if (workspace_bytes < need || (need && !workspace)) return AATC_ERR_WORKSPACE;
  paged::DecodeArgs a = {};
  a.pool = pool(desc, const_cast<void*>(pages), table, table_stride, max_pages, dev_flags);
  a.lens = lens;
  a.batch = batch;
  a.n_q = n_q_heads;
  a.group = n_q_heads / desc->n_kv_heads;
  a.q = heads(q);
  a.scale = how->scale;
  a.cap = how->cap;
  a.window = how->window;
  a.slopes = how->slopes;
  a.prior_out = how->prior_out;
  a.prior_lse = how->prior_lse;
  a.out = out;
  a.lse = lse;
  a.ws = static_cast<float*>(workspace);
  a.num_sms = sms;
  return status_from_cuda(paged::launch_decode(desc->dtype, a, static_cast<cudaStream_t>(stream)));
}

aatc_status_t aatc_pages_copy(const aatc_pages_t* desc, void* pages, int32_t n_layers, size_t layer_stride,
                              const int32_t* pairs, int32_t n_pairs, void* stream) {
  if (page_shift(desc) < 0 || n_pairs < 0 || n_layers < 0 || n_layers > 65535) return AATC_ERR_INVALID_ARG;
  if (n_pairs == 0 || n_layers == 0) return AATC_OK;
  const size_t bytes = page_bytes(desc);
  if (!pages || !aligned16(pages) || !pairs || layer_stride % 16 != 0 ||
      (n_layers > 1 && layer_stride < bytes * desc->n_pages) || n_pairs > desc->n_pages)
    return AATC_ERR_INVALID_ARG;
  // one byte a page: read by the call, or written
  enum : unsigned char { kRead = 1, kWritten = 2 };
  unsigned char* use = new (std::nothrow) unsigned char[desc->n_pages];
  if (!use) return AATC_ERR_NOMEM;
  std::memset(use, 0, desc->n_pages);
  bool ok = true;
  for (int i = 0; ok && i < n_pairs; ++i) {
    const int32_t src = pairs[2 * i], dst = pairs[2 * i + 1];
    ok = src >= 0 && src < desc->n_pages && dst >= 0 && dst < desc->n_pages && !(use[dst] & kWritten);
    if (ok) {
      use[src] |= kRead;
      use[dst] |= kWritten;
    }
  }
  for (int i = 0; ok && i < n_pairs; ++i) ok = use[pairs[2 * i]] == kRead && use[pairs[2 * i + 1]] == kWritten;
  delete[] use;
  if (!ok) return AATC_ERR_INVALID_ARG;
  return status_from_cuda(paged::launch_copy(pages, bytes, n_layers, layer_stride, pairs, n_pairs,
                                             static_cast<cudaStream_t>(stream)));
}

aatc_status_t aatc_paged_gather(const aatc_pages_t* desc, const void* pages, const int32_t* table, int32_t n_rows,
                                int32_t table_stride, int32_t max_pages, int32_t first, int32_t n_tokens,
                                const int32_t* lens, void* k_out, void* v_out, int32_t* dev_flags, void* stream) {
  if (page_shift(desc) < 0 || n_rows < 0 || n_tokens < 0 || first < 0) return AATC_ERR_INVALID_ARG;
  if (n_rows == 0 || n_tokens == 0) return AATC_OK;
  if (!pages || !aligned16(pages) || !table_ok(table, n_rows, table_stride, max_pages) || !aligned4(lens) || !k_out ||
      !v_out || !aligned16(k_out) || !aligned16(v_out) || !aligned4(dev_flags))
    return AATC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(first) + n_tokens >
      std::min<int64_t>(static_cast<int64_t>(max_pages) * desc->page_size, INT32_MAX))
    return AATC_ERR_CAPACITY;
  paged::GatherArgs a = {};
  a.pool = pool(desc, const_cast<void*>(pages), table, table_stride, max_pages, dev_flags);
  a.n_rows = n_rows;
  a.first = first;
  a.n_tokens = n_tokens;
  a.lens = lens;
  a.k_out = k_out;
  a.v_out = v_out;
  return status_from_cuda(paged::launch_gather(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
