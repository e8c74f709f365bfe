// Kernels of the paged cache: rotary positions and append, decode attention, page copies, gather.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "aatc_internal.h"
#include "paged.h"
#include "ptx.cuh"

namespace aatc {
namespace paged {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float2 widen(__nv_bfloat16, uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 widen(__half, uint32_t w) {
  __half2 h;
  *reinterpret_cast<uint32_t*>(&h) = w;
  return __half22float2(h);
}
__device__ __forceinline__ uint32_t narrow(__nv_bfloat16, float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t narrow(__half, float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void raise(int32_t* err, int32_t bits) {
  if (err) atomicOr(err, bits);
}

// ---------------------------------------------------------------- rotary positions and append
// cos and sin of position x frequency, times the factor.  turns is the frequency as a 64-bit fraction of
// a turn, so the product modulo 2^64 is the angle's fraction exactly; its upper 32 bits are the angle
// in half turns within 2^-32.
__device__ __forceinline__ float2 cos_sin(const Turn& t, int32_t position, uint64_t turns) {
  const uint64_t ph = static_cast<uint64_t>(static_cast<int64_t>(position)) * turns;
  float s, c;
  sincospif(static_cast<float>(static_cast<int32_t>(ph >> 32)) * 4.656612873077393e-10f, &s, &c);   // 2^-31
  return make_float2(c * t.factor, s * t.factor * t.sign);
}

// A head is eight units of sixteen dimensions, two 16-byte pieces each: of the rotated part, pieces whose
// values pair up (half layout: rot_dim / 2 apart; interleaved: side by side), eight pairs with
// the frequencies 8 u .. 8 u + 7; of the rest, two neighbouring pieces.
constexpr int kUnits = 8;

template <typename T>
__device__ __forceinline__ void rotate_unit(const Turn& t, int u, int32_t position, const T* x, T* out) {
  const bool turned = 16 * u < t.rot_dim;
  const int a = turned && !t.interleaved ? 8 * u : 16 * u;
  const int b = turned && !t.interleaved ? 8 * u + t.rot_dim / 2 : 16 * u + 8;
  uint4 pa = *reinterpret_cast<const uint4*>(x + a), pb = *reinterpret_cast<const uint4*>(x + b);
  if (turned) {
    uint32_t* wa = reinterpret_cast<uint32_t*>(&pa);
    uint32_t* wb = reinterpret_cast<uint32_t*>(&pb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 e0 = cos_sin(t, position, t.turns[8 * u + (t.interleaved ? i : 2 * i)]);
      const float2 e1 = cos_sin(t, position, t.turns[8 * u + (t.interleaved ? i + 4 : 2 * i + 1)]);
      const float2 va = widen(T(), wa[i]), vb = widen(T(), wb[i]);
      if (t.interleaved) {
        wa[i] = narrow(T(), va.x * e0.x - va.y * e0.y, va.x * e0.y + va.y * e0.x);
        wb[i] = narrow(T(), vb.x * e1.x - vb.y * e1.y, vb.x * e1.y + vb.y * e1.x);
      } else {
        wa[i] = narrow(T(), va.x * e0.x - vb.x * e0.y, va.y * e1.x - vb.y * e1.y);
        wb[i] = narrow(T(), va.x * e0.y + vb.x * e0.x, va.y * e1.y + vb.y * e1.x);
      }
    }
  }
  *reinterpret_cast<uint4*>(out + a) = pa;
  *reinterpret_cast<uint4*>(out + b) = pb;
}

// One CTA per token.
template <typename T>
__global__ void __launch_bounds__(256) aatc_paged_append_kernel(const AppendArgs a) {
  const int64_t t = blockIdx.x;
  const int32_t index = a.index[t];
  const int32_t position = a.positions ? a.positions[t] : index;
  const T* q = static_cast<const T*>(a.q.x) + t * a.q.token_stride;
  T* qo = static_cast<T*>(a.q_out) + t * a.q_out_token_stride;
  for (int i = threadIdx.x; i < a.n_q * kUnits; i += blockDim.x)
    rotate_unit(a.turn, i % kUnits, position, q + (i / kUnits) * a.q.head_stride,
                qo + (i / kUnits) * a.q_out_head_stride);
  const Pool& p = a.pool;
  if (!p.pages || index < 0) return;
  const int64_t row = a.rows ? a.rows[t] : t;
  if (row < 0 || row >= a.n_rows || (index >> p.page_shift) >= p.max_pages) {
    raise(p.err, kBadRow);
    return;
  }
  const int32_t id = p.table[row * p.table_stride + (index >> p.page_shift)];
  if (id < 0 || id >= p.n_pages) {
    raise(p.err, kBadPage);
    return;
  }
  // keys of all heads of a page, then values: head h of kind c at block (2 id + c) n_kv + h
  T* page = static_cast<T*>(p.pages) + ((static_cast<int64_t>(id) * 2 * p.n_kv << p.page_shift) +
                                        (index & ((1 << p.page_shift) - 1))) * D;
  const T* k = static_cast<const T*>(a.k.x) + t * a.k.token_stride;
  const T* v = static_cast<const T*>(a.v.x) + t * a.v.token_stride;
  Turn none = a.turn;
  none.rot_dim = 0;
  for (int i = threadIdx.x; i < 2 * p.n_kv * kUnits; i += blockDim.x) {
    const int h = i / kUnits;
    T* to = page + (static_cast<int64_t>(h) << p.page_shift) * D;
    if (h < p.n_kv) rotate_unit(a.turn.turns ? a.turn : none, i % kUnits, position, k + h * a.k.head_stride, to);
    else rotate_unit(none, i % kUnits, position, v + (h - p.n_kv) * a.v.head_stride, to);
  }
}

// ---------------------------------------------------------------- decode attention
constexpr int kHeadsPerCta = 8;     // query heads of one kv-head that a CTA takes
constexpr int kDecodeThreads = 256;

// One CTA per (sequence, kv-head, eight of its query heads): a warp takes every eighth token, a lane four of
// its dimensions, with an online softmax per warp; the warps are joined in shared memory.
template <typename T>
__global__ void __launch_bounds__(kDecodeThreads) aatc_paged_decode_kernel(const DecodeArgs a) {
  constexpr int kW = kDecodeThreads / 32, G = kHeadsPerCta;
  __shared__ float so[kW][G][D];
  __shared__ float sm[kW][G], sl[kW][G];
  const Pool& p = a.pool;
  const int blocks = (a.group + G - 1) / G;
  const int h = blockIdx.x / blocks, g0 = (blockIdx.x % blocks) * G, n_g = min(G, a.group - g0);
  const int b = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int n = a.lens[b];
  if (n < 0 || n > p.max_pages << p.page_shift) {
    if (threadIdx.x == 0) raise(p.err, kBadRow);
    n = min(max(n, 0), p.max_pages << p.page_shift);
  }
  const int lo = a.window > 0 ? max(0, n - a.window) : 0;
  float q[G][4], o[G][4], m[G], l[G];
  const int j0 = h * a.group + g0;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.0f;
    uint2 w = make_uint2(0, 0);
    if (g < n_g)
      w = *reinterpret_cast<const uint2*>(static_cast<const T*>(a.q.x) + b * a.q.token_stride + (j0 + g) * a.q.head_stride +
                                          4 * lane);
    const float2 x = widen(T(), w.x), y = widen(T(), w.y);
    q[g][0] = x.x; q[g][1] = x.y; q[g][2] = y.x; q[g][3] = y.y;
    o[g][0] = o[g][1] = o[g][2] = o[g][3] = 0.0f;
  }
  for (int t = lo + warp; t < n; t += kW) {
    const int32_t id = p.table[static_cast<int64_t>(b) * p.table_stride + (t >> p.page_shift)];
    if (id < 0 || id >= p.n_pages) {
      if (lane == 0) raise(p.err, kBadPage);
      continue;
    }
    const T* k = static_cast<const T*>(p.pages) + (((static_cast<int64_t>(id) * 2 * p.n_kv + h) << p.page_shift) +
                                                   (t & ((1 << p.page_shift) - 1))) * D + 4 * lane;
    const T* v = k + (static_cast<int64_t>(p.n_kv) << p.page_shift) * D;
    const uint2 kw = *reinterpret_cast<const uint2*>(k), vw = *reinterpret_cast<const uint2*>(v);
    const float2 k0 = widen(T(), kw.x), k1 = widen(T(), kw.y), v0 = widen(T(), vw.x), v1 = widen(T(), vw.y);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (g >= n_g) break;
      float s = q[g][0] * k0.x + q[g][1] * k0.y + q[g][2] * k1.x + q[g][3] * k1.y;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      s *= a.scale;
      if (a.cap > 0.0f) s = a.cap * tanhf(s / a.cap);
      if (a.slopes) s += a.slopes[j0 + g] * static_cast<float>(t - (n - 1));
      const float mn = fmaxf(m[g], s), base = mn == -INFINITY ? 0.0f : mn;
      const float r = exp2f((m[g] - base) * kLog2e), e = exp2f((s - base) * kLog2e);
      m[g] = mn;
      l[g] = l[g] * r + e;
      o[g][0] = o[g][0] * r + e * v0.x;
      o[g][1] = o[g][1] * r + e * v0.y;
      o[g][2] = o[g][2] * r + e * v1.x;
      o[g][3] = o[g][3] * r + e * v1.y;
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    *reinterpret_cast<float4*>(&so[warp][g][4 * lane]) = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
    if (lane == 0) {
      sm[warp][g] = m[g];
      sl[warp][g] = l[g];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_g * D; i += kDecodeThreads) {
    const int g = i / D, d = i % D;
    const int64_t row = static_cast<int64_t>(b) * a.n_q + j0 + g;
    float top = a.prior_lse ? a.prior_lse[row] : -INFINITY;
    for (int w = 0; w < kW; ++w) top = fmaxf(top, sm[w][g]);
    const float base = top == -INFINITY ? 0.0f : top;
    float total = 0.0f, acc = 0.0f;
    if (a.prior_lse) {
      total = exp2f((a.prior_lse[row] - base) * kLog2e);
      if (total > 0.0f) acc = total * a.prior_out[row * D + d];
    }
    for (int w = 0; w < kW; ++w) {
      const float f = exp2f((sm[w][g] - base) * kLog2e);
      total += f * sl[w][g];
      acc += f * so[w][g][d];
    }
    a.out[row * D + d] = total == 0.0f ? 0.0f : acc / total;
    if (a.lse) so[0][g][d] = base + logf(total);
  }
  __syncthreads();
  if (a.lse && threadIdx.x < n_g) a.lse[static_cast<int64_t>(b) * a.n_q + j0 + threadIdx.x] = so[0][threadIdx.x][0];
}

// ---------------------------------------------------------------- page copies
template <int N>
__global__ void __launch_bounds__(256) aatc_pages_copy_kernel(uint4* pages, int64_t page_vecs, int64_t layer_vecs,
                                                              const __grid_constant__ CopyPairs<N> pairs) {
  const int2 pr = pairs.pair[blockIdx.x];
  const uint4* src = pages + blockIdx.y * layer_vecs + pr.x * page_vecs;
  uint4* dst = pages + blockIdx.y * layer_vecs + pr.y * page_vecs;
  for (int64_t i = threadIdx.x; i < page_vecs; i += blockDim.x) dst[i] = src[i];
}

// ---------------------------------------------------------------- gather
// One CTA per token: the keys of all kv-heads, then the values.
__global__ void __launch_bounds__(256) aatc_paged_gather_kernel(const GatherArgs a) {
  const Pool& p = a.pool;
  const int r = blockIdx.y, t = a.first + blockIdx.x;
  bool seen = !a.lens || t < a.lens[r];
  int32_t id = 0;
  if (seen) {
    id = p.table[static_cast<int64_t>(r) * p.table_stride + (t >> p.page_shift)];
    if (id < 0 || id >= p.n_pages) {
      if (threadIdx.x == 0) raise(p.err, kBadPage);
      seen = false;
    }
  }
  constexpr int kVecs = D / 8;                                 // 16-byte pieces of a head
  const uint4* page = static_cast<const uint4*>(p.pages) +
                      ((static_cast<int64_t>(id) * 2 * p.n_kv << p.page_shift) + (t & ((1 << p.page_shift) - 1))) * kVecs;
  const int64_t to = (static_cast<int64_t>(r) * a.n_tokens + blockIdx.x) * p.n_kv;
  for (int i = threadIdx.x; i < 2 * p.n_kv * kVecs; i += blockDim.x) {
    const int h = i / kVecs, c = i % kVecs;
    const uint4 x = seen ? page[(static_cast<int64_t>(h) << p.page_shift) * kVecs + c] : make_uint4(0, 0, 0, 0);
    uint4* out = static_cast<uint4*>(h < p.n_kv ? a.k_out : a.v_out);
    out[(to + (h < p.n_kv ? h : h - p.n_kv)) * kVecs + c] = x;
  }
}

}  // namespace

cudaError_t launch_append(int dtype, const AppendArgs& a, cudaStream_t st) {
  if (dtype == AATC_BF16) aatc_paged_append_kernel<__nv_bfloat16><<<a.n_tokens, 256, 0, st>>>(a);
  else aatc_paged_append_kernel<__half><<<a.n_tokens, 256, 0, st>>>(a);
  return cudaGetLastError();
}

size_t decode_workspace(int, int, int) { return 0; }

cudaError_t launch_decode(int dtype, const DecodeArgs& a, cudaStream_t st) {
  const dim3 grid(a.pool.n_kv * ((a.group + kHeadsPerCta - 1) / kHeadsPerCta), a.batch);
  if (dtype == AATC_BF16) aatc_paged_decode_kernel<__nv_bfloat16><<<grid, kDecodeThreads, 0, st>>>(a);
  else aatc_paged_decode_kernel<__half><<<grid, kDecodeThreads, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_copy(void* pages, size_t page_bytes, int n_layers, size_t layer_stride, const int32_t* pairs,
                        int n_pairs, cudaStream_t st) {
  constexpr int kMost = 500;                                   // pairs of a launch: 4000 bytes of parameters
  for (int i0 = 0; i0 < n_pairs; i0 += kMost) {
    CopyPairs<kMost> cp;
    const int n = std::min(kMost, n_pairs - i0);
    for (int i = 0; i < n; ++i) cp.pair[i] = make_int2(pairs[2 * (i0 + i)], pairs[2 * (i0 + i) + 1]);
    aatc_pages_copy_kernel<kMost><<<dim3(n, n_layers), 256, 0, st>>>(static_cast<uint4*>(pages), page_bytes / 16,
                                                                     layer_stride / 16, cp);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_gather(const GatherArgs& a, cudaStream_t st) {
  for (int r0 = 0; r0 < a.n_rows; r0 += 65535) {               // (a grid's y extent)
    GatherArgs s = a;
    s.n_rows = std::min(65535, a.n_rows - r0);
    s.pool.table += static_cast<int64_t>(r0) * a.pool.table_stride;
    if (a.lens) s.lens += r0;
    const size_t skip = static_cast<size_t>(r0) * a.n_tokens * a.pool.n_kv * D * 2;
    s.k_out = static_cast<char*>(a.k_out) + skip;
    s.v_out = static_cast<char*>(a.v_out) + skip;
    aatc_paged_gather_kernel<<<dim3(a.n_tokens, s.n_rows), 256, 0, st>>>(s);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace paged
}  // namespace aatc
