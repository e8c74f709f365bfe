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
// The work of a call is its units of 16 tokens: those of sequence 0's kv-head 0, then kv-head 1, ...,
// then sequence 1's, a (sequence, kv-head) being a segment.  CTA c of n takes the units
// [c U / n, (c + 1) U / n) of all U and each of its warps a quarter of those, so every warp has the same
// share whatever the lengths.  A segment that lies inside a warp's share is finished by the warp, the pieces of one
// that lies in several warps are joined in shared memory, and those of one in several CTAs
// through the workspace by the second launch.  (Query heads beyond eight of a kv-head are further segments over
// the same tokens.)  A warp's loads run ahead of its sums across the segments of its share: with
// shares by CTA and a barrier per segment, 61 sequences of 62 to 4001 tokens took twice as long as as many tokens
// in equal sequences.
constexpr int kSegHeads = 8;        // query heads of a segment: the columns of the MMAs
constexpr int kUnit = 16;           // tokens
constexpr int kDecodeWarps = 8;
constexpr int kDecodeCtas = 1;      // per SM
constexpr int kUnitsPerCta = 8;     // fewer CTAs where they would get less
constexpr int kStages = 3;          // units of a warp on their way: keys and values, 8 KB each
constexpr int kHalf = 8 * D * 2;    // bytes of eight tokens' keys (or values) of one head
constexpr int kStage = 4 * kHalf;   // keys of the unit's two halves, then values
constexpr int kPiece = kSegHeads * (D + 2);   // floats of a piece: sums [8][128], maxima [8], totals [8]

// Workspace: pieces [2 n_ctas] (CTA c's share begins inside a segment: piece 2 c; ends inside one that it began:
// 2 c + 1), then int4 per CTA: the segment that it began and did not end (sequence, segment of the
// sequence, last CTA with a piece of it; sequence -1: none).
struct Share {
  int64_t total;                    // units
  int n_ctas;                       // CTAs that get any
};

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of an 8 x 8 matrix of 16-bit values over the warp
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_of(float x) {            // (-inf: 0)
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint4 lds_16(uint32_t p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(p));
  return v;
}

// A weight p as a sum of 16-bit values, so that products with 16-bit values on the tensor cores lose
// nothing of it: bf16, three truncations of eight significant bits (all of p's 24); f16, a truncation and the
// rounded rest (22 bits; p <= 2^14 and its scale keep the rest above the format's smallest step for
// any p over 2^-30 of the largest).  No part is negative, and no bf16 part zero, as an infinite value
// times it would turn into NaN.
template <typename T>
struct Parts;
template <>
struct Parts<__nv_bfloat16> {
  static constexpr int kN = 3;
  static constexpr float kShift = 0.0f;                        // log2 of the scale on p
  static __device__ __forceinline__ void split(float p, float q, uint32_t (&out)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint32_t a = __float_as_uint(p), b = __float_as_uint(q);
      out[i] = __byte_perm(a, b, 0x7632);
      p = fmaxf(p - __uint_as_float(a & 0xFFFF0000u), 7.8886e-31f);   // about 2^-100
      q = fmaxf(q - __uint_as_float(b & 0xFFFF0000u), 7.8886e-31f);
    }
  }
};
template <>
struct Parts<__half> {
  static constexpr int kN = 2;
  static constexpr float kShift = 6.0f;
  static __device__ __forceinline__ void split(float p, float q, uint32_t (&out)[2]) {
    const __half2 h = __halves2half2(__float2half_rz(p), __float2half_rz(q));
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(p - f.x, q - f.y);
    out[0] = *reinterpret_cast<const uint32_t*>(&h);
    out[1] = *reinterpret_cast<const uint32_t*>(&l);
  }
};

// First token and unit count of a sequence: the tokens [lo, n) in units from lo / 16 on; one unit, of nothing,
// for an empty one (somebody has to write its result).
struct Extent {
  int n, lo, units;
};
__device__ __forceinline__ Extent extent_of(const DecodeArgs& a, int len) {
  Extent e;
  e.n = min(max(len, 0), a.pool.max_pages << a.pool.page_shift);
  e.lo = a.window > 0 ? max(0, e.n - a.window) : 0;
  e.units = max(1, (e.n + kUnit - 1) / kUnit - e.lo / kUnit);
  return e;
}

// Unit u of all is in the share of CTA ((u + 1) n - 1) / U.
__device__ __forceinline__ int cta_of(const Share& s, int64_t unit) {
  return static_cast<int>(((unit + 1) * s.n_ctas - 1) / s.total);
}

// K and V fragments of a unit.  Lane (g, t) = (lane / 4, lane % 4) needs of K the token of row g of each half
// (A operand of the score MMAs: rows are tokens; the order of the dimensions is free as long as the query's
// is the same) and of V the tokens of rows 2 t and 2 t + 1 of each half, dimensions 8 g .. + 7 and 64 + 8 g .. + 7
// (A operand of the output MMAs after pairs of tokens are interleaved: rows are dimensions).  A token
// is two rows of 128 bytes in shared memory, whose 16-byte pieces the copy has permuted by the row's
// number modulo 8 (2 (token % 4) + the row's half).  Row r of a half is token r / 2 for even r and 4 + (r / 2 ^ 1)
// for odd r: with it the eight lanes of every quarter of a 128-bit load of keys or values touch eight
// different pieces.
__device__ __forceinline__ int token_of_row(int r) { return r % 2 ? 4 + (r / 2 ^ 1) : r / 2; }
// Piece of row half j / 2 that lane t takes in step j of the keys: {0, 1, 4, 5} and those + 2.
__device__ __forceinline__ int piece_of(int t, int j) { return (t & 1) | (t & 2) << 1 | (j & 1) << 1; }

// A warp's piece of a segment that it does not have whole, in shared memory.
struct Piece {
  float sum[kSegHeads][D];
  float top[kSegHeads], total[kSegHeads];
};
struct PieceOf {
  int b, seg;                       // b < 0: none
  int ends;
  int64_t last_unit;                // of the segment, among all units
};

// Shared memory: every warp's ring of stages, which its piece of the segment that it began takes over at the end
// of its share, then the pieces of the segments that it found begun.
constexpr size_t kDecodeSmem = 1024 + static_cast<size_t>(kDecodeWarps) * (kStages * kStage + sizeof(Piece));
static_assert(sizeof(Piece) <= kStages * kStage && sizeof(Piece) % 16 == 0, "a piece in the place of a ring");

template <typename T>
__global__ void __launch_bounds__(kDecodeWarps * 32, kDecodeCtas)
    aatc_paged_decode_kernel(const DecodeArgs a, const __grid_constant__ CUtensorMap map) {
  constexpr int kW = kDecodeWarps, kT = kW * 32;
  constexpr float kUnshift = 1.0f / (1 << static_cast<int>(Parts<T>::kShift));
  extern __shared__ unsigned char dyn_smem[];
  __shared__ PieceOf s_of[kW][2];
  __shared__ int64_t s_part[kW], s_before[kW];
  __shared__ int s_seq[kW], s_len[kW];
  __shared__ uint64_t s_full[kW][kStages];
  __shared__ int s_abort;
  const Pool& p = a.pool;
  const int tid = threadIdx.x, warp = ptx::warp_uniform(tid / 32), lane = tid % 32, g = lane / 4, t4 = lane % 4;
  const int seg_blocks = (a.group + kSegHeads - 1) / kSegHeads, n_seg = p.n_kv * seg_blocks;
  int4* desc = reinterpret_cast<int4*>(a.ws + static_cast<size_t>(gridDim.x) * 2 * kPiece);
  unsigned char* rings = dyn_smem + (1024 - ptx::smem_u32(dyn_smem) % 1024) % 1024;
  unsigned char* ring = rings + warp * (kStages * kStage);
  auto piece_at = [&](int w, int begins) {
    return reinterpret_cast<Piece*>(begins ? rings + w * (kStages * kStage) : rings + kW * (kStages * kStage) + w * sizeof(Piece));
  };
  if (tid < kW * kStages) ptx::mbar_init(&s_full[0][0] + tid, 1);
  if (tid == 0) {
    s_abort = 0;
    ptx::prefetch_tmap(&map);
  }
  ptx::fence_mbar_init();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  // ---- the total, and the sequences in which the warps' shares begin: prefix sums over kT sequences at a time
  int len = 0;
  int64_t units = 0, upto = 0;                       // of sequence i0 + tid; up to it within the chunk
  auto scan = [&](int i0) {
    const int i = i0 + tid;
    len = i < a.batch ? __ldg(a.lens + i) : 0;
    units = i < a.batch ? static_cast<int64_t>(extent_of(a, len).units) * n_seg : 0;
    upto = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    __syncthreads();                                 // (the last chunk's sums have been read)
    if (lane == 31) s_part[warp] = upto;
    __syncthreads();
    int64_t sum = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      if (w == warp) upto += sum;
      sum += s_part[w];
    }
    return sum;
  };
  Share share;
  share.total = 0;
  for (int i0 = 0; i0 < a.batch; i0 += kT) {
    share.total += scan(i0);
    if (blockIdx.x == 0 && i0 + tid < a.batch && (len < 0 || len > p.max_pages << p.page_shift)) raise(p.err, kBadRow);
  }
  share.n_ctas = static_cast<int>(min(static_cast<int64_t>(gridDim.x), (share.total + kUnitsPerCta - 1) / kUnitsPerCta));
  if (tid == 0) desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
  if (blockIdx.x >= share.n_ctas) return;
  const int64_t first = blockIdx.x * share.total / share.n_ctas;
  const int64_t here = (blockIdx.x + 1) * share.total / share.n_ctas - first;
  {
    const int64_t begin_last = first + here * (kW - 1) / kW;
    int64_t before = 0;
    for (int i0 = 0; i0 < a.batch; i0 += kT) {
      const int64_t sum = a.batch > kT ? scan(i0) : share.total;
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const int64_t x = first + here * w / kW - before;
        if (upto - units <= x && x < upto) {
          s_seq[w] = i0 + tid;
          s_len[w] = len;
          s_before[w] = before + upto - units;
        }
      }
      before += sum;
      if (before > begin_last) break;
    }
    if (tid < 2 * kW) s_of[tid / 2][tid % 2].b = -1;
    __syncthreads();
  }
  int64_t x = first + here * warp / kW;              // the unit that is summed, among all
  const int64_t x_end = first + here * (warp + 1) / kW;

  // ---- the units ahead: a walk whose next unit has its page ids on the way, and behind it the units whose keys and
  // values are (lane 0 issues the copies)
  struct Walk {
    int b, seg, u;
    Extent ext;
    int len_next;
  };
  auto step = [&](Walk& w) {
    if (++w.u < w.ext.units) return;
    w.u = 0;
    if (++w.seg < n_seg) return;
    w.seg = 0;
    ++w.b;
    w.ext = extent_of(a, w.len_next);
    w.len_next = w.b + 1 < a.batch ? __ldg(a.lens + w.b + 1) : 0;
  };
  Walk cur;                                          // the unit that is summed
  cur.b = s_seq[warp];
  cur.ext = extent_of(a, s_len[warp]);
  cur.seg = static_cast<int>((x - s_before[warp]) / cur.ext.units);
  cur.u = static_cast<int>((x - s_before[warp]) % cur.ext.units);
  cur.len_next = cur.b + 1 < a.batch ? __ldg(a.lens + cur.b + 1) : 0;
  Walk ahead = cur;                                  // the unit whose page ids are in `id`
  int64_t x_ahead = x;
  int id[2] = {-1, -1};
  uint32_t good = 0;                                 // two bits a stage: the half's page is in the pool
  auto first_token = [&](const Walk& w) { return (w.ext.lo / kUnit + w.u) * kUnit; };
  auto fetch_ids = [&]() {
    const int t = first_token(ahead);
    if (x_ahead >= x_end || t >= ahead.ext.n) return;
    const int32_t* row = p.table + static_cast<int64_t>(ahead.b) * p.table_stride;
    id[0] = __ldg(row + (t >> p.page_shift));
    id[1] = p.page_shift > 3 ? id[0] : t + 8 < ahead.ext.n ? __ldg(row + ((t + 8) >> p.page_shift)) : -1;
  };
  auto issue = [&](int stage) {                      // copies of the unit `ahead`, and the step to the next
    if (x_ahead >= x_end) return;
    const int t = first_token(ahead), in_page = t & ((1 << p.page_shift) - 1);
    uint32_t ok = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bool live = t + 8 * e < ahead.ext.n && t + 8 * e + 8 > ahead.ext.lo;
      if (live && static_cast<uint32_t>(id[e]) < static_cast<uint32_t>(p.n_pages)) ok |= 1u << e;
      else if (live && lane == 0) raise(p.err, kBadPage);
    }
    good = (good & ~(3u << 2 * stage)) | ok << 2 * stage;
    if (lane == 0) {
      unsigned char* to = ring + stage * kStage;
      uint64_t* bar = &s_full[warp][stage];
      const int row = 2 * (((ahead.seg / seg_blocks) << p.page_shift) + in_page), v_row = 2 * (p.n_kv << p.page_shift);
      if (p.page_shift > 3) {                        // a unit lies in one page: boxes of sixteen tokens
        ptx::mbar_arrive_expect_tx(bar, ok ? kStage : 0);
        if (ok) {
          ptx::tma_load_3d(to, &map, bar, 0, row, id[0]);
          ptx::tma_load_3d(to + 2 * kHalf, &map, bar, 0, row + v_row, id[0]);
        }
      } else {
        ptx::mbar_arrive_expect_tx(bar, __popc(ok) * 2 * kHalf);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (ok >> e & 1) {
            ptx::tma_load_3d(to + e * kHalf, &map, bar, 0, row, id[e]);
            ptx::tma_load_3d(to + (2 + e) * kHalf, &map, bar, 0, row + v_row, id[e]);
          }
      }
    }
    if (++x_ahead < x_end) step(ahead);
    fetch_ids();
  };
  uint32_t qf[4][4];                                 // B operand of the score MMAs: column g
  float slope0 = 0.0f, slope1 = 0.0f;
  auto load_q = [&](const Walk& n) {
    const int h = n.seg / seg_blocks, head0 = h * a.group + (n.seg % seg_blocks) * kSegHeads;
    const int n_g = min(kSegHeads, (h + 1) * a.group - head0);
    const T* q = static_cast<const T*>(a.q.x) + n.b * a.q.token_stride + (head0 + g) * a.q.head_stride;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 w = g < n_g ? *reinterpret_cast<const uint4*>(q + 64 * (j / 2) + 8 * piece_of(t4, j)) : make_uint4(0, 0, 0, 0);
      qf[j][0] = w.x; qf[j][1] = w.y; qf[j][2] = w.z; qf[j][3] = w.w;
    }
    if (a.slopes) {
      slope0 = 2 * t4 < n_g ? a.slopes[head0 + 2 * t4] * kLog2e : 0.0f;
      slope1 = 2 * t4 + 1 < n_g ? a.slopes[head0 + 2 * t4 + 1] * kLog2e : 0.0f;
    }
  };

  float acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;
  const int64_t x_begin = x;
  // this lane's pieces: keys of row g, step j (one address for j and j ^ 2 apart); values of rows 2 t4, 2 t4 + 1
  uint32_t k_off[4], v_off[2][2];
  {
    const int tok = token_of_row(g);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      k_off[j] = (2 * tok + j / 2) * 128 + ((piece_of(t4, j) ^ (2 * (tok & 3) + j / 2)) * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int tk = token_of_row(2 * t4 + i);
        v_off[i][d] = 2 * kHalf + (2 * tk + d) * 128 + ((g ^ (2 * (tk & 3) + d)) * 16);
      }
  }
  bool dead = false;
  if (x < x_end) {
    fetch_ids();
    load_q(cur);
#pragma unroll
    for (int i = 0; i < kStages; ++i) issue(i);
    int stage = 0;
    uint32_t phase = 0;
    for (; x < x_end; ++x) {
      if (!ptx::mbar_wait_bounded(&s_full[warp][stage], phase, &s_abort)) {
        dead = true;
        break;
      }
      const uint32_t at = ptx::smem_u32(ring) + stage * kStage;
      float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 k0 = lds_16(at + k_off[j]), k1 = lds_16(at + kHalf + k_off[j]);
        mma<T>(s, k0.x, k1.x, k0.y, k1.y, qf[j][0], qf[j][1]);
        mma<T>(s, k0.z, k1.z, k0.w, k1.w, qf[j][2], qf[j][3]);
      }
      uint4 v[2][2][2];                              // [token half][token][dimension half]
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int d = 0; d < 2; ++d) v[e][i][d] = lds_16(at + e * kHalf + v_off[i][d]);
      const int t_unit = first_token(cur);
      const uint32_t ok = good >> 2 * stage;
      const bool edge = t_unit < cur.ext.lo || t_unit + kUnit > cur.ext.n || (ok & 3u) != 3u;
      __syncwarp();                                  // every lane has read the stage
      issue(stage);
      // ---- scores in units of ln 2: s[0], s[1] row g, s[2], s[3] row 8 + g; queries 2 t4, 2 t4 + 1
      if (a.cap > 0.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = a.cap * kLog2e * tanhf(s[i] * a.scale / a.cap);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] *= a.scale * kLog2e;
      }
      const int tok = t_unit + token_of_row(g);
      if (a.slopes) {
        const float back0 = static_cast<float>(tok - (cur.ext.n - 1)), back1 = static_cast<float>(tok + 8 - (cur.ext.n - 1));
        s[0] = fmaf(slope0, back0, s[0]);
        s[1] = fmaf(slope1, back0, s[1]);
        s[2] = fmaf(slope0, back1, s[2]);
        s[3] = fmaf(slope1, back1, s[3]);
      }
      if (edge) {
        if (!(ok & 1u) || tok < cur.ext.lo || tok >= cur.ext.n) s[0] = s[1] = -INFINITY;
        if (!(ok & 2u) || tok + 8 < cur.ext.lo || tok + 8 >= cur.ext.n) s[2] = s[3] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 2; ++i) {              // a masked token's weight is 0, but 0 x NaN is not
            const int t = t_unit + 8 * e + token_of_row(2 * t4 + i);
            if (!(ok >> e & 1u) || t < cur.ext.lo || t >= cur.ext.n) v[e][i][0] = v[e][i][1] = make_uint4(0, 0, 0, 0);
          }
      }
      // ---- the running reference of the exponents follows the maximum only when that is 2^8 past it
      const float top0 = fmaxf(s[0], s[2]), top1 = fmaxf(s[1], s[3]);
      if (__any_sync(0xffffffffu, top0 > m0 + 8.0f || top1 > m1 + 8.0f)) {
        float n0 = fmaxf(m0, top0), n1 = fmaxf(m1, top1);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, o));
          n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
        }
        const float r0 = n0 == -INFINITY ? 1.0f : exp2_of(m0 - n0), r1 = n1 == -INFINITY ? 1.0f : exp2_of(m1 - n1);
        m0 = n0;
        m1 = n1;
        l0 *= r0;
        l1 *= r1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[i][0] *= r0;
          acc[i][1] *= r1;
          acc[i][2] *= r0;
          acc[i][3] *= r1;
        }
      }
      const float base0 = m0 == -INFINITY ? 0.0f : m0 - Parts<T>::kShift;
      const float base1 = m1 == -INFINITY ? 0.0f : m1 - Parts<T>::kShift;
      s[0] = exp2_of(s[0] - base0);
      s[1] = exp2_of(s[1] - base1);
      s[2] = exp2_of(s[2] - base0);
      s[3] = exp2_of(s[3] - base1);
      l0 += s[0] + s[2];
      l1 += s[1] + s[3];
      uint32_t w[2][Parts<T>::kN];
      Parts<T>::split(s[0], s[1], w[0]);
      Parts<T>::split(s[2], s[3], w[1]);
#pragma unroll
      for (int i = 0; i < Parts<T>::kN; ++i) {
        w[0][i] = transposed(w[0][i]);
        w[1][i] = transposed(w[1][i]);
      }
      // ---- rows 8 g + i and 64 + 8 g + i of V^T
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t f[4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            const uint32_t y0 = reinterpret_cast<const uint32_t*>(&v[e][0][d])[i / 2];
            const uint32_t y1 = reinterpret_cast<const uint32_t*>(&v[e][1][d])[i / 2];
            f[2 * e + d] = __byte_perm(y0, y1, i % 2 ? 0x7632 : 0x5410);
          }
#pragma unroll
        for (int y = 0; y < Parts<T>::kN; ++y) mma<T>(acc[i], f[0], f[1], f[2], f[3], w[0][y], w[1][y]);
      }

      const bool ends = cur.u == cur.ext.units - 1;
      if (ends || x + 1 == x_end) {                  // the segment's or the share's last unit
        Walk next = cur;
        step(next);
        if (x + 1 < x_end) load_q(next);
        const bool begins = x - cur.u >= x_begin;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          l0 += __shfl_xor_sync(0xffffffffu, l0, o);
          l1 += __shfl_xor_sync(0xffffffffu, l1, o);
        }
        l0 *= kUnshift;
        l1 *= kUnshift;
        const int h = cur.seg / seg_blocks, head0 = h * a.group + (cur.seg % seg_blocks) * kSegHeads;
        const int n_g = min(kSegHeads, (h + 1) * a.group - head0);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int q = 2 * t4 + c;
          const int64_t out_row = static_cast<int64_t>(cur.b) * a.n_q + head0 + q;
          const float m = c ? m1 : m0, l = c ? l1 : l0;
          float f = kUnshift, fp = 0.0f, base = 0.0f, total = l;
          if (begins && ends) {
            const float prior = a.prior_lse && q < n_g ? a.prior_lse[out_row] * kLog2e : -INFINITY;
            base = fmaxf(m, prior);
            if (base == -INFINITY) base = 0.0f;
            const float fm = exp2_of(m - base);
            fp = exp2_of(prior - base);
            total = fmaf(l, fm, fp);
            f *= fm;
          }
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
          __syncwarp();                              // (the log-sum may be written over the prior's)
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = acc[i][2 * d + c] * f;
            if (begins && ends) {
              if (q >= n_g) continue;
              float* to = a.out + out_row * D + 64 * d + 8 * g;
              const float* from = a.prior_out + out_row * D + 64 * d + 8 * g;
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = (fp > 0.0f ? fmaf(fp, from[i], o[i]) : o[i]) * inv;
              *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<float4*>(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
            } else {
              float* to = &piece_at(warp, begins)->sum[q][64 * d + 8 * g];
              *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<float4*>(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
            }
          }
          if (g == 0) {
            if (begins && ends) {
              if (a.lse && q < n_g) a.lse[out_row] = base * kLn2 + logf(total);
            } else {
              piece_at(warp, begins)->top[q] = m;
              piece_at(warp, begins)->total[q] = l;
            }
          }
        }
        if (!(begins && ends) && lane == 0)
          s_of[warp][begins] = {cur.b, cur.seg, ends, x - cur.u + cur.ext.units - 1};
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.0f;
      }
      if (x + 1 < x_end) step(cur);
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1;
      }
    }
    if (dead) {                                      // a copy did not arrive: tell, and wait out those under way
      if (lane == 0) raise(p.err, kTimeout);
      for (++x; x < x_ahead; ++x) {
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1;
        }
        ptx::mbar_wait_bounded(&s_full[warp][stage], phase, &s_abort);
      }
    }
  }
  __syncthreads();

  // ---- join the warps' pieces, which are in the order of the units
  const PieceOf* of = s_of[0];
  const int dim = tid % D;                           // a thread takes this dimension of every (kT / D)-th head
  for (int i = 0; i < 2 * kW; ++i) {
    const PieceOf one = of[i];
    if (one.b < 0) continue;
    int n = i;                                       // the last piece of the same segment
    for (int j = i + 1; j < 2 * kW; ++j)
      if (of[j].b == one.b && of[j].seg == one.seg) n = j;
    const bool begins = i % 2, whole = begins && of[n].ends;
    const int h = one.seg / seg_blocks, head0 = h * a.group + (one.seg % seg_blocks) * kSegHeads;
    const int n_g = min(kSegHeads, (h + 1) * a.group - head0);
    float* piece = a.ws + (static_cast<size_t>(blockIdx.x) * 2 + begins) * kPiece;
    for (int q = tid / D; q < n_g; q += kT / D) {
      const int64_t out_row = static_cast<int64_t>(one.b) * a.n_q + head0 + q;
      const float prior = whole && a.prior_lse ? a.prior_lse[out_row] * kLog2e : -INFINITY;
      float top = prior;
      for (int j = i; j <= n; ++j)
        if (of[j].b >= 0) top = fmaxf(top, piece_at(j / 2, j % 2)->top[q]);
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f, total = 0.0f;
      for (int j = i; j <= n; ++j)
        if (of[j].b >= 0) {
          const Piece* one_of = piece_at(j / 2, j % 2);
          const float f = exp2_of(one_of->top[q] - base);
          sum = fmaf(f, one_of->sum[q][dim], sum);
          total = fmaf(f, one_of->total[q], total);
        }
      if (whole) {
        if (prior > -INFINITY) {
          const float f = exp2_of(prior - base);
          sum = fmaf(f, a.prior_out[out_row * D + dim], sum);
          total += f;
        }
        a.out[out_row * D + dim] = total == 0.0f ? 0.0f : sum / total;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + tid / D), "n"(D) : "memory");   // (the log-sum may replace the prior's)
        if (a.lse && dim == 0) a.lse[out_row] = base * kLn2 + logf(total);
      } else {
        piece[q * D + dim] = sum;
        if (dim == 0) {
          piece[kSegHeads * D + q] = top;
          piece[kSegHeads * D + kSegHeads + q] = total;
        }
      }
    }
    if (begins && !whole && tid == 0) desc[blockIdx.x] = make_int4(one.b, one.seg, cta_of(share, one.last_unit), 0);
    i = n;
  }
}

// Joins the pieces of the segments that CTA blockIdx.x of the first launch began and did not end; one CTA
// a query head, a warp takes every eighth piece, a lane four dimensions.
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(kJoinWarps * 32) aatc_paged_join_kernel(const DecodeArgs a, int n_ctas) {
  __shared__ float so[kJoinWarps][D];
  __shared__ float sm[kJoinWarps], sl[kJoinWarps];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int4 what = __ldcg(reinterpret_cast<const int4*>(a.ws + static_cast<size_t>(n_ctas) * 2 * kPiece) + blockIdx.x);
  if (what.x < 0) return;
  const int seg_blocks = (a.group + kSegHeads - 1) / kSegHeads, h = what.y / seg_blocks;
  const int head = h * a.group + (what.y % seg_blocks) * kSegHeads + blockIdx.y;
  if (head >= (h + 1) * a.group) return;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, q = blockIdx.y;
  const int c0 = blockIdx.x, n = what.z - c0 + 1;                // pieces 2 c0 + 1, 2 (c0 + 1), 2 (c0 + 2), ...
  float top = -INFINITY, total = 0.0f;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i = warp; i < n; i += kJoinWarps) {
    const float* piece = a.ws + (static_cast<size_t>(c0 + i) * 2 + (i == 0 ? 1 : 0)) * kPiece;
    const float m = __ldcg(piece + kSegHeads * D + q), l = __ldcg(piece + kSegHeads * D + kSegHeads + q);
    const float4 o = __ldcg(reinterpret_cast<const float4*>(piece + q * D) + lane);
    const float next = fmaxf(top, m), base = next == -INFINITY ? 0.0f : next;
    const float r = exp2_of(top - base), f = exp2_of(m - base);
    total = fmaf(total, r, f * l);
    sum.x = fmaf(sum.x, r, f * o.x);
    sum.y = fmaf(sum.y, r, f * o.y);
    sum.z = fmaf(sum.z, r, f * o.z);
    sum.w = fmaf(sum.w, r, f * o.w);
    top = next;
  }
  *reinterpret_cast<float4*>(&so[warp][4 * lane]) = sum;
  if (lane == 0) {
    sm[warp] = top;
    sl[warp] = total;
  }
  const int64_t out_row = static_cast<int64_t>(what.x) * a.n_q + head;
  const float prior = a.prior_lse ? a.prior_lse[out_row] * kLog2e : -INFINITY;
  __syncthreads();
  if (tid >= D) return;
  top = prior;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, sm[w]);
  const float base = top == -INFINITY ? 0.0f : top;
  float s = 0.0f, l = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    const float f = exp2_of(sm[w] - base);
    s = fmaf(f, so[w][tid], s);
    l = fmaf(f, sl[w], l);
  }
  if (prior > -INFINITY) {
    const float f = exp2_of(prior - base);
    s = fmaf(f, a.prior_out[out_row * D + tid], s);
    l += f;
  }
  a.out[out_row * D + tid] = l == 0.0f ? 0.0f : s / l;
  if (a.lse && tid == 0) a.lse[out_row] = base * kLn2 + logf(l);   // (every thread has read the prior's)
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

size_t decode_workspace(int num_sms) {
  const size_t ctas = static_cast<size_t>(std::max(1, num_sms)) * kDecodeCtas;
  return ctas * (2 * kPiece * sizeof(float) + sizeof(int4));
}

cudaError_t launch_decode(int dtype, const DecodeArgs& a, cudaStream_t st) {
  const int ctas = std::max(1, a.num_sms) * kDecodeCtas;
  const auto kernel = dtype == AATC_BF16 ? aatc_paged_decode_kernel<__nv_bfloat16> : aatc_paged_decode_kernel<__half>;
  // pages as rows of 128 bytes, two a token; a box is a unit's tokens in a page
  CUtensorMap map;
  const uint64_t rows = static_cast<uint64_t>(4) * a.pool.n_kv << a.pool.page_shift;
  cudaError_t e = make_tensor_map_3d(&map, a.pool.pages, D / 2, rows, a.pool.n_pages, D, rows * D, D / 2,
                                     2 * std::min(kUnit, 1 << a.pool.page_shift));
  if (e != cudaSuccess) return e;
  e = ensure_smem_optin(reinterpret_cast<const void*>(kernel), kDecodeSmem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(ctas), dim3(kDecodeWarps * 32), kDecodeSmem, st, a, map);
  if (e != cudaSuccess) return e;
  return launch_pdl(aatc_paged_join_kernel, dim3(ctas, std::min(a.group, kSegHeads)), dim3(kJoinWarps * 32), 0, st, a, ctas);
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
