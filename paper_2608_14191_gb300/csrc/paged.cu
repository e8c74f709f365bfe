// Kernels of the paged cache: rotary positions and append, decode attention, page copies, gather.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

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

// a / b of values that are not negative, of 32 bits or mostly so
__device__ __forceinline__ int quotient(int a, int b) { return static_cast<unsigned>(a) / static_cast<unsigned>(b); }
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
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
// the frequencies 8 u .. 8 u + 7; of the rest, two neighbouring pieces.  A thread takes unit u of kHeads heads of a
// token: all its loads first; while they are under way the CTA makes the sines and cosines of its tokens, each
// once.  Memory is the bound.  (Prompts of 9911 tokens appended, 36 heads and page writes: three heads a thread, 96
// bytes of loads, in CTAs of 128 threads 29.0 us, 6.3 TB/s read and written; two 30.4; three in CTAs of 256 threads
// 29.6, where more wait at the barrier; 32.0 where the page's id was waited for before the angles.)
constexpr int kUnits = 8;
constexpr int kAppendThreads = 128;
constexpr int kJobs = kAppendThreads / kUnits;   // (token, group of heads) pairs of a CTA
constexpr int kHeads = 3;

template <typename T>
__global__ void __launch_bounds__(kAppendThreads) aatc_paged_append_kernel(const AppendArgs a, int groups) {
  // (cos, sin) of pairs 8 u + 2 j, 8 u + 2 j + 1 of a token at [j][u]: neighbouring units read neighbouring 16 bytes
  __shared__ float4 s_turn[kJobs][4][kUnits];
  const Pool& p = a.pool;
  const int n_heads = a.n_q + (p.pages ? 2 * p.n_kv : 0);
  const int64_t job0 = static_cast<int64_t>(blockIdx.x) * kJobs, t0 = quotient(job0, static_cast<int64_t>(groups));
  const unsigned in = static_cast<unsigned>(job0 - t0 * groups), job = in + threadIdx.x / kUnits;   // from token t0 on
  const unsigned slot = job / static_cast<unsigned>(groups);
  const int64_t t = t0 + slot;
  const int group = static_cast<int>(job - slot * groups), u = threadIdx.x % kUnits;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int rot = a.turn.turns ? a.turn.rot_dim : 0;
  const bool turned = 16 * u < rot, apart = turned && !a.turn.interleaved;
  const int off_a = 2 * (apart ? 8 * u : 16 * u), off_b = 2 * (apart ? 8 * u + rot / 2 : 16 * u + 8);   // bytes
  const bool in_range = t < a.n_tokens;
  uint4 x[kHeads][2];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = group + i * groups;
    if (h >= n_heads || !in_range) break;
    const Heads& from = h < a.n_q ? a.q : h < a.n_q + p.n_kv ? a.k : a.v;
    const int head = h < a.n_q ? h : h < a.n_q + p.n_kv ? h - a.n_q : h - a.n_q - p.n_kv;
    const char* src = static_cast<const char*>(from.x) + 2 * (t * from.token_stride + head * from.head_stride);
    x[i][0] = *reinterpret_cast<const uint4*>(src + off_a);
    x[i][1] = *reinterpret_cast<const uint4*>(src + off_b);
  }
  // the token's page, whose id comes while the angles are made
  const bool stores = p.pages && in_range && group + (kHeads - 1) * groups >= a.n_q;
  const int32_t index = stores ? a.index[t] : -1;
  const int64_t row = stores && a.rows ? a.rows[t] : t;
  bool placed = index >= 0;
  if (placed && (row < 0 || row >= a.n_rows || (index >> p.page_shift) >= p.max_pages)) {
    raise(p.err, kBadRow);
    placed = false;
  }
  const int32_t id = placed ? p.table[row * p.table_stride + (index >> p.page_shift)] : 0;
  if (rot > 0) {
    const int pairs = rot / 2, n = static_cast<int>(min(static_cast<int64_t>((in + kJobs - 1) / static_cast<unsigned>(groups)), a.n_tokens - 1 - t0)) + 1;
    const int32_t* positions = (a.positions ? a.positions : a.index) + t0;
    for (int i = threadIdx.x; i < n * pairs; i += kAppendThreads) {
      const int k = i / pairs, w = i - k * pairs;
      reinterpret_cast<float2*>(&s_turn[k][w / 2 % 4][w / 8])[w % 2] = cos_sin(a.turn, positions[k], a.turn.turns[w]);
    }
    __syncthreads();
  }
  if (!in_range) return;
  if (placed && (id < 0 || id >= p.n_pages)) {
    raise(p.err, kBadPage);
    placed = false;
  }
  // keys of all heads of a page, then values; head h of kind c is block (2 id + c) n_kv + h
  char* place = static_cast<char*>(p.pages) +
                ((static_cast<int64_t>(id) * 2 * p.n_kv << p.page_shift) + (index & ((1 << p.page_shift) - 1))) * (2 * D);
  float2 e[8];
  if (turned) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 two = s_turn[slot][j][u];
      e[2 * j] = make_float2(two.x, two.y);
      e[2 * j + 1] = make_float2(two.z, two.w);
    }
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = group + i * groups;
    if (h >= n_heads) break;
    if (turned && h < a.n_q + p.n_kv) {
      uint32_t* wa = reinterpret_cast<uint32_t*>(&x[i][0]);
      uint32_t* wb = reinterpret_cast<uint32_t*>(&x[i][1]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 va = widen(T(), wa[j]), vb = widen(T(), wb[j]);
        if (a.turn.interleaved) {
          wa[j] = narrow(T(), va.x * e[j].x - va.y * e[j].y, va.x * e[j].y + va.y * e[j].x);
          wb[j] = narrow(T(), vb.x * e[4 + j].x - vb.y * e[4 + j].y, vb.x * e[4 + j].y + vb.y * e[4 + j].x);
        } else {
          const float2 e0 = e[2 * j], e1 = e[2 * j + 1];
          wa[j] = narrow(T(), va.x * e0.x - vb.x * e0.y, va.y * e1.x - vb.y * e1.y);
          wb[j] = narrow(T(), va.x * e0.y + vb.x * e0.x, va.y * e1.y + vb.y * e1.x);
        }
      }
    }
    char* dst;
    if (h < a.n_q) dst = static_cast<char*>(a.q_out) + 2 * (t * a.q_out_token_stride + h * a.q_out_head_stride);
    else if (placed) dst = place + (static_cast<int64_t>(h - a.n_q) << p.page_shift) * (2 * D);
    else continue;
    *reinterpret_cast<uint4*>(dst + off_a) = x[i][0];
    *reinterpret_cast<uint4*>(dst + off_b) = x[i][1];
  }
}

// ---------------------------------------------------------------- decode attention
// The work of a call is its units of 16 tokens: those of sequence 0's kv-head 0, then kv-head 1, ...,
// then sequence 1's, a (sequence, kv-head) being a segment.  They are laid out on a line, with a gap before
// every segment for what its begin and end cost a warp; every CTA takes an equal part of the line and each of its
// consumer warps an eighth of that, so the shares are alike whatever the lengths (with shares by CTA and
// a barrier per segment, ragged sequences took twice as long as as many tokens in equal ones).  A segment that
// lies inside a warp's share is finished by the warp, the pieces of one that lies in several warps are joined
// in shared memory, and those of one in several CTAs through the workspace by the second launch.  (Query heads
// beyond eight of a kv-head are further segments over the same tokens, whose keys and values are brought again: 131072 tokens x
// 8 kv-heads of 8 heads 85 us, 12 or 16 heads 128, 32 heads 237; x 1 kv-head 21, 28 and 40.)
// Producer warps bring the units: a lane walks one consumer's share, across the segments, and keeps a ring of
// units under way by TMA, so the consumers execute little more than the matrix instructions and the softmax
// (with the walk in every warp a unit took 530 instructions, and eight warps an SM were held up by issue
// latency before the memory was).  The tensor work is small (4 G flops per byte of cache, G query heads a kv-head), so
// mma.sync on register fragments serves it: the queries are its eight columns, tokens or dimensions its sixteen
// rows.  Between the first copy and the last the memory runs at its full rate; what a call takes beyond that is
// some 3 us to the first copy (dependent loads of lengths and page ids), 2 us from the last one, and the join.
// Measured (graph replay; K and V bytes over the whole time): 131072 tokens x 8 kv-heads 86 us, 6.3 TB/s; 16 x
// 8192 x 4 in f16 47 us, 5.7 TB/s; 61 ragged sequences of 61 876 tokens x 8 with cap and prior 49 us; 1001 tokens 7.4 us.
constexpr int kSegHeads = 8;        // query heads of a segment: the columns of the MMAs
constexpr int kUnit = 16;           // tokens
constexpr int kConsumers = 8;       // consumer warps of a CTA, one CTA an SM; a power of two, at most 16
constexpr int kProducers = 4;       // producer warps (131072 tokens: 87.5 us with two, 86.5 with four)
constexpr int kServes = kConsumers / kProducers;
constexpr int kDecodeThreads = (kConsumers + kProducers) * 32;
constexpr int kUnitsPerCta = 8;     // fewer CTAs where they would get less (1001 tokens: 7.6 us; 16: 8.5, 24: 9.1)
constexpr int kSeqs = 4;            // sequences of a thread in the prefix sums, where one is not enough
constexpr int kChunk = kSeqs * kDecodeThreads;
constexpr int kStages = 2;          // units of a consumer on their way: keys and values, 8 KB each (one: 131072 tokens 104 us,
                                    // 86 with two, as with three when those fitted)
constexpr int kGap = 8;             // units' time that a segment costs beside its units (61 ragged sequences: 5 49.8 us,
                                    // 8 49.7, 12 51.3; 600 of up to 40 tokens 24.7, 24.1, 22.4)
// Where every segment has fewer tokens than this (by the table's width or the window), the CTAs' parts of the line are
// moved to whole segments and there is no second launch.  300 sequences of 1 to 40 tokens x 4 kv-heads: 10.7 us against 17.1
// with it; one sequence x 8 kv-heads of 100 tokens 6.0 against 7.0, of 250 7.3 against 7.1 (and a launch less for the host, 2
// us), of 500 9.5 against 7.3.
constexpr int kWholeTokens = 17 * kUnit;
// Pieces that a segment can have from which sixteen warps join them, not four: 131072 tokens x 1 kv-head 21.2 us against 23.0;
// but 4000 tokens x 1 kv-head (at most 35 pieces) 9.2 against 7.6.
constexpr int kManyPieces = 64;
constexpr int kRow = 128;           // bytes of half a token's key or value: a row in shared memory
constexpr int kStage = kUnit * 4 * kRow;      // keys, then values
constexpr int kPiece = kSegHeads * (D + 2);   // floats of a piece: sums [8][128], maxima [8], totals [8]

// Workspace: pieces [2 n_ctas] (CTA c's share begins inside a segment: piece 2 c; ends inside one that it began:
// 2 c + 1), then int4 per CTA: the segment that it began and did not end (sequence, segment of the
// sequence, last CTA with a piece of it; sequence -1: none).

// The line in even parts: CTA c has [begin(c), begin(c + 1)).  Pos is 32 bits where the table's width bounds the
// line below 2^31, else 64: divisions of 64 bits are 100 instructions each, in the part of the kernel before its
// first load (1001 tokens: 7.6 us with 32 bits, 8.2 with 64).
template <typename Pos>
struct Share {
  Pos each;
  int n_ctas, longer;               // CTAs that get anything; the first of them get one more
  __device__ Pos begin(int c) const { return c * each + min(c, longer); }
  __device__ int cta_of(Pos at) const {
    const Pos big = longer * (each + 1);
    return static_cast<int>(at < big ? quotient(at, each + 1) : longer + quotient(at - big, each));
  }
};

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Four 8 x 8 matrices of 16-bit values, lane l giving the address of row l % 8 of matrix l / 8; lane
// (g, t) = (l / 4, l % 4) gets values 2 t, 2 t + 1 of row g, of the transposed matrices in the second form.
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of an 8 x 8 matrix of 16-bit values over the warp
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_of(float x) {            // (-inf: 0)
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh x = 1 - 2 / (e^(2 x) + 1), and where that cancels its Taylor series: either within 4e-7 of its value
__device__ __forceinline__ float tanh_of(float x) {
  const float a = fabsf(x), x2 = x * x;
  const float big = 1.0f - __fdividef(2.0f, exp2_of(2.0f * kLog2e * a) + 1.0f);
  const float small = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return a < 0.25f ? x * small : copysignf(a > 20.0f ? 1.0f : big, x);
}

// A weight p as a sum of 16-bit values, so that products with 16-bit values on the tensor cores lose
// next to nothing of it.  bf16: three truncations of eight significant bits (all of p's 24).  No part is negative or
// zero, as an infinite value times it would turn into NaN.
// f16: p 2^6 truncated (p is at most 2^8, so at most 2^14) and 2^11 times the rest, rounded, whose products are summed apart and
// scaled back: 22 bits of a weight down to 2^-20 of the reference (the step of the rest's format), below that within
// 2^-42 of the reference, which for a tail of 131072 such tokens is 2^-25 of it (with the rest on the first part's scale
// 2^-14: at that size a tail of weights of 2^-33 was lost).  Parts can be zero, so a unit with infinities or NaN among
// its values is summed by `exact_unit`.  (16 x 8192 tokens x 4 kv-heads: 47.4 us, 47.3 without either.)
template <typename T>
struct Parts;
template <>
struct Parts<__nv_bfloat16> {
  static constexpr int kN = 3;
  static constexpr bool kMayBeZero = false;
  static constexpr float kRest = 1.0f;                         // the scale on the last part, whose products are summed apart if it is not 1
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
  static constexpr bool kMayBeZero = true;
  static constexpr float kRest = 2048.0f;
  static constexpr float kShift = 6.0f;
  static __device__ __forceinline__ void split(float p, float q, uint32_t (&out)[2]) {
    const __half2 h = __halves2half2(__float2half_rz(p), __float2half_rz(q));
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn((p - f.x) * kRest, (q - f.y) * kRest);
    out[0] = *reinterpret_cast<const uint32_t*>(&h);
    out[1] = *reinterpret_cast<const uint32_t*>(&l);
  }
};

// The sums of half a unit's values (64 dimensions, a row of kRow bytes a token) under the fp32 weights s themselves: what the
// MMAs give, but where a value is infinite or NaN also that.  `values`: the first row, in the order in which the copies leave them
// (`half`: which one of the two); lane (g, t4) has the weights of tokens g (s[0], s[1]) and 8 + g (s[2], s[3]) for queries
// 2 t4, 2 t4 + 1.
__device__ __forceinline__ void exact_unit(const unsigned char* values, int half, const float (&s)[4], float (&part)[4][4]) {
  const int lane = threadIdx.x % 32, g = lane / 4, t4 = lane % 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) part[i][0] = part[i][1] = part[i][2] = part[i][3] = 0.0f;
#pragma unroll 1
  for (int tok = 0; tok < kUnit; ++tok) {
    const int from = tok % 8 * 4 + t4, row = 2 * tok + half;
    const float w0 = __shfl_sync(0xffffffffu, tok < 8 ? s[0] : s[2], from);
    const float w1 = __shfl_sync(0xffffffffu, tok < 8 ? s[1] : s[3], from);
#pragma unroll
    for (int i = 0; i < 8; ++i) {                              // dimensions 8 i + g of the half
      const float v = __half2float(reinterpret_cast<const __half*>(values + row * kRow + (i ^ row % 8) * 16)[g]);
      part[i / 2][i % 2 * 2] = fmaf(w0, v, part[i / 2][i % 2 * 2]);
      part[i / 2][i % 2 * 2 + 1] = fmaf(w1, v, part[i / 2][i % 2 * 2 + 1]);
    }
  }
}

// First token and unit count of a sequence: the tokens [lo, n) in units from lo / 16 on; one unit, of nothing,
// for an empty one (somebody has to write its result).
struct Extent {
  int n, lo, units;
};
__device__ __forceinline__ Extent extent_of(const DecodeArgs& a, int len) {
  Extent e;
  e.n = min(max(len, 0), a.pool.max_pages << a.pool.page_shift);
  e.lo = a.window > 0 ? max(0, e.n - a.window) : 0;
  e.units = max(1, e.n / kUnit + (e.n % kUnit > 0) - e.lo / kUnit);   // (n + 15 may pass 31 bits)
  return e;
}

// What a consumer learns of a unit: its first token, the live ones [lo, n) of its sequence, whether the pages of
// its halves are in the pool (bits 0, 1 of `ok`), and where it belongs.
struct __align__(16) Unit {
  int t, lo, n, ok;
  int b, seg, u, units;
};

// A warp's piece of a segment that it does not have whole, in shared memory (four heads' rows apart: other banks).
struct Piece {
  float sum[kSegHeads][D + 4];
  float top[kSegHeads], total[kSegHeads];
};
template <typename Pos>
struct PieceOf {
  int b, seg;                       // b < 0: none
  int ends;
  Pos last_unit;                    // of the segment, on the line
};

// Shared memory: every consumer's ring of stages, which its piece of the segment that it began takes over at the
// end of its share, then the pieces of the segments that it found begun.
constexpr size_t kDecodeSmem = static_cast<size_t>(kConsumers) * (kStages * kStage + sizeof(Piece));
static_assert(sizeof(Piece) <= kStages * kStage && sizeof(Piece) % 16 == 0, "a piece in the place of a ring");

// What one lane of the producer does for its consumer: the walk over the share's units.
struct Walk {
  int b, seg, u, len_next;
  Extent ext;                       // of sequence b
};

// Query heads of a segment: head0 .. head0 + n, of kv-head h.
struct SegHeads {
  int h, head0, n;
};
__device__ __forceinline__ SegHeads heads_of(const DecodeArgs& a, int seg_blocks, int seg) {
  SegHeads s;
  int block = 0;
  s.h = seg;
  if (seg_blocks > 1) {                              // (a division is slow, and rarely needed)
    s.h = seg / seg_blocks;
    block = seg - s.h * seg_blocks;
  }
  s.head0 = s.h * a.group + block * kSegHeads;
  s.n = min(kSegHeads, (s.h + 1) * a.group - s.head0);
  return s;
}

template <typename T, typename Pos>
__global__ void __launch_bounds__(kDecodeThreads, 1)
    aatc_paged_decode_kernel(const DecodeArgs a, const __grid_constant__ CUtensorMap map) {
  constexpr int kW = kConsumers;
  constexpr float kUnshift = 1.0f / (1 << static_cast<int>(Parts<T>::kShift));
  extern __shared__ __align__(1024) unsigned char rings[];   // (the copies' permutation goes by 1024-byte blocks)
  __shared__ PieceOf<Pos> s_of[kW][2];
  __shared__ Unit s_unit[kW][kStages];
  __shared__ Pos s_part[kW + kProducers], s_upto[kChunk];
  __shared__ int s_len[kChunk];
  __shared__ uint64_t s_full[kW][kStages], s_free[kW][kStages];
  __shared__ int s_abort;
  const Pool& p = a.pool;
  const int tid = threadIdx.x, warp = ptx::warp_uniform(tid / 32), lane = tid % 32;
  const int seg_blocks = (a.group + kSegHeads - 1) / kSegHeads, n_seg = p.n_kv * seg_blocks;
  int4* desc = reinterpret_cast<int4*>(a.ws + static_cast<size_t>(gridDim.x) * 2 * kPiece);
  auto piece_at = [&](int w, int begins) {
    return reinterpret_cast<Piece*>(begins ? rings + w * (kStages * kStage) : rings + kW * (kStages * kStage) + w * sizeof(Piece));
  };
  if (tid < kW * kStages) {
    ptx::mbar_init(&s_full[0][0] + tid, 1);
    ptx::mbar_init(&s_free[0][0] + tid, 1);
  }
  if (tid < 2 * kW) s_of[tid / 2][tid % 2].b = -1;
  if (tid == 0) {
    s_abort = 0;
    ptx::prefetch_tmap(&map);
  }
  ptx::fence_mbar_init();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  // ---- the length of the line, and the sequences in which the warps' shares begin: prefix sums over kChunk sequences
  // at a time, which every warp looks its own begin up in
  Pos in_chunk = 0;
  auto scan = [&](int i0, auto seqs) {
    constexpr int kN = decltype(seqs)::value;
    int len[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const int i = i0 + kN * tid + k;
      len[k] = i < a.batch ? __ldcg(a.lens + i) : 0;
    }
    Pos own[kN], upto = 0;                        // up to and with each of the thread's, all of the thread's
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      if (blockIdx.x == 0 && (len[k] < 0 || len[k] > p.max_pages << p.page_shift)) raise(p.err, kBadRow);
      if (i0 + kN * tid + k < a.batch) upto += static_cast<Pos>(extent_of(a, len[k]).units + kGap) * n_seg;
      own[k] = upto;
    }
    const Pos mine = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Pos y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    __syncthreads();                                 // (the last chunk's sums have been read)
    if (lane == 31) s_part[warp] = upto;
#pragma unroll
    for (int k = 0; k < kN; ++k) s_len[kN * tid + k] = len[k];
    __syncthreads();
    in_chunk = 0;
#pragma unroll
    for (int w = 0; w < kW + kProducers; ++w) {
      if (w == warp) upto += in_chunk;
      in_chunk += s_part[w];
    }
#pragma unroll
    for (int k = 0; k < kN; ++k) s_upto[kN * tid + k] = upto - mine + own[k];
  };
  Pos total = 0;
  if (a.batch <= kDecodeThreads) {
    scan(0, std::integral_constant<int, 1>());
    total = in_chunk;
  } else {
    for (int i0 = 0; i0 < a.batch; i0 += kChunk) {
      scan(i0, std::integral_constant<int, kSeqs>());
      total += in_chunk;
    }
  }
  Share<Pos> share;
  share.n_ctas = static_cast<int>(min(static_cast<Pos>(gridDim.x), (total + kUnitsPerCta - 1) / kUnitsPerCta));
  if (tid == 0) desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
  if (blockIdx.x >= share.n_ctas) return;
  share.each = static_cast<Pos>(quotient(total, static_cast<Pos>(share.n_ctas)));
  share.longer = static_cast<int>(total - share.each * share.n_ctas);
  Pos first = share.begin(blockIdx.x), next = share.begin(blockIdx.x + 1);
  if (a.whole) {                                     // (one chunk of sequences)
    __syncthreads();
    auto segment_from = [&](Pos y) {                 // the begin of the first segment that does not begin before y
      if (y >= total) return total;
      int lo = 0, hi = a.batch - 1;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (s_upto[mid] > y) hi = mid;
        else lo = mid + 1;
      }
      const Pos from = lo > 0 ? s_upto[lo - 1] : 0, each = extent_of(a, s_len[lo]).units + kGap;
      return from + static_cast<Pos>(quotient(y - from + each - 1, each)) * each;
    };
    first = segment_from(first);
    next = segment_from(next);
  }
  const Pos here = next - first;
  // This warp's consumers: itself, or those that the first lanes of a producer serve.  A lane's walk begins at its
  // consumer's share: the segment and, behind the gap, the unit there.
  const int w0 = warp < kW ? warp : (warp - kW) * kServes + min(lane, kServes - 1);
  auto share_of = [&](int w) { return first + static_cast<Pos>(static_cast<int64_t>(here) * w / kW); };
  const Pos x_end = share_of(w0 + 1);
  Pos x = share_of(w0);
  Walk at = {};
  {
    int skip = 0;
    bool found = false;
    Pos before = 0;
    for (int i0 = 0; i0 < a.batch; i0 += kChunk) {
      if (a.batch > kChunk) scan(i0, std::integral_constant<int, kSeqs>());
      __syncthreads();
      const Pos begin = x - before;
      if (begin >= 0 && begin < in_chunk) {
        int lo = 0, hi = min(a.batch - i0, kChunk) - 1;  // the first sequence whose end is past `begin`
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (s_upto[mid] > begin) hi = mid;
          else lo = mid + 1;
        }
        at.b = i0 + lo;
        at.ext = extent_of(a, s_len[lo]);
        const Pos in_seq = begin - (lo > 0 ? s_upto[lo - 1] : 0);
        at.seg = static_cast<int>(quotient(in_seq, static_cast<Pos>(at.ext.units + kGap)));
        const int in_seg = static_cast<int>(in_seq - static_cast<Pos>(at.seg) * (at.ext.units + kGap));
        at.u = max(0, in_seg - kGap);
        skip = max(0, kGap - in_seg);
        found = true;
      }
      before += in_chunk;
      if (before > share_of(kW - 1)) break;
    }
    x = found ? x + skip : x_end;                    // (not found: lengths that changed between two reads of them)
  }
  if (warp >= kW) {
    // ---- a producer: each of its first lanes serves a consumer
    const bool on = lane < kServes;
    const int w = w0;
    at.len_next = on && at.b + 1 < a.batch ? __ldcg(a.lens + at.b + 1) : 0;
    int id0 = -1, id1 = -1;                          // pages of the unit's halves
    auto fetch_ids = [&]() {
      const int t = (at.ext.lo / kUnit + at.u) * kUnit;
      if (!on || x >= x_end || t >= at.ext.n) return;
      const int32_t* row = p.table + static_cast<int64_t>(at.b) * p.table_stride;
      id0 = row[t >> p.page_shift];
      id1 = p.page_shift > 3 ? id0 : t + 8 < at.ext.n ? row[(t + 8) >> p.page_shift] : -1;
    };
    fetch_ids();
    int stage = 0, round = 0;
    uint64_t idle_since = 0;
    for (;;) {
      const bool work = on && x < x_end;
      if (!__any_sync(0xffffffffu, work)) break;
      const bool can = work && (round == 0 || ptx::mbar_test_wait(&s_free[w][stage], (round - 1) & 1));
      if (can) {
        const int t = (at.ext.lo / kUnit + at.u) * kUnit;
        bool ok0 = t < at.ext.n && t + 8 > at.ext.lo, ok1 = t + 8 < at.ext.n;      // live (a unit has t + 16 > lo)
        if ((ok0 && static_cast<uint32_t>(id0) >= static_cast<uint32_t>(p.n_pages)) ||
            (ok1 && static_cast<uint32_t>(id1) >= static_cast<uint32_t>(p.n_pages))) {
          raise(p.err, kBadPage);
          ok0 = ok0 && static_cast<uint32_t>(id0) < static_cast<uint32_t>(p.n_pages);
          ok1 = ok1 && static_cast<uint32_t>(id1) < static_cast<uint32_t>(p.n_pages);
        }
        Unit* un = &s_unit[w][stage];
        *reinterpret_cast<int4*>(&un->t) = make_int4(t, at.ext.lo, at.ext.n, (ok0 ? 1 : 0) | (ok1 ? 2 : 0));
        *reinterpret_cast<int4*>(&un->b) = make_int4(at.b, at.seg, at.u, at.ext.units);
        unsigned char* to = rings + (w * kStages + stage) * kStage;
        uint64_t* bar = &s_full[w][stage];
        const int row = (heads_of(a, seg_blocks, at.seg).h << p.page_shift) + (t & ((1 << p.page_shift) - 1)), v_row = p.n_kv << p.page_shift;
        if (p.page_shift > 3) {                      // a unit lies in one page: boxes of sixteen tokens
          ptx::mbar_arrive_expect_tx(bar, ok0 || ok1 ? kStage : 0);
          if (ok0 || ok1) {
            ptx::tma_load_4d(to, &map, bar, 0, 0, row, id0);
            ptx::tma_load_4d(to + kStage / 2, &map, bar, 0, 0, row + v_row, id0);
          }
        } else {
          ptx::mbar_arrive_expect_tx(bar, (ok0 ? kStage / 2 : 0) + (ok1 ? kStage / 2 : 0));
          if (ok0) {
            ptx::tma_load_4d(to, &map, bar, 0, 0, row, id0);
            ptx::tma_load_4d(to + kStage / 2, &map, bar, 0, 0, row + v_row, id0);
          }
          if (ok1) {
            ptx::tma_load_4d(to + kStage / 4, &map, bar, 0, 0, row, id1);
            ptx::tma_load_4d(to + kStage / 4 * 3, &map, bar, 0, 0, row + v_row, id1);
          }
        }
        ++x;
        if (++at.u == at.ext.units) {
          at.u = 0;
          x += kGap;
          if (++at.seg == n_seg) {
            at.seg = 0;
            ++at.b;
            at.ext = extent_of(a, at.len_next);      // (of nothing past the last sequence)
            if (at.b >= a.batch) x = x_end;
            at.len_next = at.b + 1 < a.batch ? __ldcg(a.lens + at.b + 1) : 0;
          }
        }
        fetch_ids();
        if (++stage == kStages) {
          stage = 0;
          ++round;
        }
      }
      if (__any_sync(0xffffffffu, can)) {            // (whichever lane went on: the others may have nothing to do for long)
        idle_since = 0;
      } else {                                       // (a consumer that stopped, stops this too)
        if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&s_abort))) break;
        const uint64_t now = ptx::globaltimer_ns();
        if (idle_since == 0) idle_since = now;
        if (__any_sync(0xffffffffu, now - idle_since > 2000000000ull)) break;
      }
    }
  } else {
    // ---- a consumer
    const int g = lane / 4, t4 = lane % 4;
    const Pos x_begin = x;
    unsigned char* ring = rings + warp * (kStages * kStage);
    // Rows of 128 bytes: [token][half of the head's values], their 16-byte pieces permuted by the row's number modulo
    // 8.  Keys: matrices (tokens 0 .. 7, 8 .. 15) x (piece, next piece), the A operand of a score MMA,
    // whose rows are tokens; values: (piece, next) x (tokens 0 .. 7, 8 .. 15), transposed the A operand of an
    // output MMA, whose rows are dimensions.  (Tokens t and t + 4 of a matrix lie in the same banks.)
    const int k_row = 2 * (lane / 8 % 2 * 8 + lane % 8), v_row = 2 * (lane / 16 * 8 + lane % 8);
    const uint32_t k_at = k_row * kRow + ((lane / 16) ^ k_row % 8) * 16;
    const uint32_t v_at = kStage / 2 + v_row * kRow + ((lane / 8 % 2) ^ v_row % 8) * 16;
    const float unit_scale = a.scale * kLog2e, cap_in = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap_out = a.cap * kLog2e;
    const bool plain = a.cap <= 0.0f && !a.slopes;
    uint32_t qf[8][2], q_next[8][2];                 // B operand of the score MMAs: column g; of the next segment
    auto load_q = [&](int b, int seg, uint32_t (&to)[8][2]) {
      const SegHeads sh = heads_of(a, seg_blocks, seg);
      const T* q = static_cast<const T*>(a.q.x) + b * a.q.token_stride + (sh.head0 + g) * a.q.head_stride + 2 * t4;
      const bool in = b < a.batch && g < sh.n;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        to[j][0] = in ? *reinterpret_cast<const uint32_t*>(q + 16 * j) : 0u;
        to[j][1] = in ? *reinterpret_cast<const uint32_t*>(q + 16 * j + 8) : 0u;
      }
    };
    if (x < x_end) load_q(at.b, at.seg, q_next);
    float slope0 = 0.0f, slope1 = 0.0f;
    float acc[8][4];                                 // dimensions 16 i + g, 16 i + 8 + g; queries 2 t4, 2 t4 + 1
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;
    int stage = 0;
    uint32_t phase = 0;
    bool fresh = true;                               // the next unit is of another segment
    while (x < x_end) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(&s_full[warp][stage], phase, &s_abort))) {
        if (lane == 0) {                             // a copy did not arrive: tell, and stop the others
          raise(p.err, kTimeout);
          *reinterpret_cast<volatile int*>(&s_abort) = 1;
        }
        break;
      }
      const int4 ua = *reinterpret_cast<const int4*>(&s_unit[warp][stage].t);      // t, lo, n, ok
      const int4 ub = *reinterpret_cast<const int4*>(&s_unit[warp][stage].b);      // b, seg, u, units
      const SegHeads sh = heads_of(a, seg_blocks, ub.y);
      const int head0 = sh.head0, n_g = sh.n;
      const bool ends = ub.z == ub.w - 1;
      const Pos x_next = x + (ends ? 1 + kGap : 1);
      if (fresh) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          qf[j][0] = q_next[j][0];
          qf[j][1] = q_next[j][1];
        }
        if (a.slopes) {
          slope0 = 2 * t4 < n_g ? a.slopes[head0 + 2 * t4] * kLog2e : 0.0f;
          slope1 = 2 * t4 + 1 < n_g ? a.slopes[head0 + 2 * t4 + 1] * kLog2e : 0.0f;
        }
        if (a.prior_lse && lane / 4 < n_g) {         // to L2, for whoever finishes the segment
          const int64_t row = static_cast<int64_t>(ub.x) * a.n_q + head0 + lane / 4;
          asm volatile("prefetch.global.L2 [%0];" ::"l"(a.prior_out + row * D + lane % 4 * 32));
          asm volatile("prefetch.global.L2 [%0];" ::"l"(a.prior_lse + row));
        }
        fresh = false;
      }
      if (ends && x_next < x_end) load_q(ub.y + 1 < n_seg ? ub.x : ub.x + 1, ub.y + 1 < n_seg ? ub.y + 1 : 0, q_next);
      const uint32_t base = ptx::smem_u32(ring) + stage * kStage;
      const bool edge = ua.x < ua.y || ua.z - ua.x < kUnit || ua.w != 3;
      if (edge) {                                    // values of masked tokens: their weight is 0, but 0 x NaN is not
        for (int i = lane; i < kUnit * 2 * kRow / 16; i += 32) {
          const int tok = i / 16;
          if (!(ua.w >> tok / 8 & 1) || ua.x + tok < ua.y || ua.x + tok >= ua.z)
            *reinterpret_cast<uint4*>(ring + stage * kStage + kStage / 2 + i * 16) = make_uint4(0, 0, 0, 0);
        }
        ptx::fence_proxy_async_smem();               // (the next copy to the stage comes after)
        __syncwarp();
      }
      float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s2[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      {
        uint32_t k[2][4][4];                         // (all loads before the products: a warp issues in order)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ldsm(k[0][j], base + (k_at ^ 32 * j));
          ldsm(k[1][j], base + (k_at ^ 32 * j ^ 16) + kRow);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          mma<T>(s, k[0][j], qf[j][0], qf[j][1]);
          mma<T>(s2, k[1][j], qf[4 + j][0], qf[4 + j][1]);
        }
      }
      // ---- scores in units of ln 2 after `c`: s[0], s[1] token g, s[2], s[3] token 8 + g; queries 2 t4, 2 t4 + 1
      float c = unit_scale;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += s2[i];
      if (!plain) {
        if (a.cap > 0.0f) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[i] = cap_out * tanh_of(s[i] * cap_in);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[i] *= c;
        }
        const float back0 = static_cast<float>(ua.x + g - (ua.z - 1)), back1 = static_cast<float>(ua.x + g + 8 - (ua.z - 1));
        s[0] = fmaf(slope0, back0, s[0]);
        s[1] = fmaf(slope1, back0, s[1]);
        s[2] = fmaf(slope0, back1, s[2]);
        s[3] = fmaf(slope1, back1, s[3]);
        c = 1.0f;
      }
      if (edge || c < 0.0f) {
        // (a scale below 0 would turn the masked scores around: apply it first)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] *= c;
        c = 1.0f;
        if (!(ua.w & 1) || ua.x + g < ua.y || ua.x + g >= ua.z) s[0] = s[1] = -INFINITY;
        if (!(ua.w & 2) || ua.x + g + 8 < ua.y || ua.x + g + 8 >= ua.z) s[2] = s[3] = -INFINITY;
      }
      // ---- the running reference of the exponents follows the maximum only when that is 2^8 past it
      const float top0 = fmaxf(s[0], s[2]) * c, top1 = fmaxf(s[1], s[3]) * c;
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
      s[0] = exp2_of(fmaf(s[0], c, -base0));
      s[1] = exp2_of(fmaf(s[1], c, -base1));
      s[2] = exp2_of(fmaf(s[2], c, -base0));
      s[3] = exp2_of(fmaf(s[3], c, -base1));
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
      // the tensor cores' sums are cut off, not rounded: over a long chain into one accumulator that adds up, so a
      // unit's are added to it by rounded additions.  Four independent chains at a time.
#pragma unroll
      for (int i0 = 0; i0 < 8; i0 += 4) {
        uint32_t v[4][4];
        float part[4][4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) ldsm_t(v[i], base + (i0 / 4) * kRow + (v_at ^ 32 * i ^ (i0 / 4) * 16));
        float rest[4][4] = {};
#pragma unroll
        for (int y = Parts<T>::kN - 1; y >= 0; --y)
#pragma unroll
          for (int i = 0; i < 4; ++i) mma<T>(Parts<T>::kRest != 1.0f && y == Parts<T>::kN - 1 ? rest[i] : part[i], v[i], w[0][y], w[1][y]);
        if constexpr (Parts<T>::kRest != 1.0f) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y) part[i][y] = fmaf(rest[i][y], 1.0f / Parts<T>::kRest, part[i][y]);
        }
        if constexpr (Parts<T>::kMayBeZero) {
          float probe[4] = {};                       // not finite where a sum is not
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y) probe[y] += part[i][y];
          if (__any_sync(0xffffffffu, !(fabsf((probe[0] + probe[1]) + (probe[2] + probe[3])) < INFINITY)))
            exact_unit(ring + stage * kStage + kStage / 2, i0 / 4, s, part);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) acc[i0 + i][y] += part[i][y];
      }
      __syncwarp();                                  // every lane has read the stage
      if (lane == 0) ptx::mbar_arrive(&s_free[warp][stage]);
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1;
      }

      if (ends || x_next >= x_end) {                 // the segment's or the share's last unit
        fresh = true;
        const bool begins = x - ub.z >= x_begin, whole = begins && ends;
        const int64_t row0 = static_cast<int64_t>(ub.x) * a.n_q + head0 + 2 * t4;
        float prior[2] = {-INFINITY, -INFINITY}, prior_out[2][16];   // (all loads before the stores, which may be to the same place)
        const bool joins = whole && a.prior_lse;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (joins && 2 * t4 + i < n_g) {
            prior[i] = a.prior_lse[row0 + i] * kLog2e;
#pragma unroll
            for (int j = 0; j < 16; ++j) prior_out[i][j] = a.prior_out[(row0 + i) * D + g + 8 * j];
          }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          l0 += __shfl_xor_sync(0xffffffffu, l0, o);
          l1 += __shfl_xor_sync(0xffffffffu, l1, o);
        }
        l0 *= kUnshift;
        l1 *= kUnshift;
        __syncwarp();                                // (the log-sum may replace the prior's)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int q = 2 * t4 + i;
          const float m = i ? m1 : m0, l = i ? l1 : l0;
          if (whole) {
            float top = fmaxf(m, prior[i]);
            if (top == -INFINITY) top = 0.0f;
            const float fm = exp2_of(m - top), fp = exp2_of(prior[i] - top);
            const float total = fmaf(l, fm, fp), inv = total == 0.0f ? 0.0f : 1.0f / total;
            if (q < n_g) {
              float* to = a.out + (row0 + i) * D + g;
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                float o = acc[j / 2][2 * (j % 2) + i] * (fm * kUnshift);
                if (fp > 0.0f) o = fmaf(fp, prior_out[i][j], o);
                to[8 * j] = o * inv;
              }
              if (a.lse && g == 0) a.lse[row0 + i] = top * kLn2 + logf(total);
            }
          } else {
            Piece* to = piece_at(warp, begins);
#pragma unroll
            for (int j = 0; j < 16; ++j) to->sum[q][8 * j + g] = acc[j / 2][2 * (j % 2) + i] * kUnshift;
            if (g == 0) {
              to->top[q] = m;
              to->total[q] = l;
            }
          }
        }
        if (!(begins && ends) && lane == 0) s_of[warp][begins] = {ub.x, ub.y, ends, x - ub.z + ub.w - 1};
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.0f;
      }
      x = x_next;
    }
  }
  __syncthreads();
  if (s_abort) {                                     // copies under way write to this CTA's memory: wait them out
    if (tid == 0) {
      const uint64_t t0 = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - t0 < 100000000ull) __nanosleep(1000000);
    }
    __syncthreads();
    return;
  }

  // ---- join the warps' pieces, which are in the order of the units: a warp takes a query head of a segment
  if (warp >= kW) return;
  const PieceOf<Pos>* of = s_of[0];
  unsigned left = __ballot_sync(0xffffffffu, lane < 2 * kW && of[lane % (2 * kW)].b >= 0);
  int heads_before = 0;
  while (left) {
    const int i = __ffs(left) - 1;
    const PieceOf<Pos> one = of[i];
    const unsigned same = __ballot_sync(0xffffffffu, lane < 2 * kW && of[lane % (2 * kW)].b == one.b &&
                                                         of[lane % (2 * kW)].seg == one.seg);
    left &= ~same;
    const bool begins = i % 2, whole = begins && of[31 - __clz(same)].ends;
    const SegHeads sh = heads_of(a, seg_blocks, one.seg);
    const int head0 = sh.head0, n_g = sh.n;
    float* piece = a.ws + (static_cast<size_t>(blockIdx.x) * 2 + begins) * kPiece;
    for (int q = (warp - heads_before) & (kW - 1); q < n_g; q += kW) {
      const int64_t out_row = static_cast<int64_t>(one.b) * a.n_q + head0 + q;
      float prior = -INFINITY;
      float4 prior_out = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (whole && a.prior_lse) {
        prior = a.prior_lse[out_row] * kLog2e;
        prior_out = *reinterpret_cast<const float4*>(a.prior_out + out_row * D + 4 * lane);
      }
      const bool has = same >> lane & 1;             // lane j has piece j's factor
      const Piece* of_lane = piece_at(lane / 2 % kW, lane % 2);
      const float top = has ? of_lane->top[q] : -INFINITY;
      float best = fmaxf(top, prior);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
      const float base = best == -INFINITY ? 0.0f : best, f = exp2_of(top - base);
      float total = has ? f * of_lane->total[q] : 0.0f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      float4 v[kW];                                  // (a warp has one piece of a segment at most; all loads first)
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const unsigned mine = same >> 2 * w & 3u;
        v[w] = mine ? *reinterpret_cast<const float4*>(&piece_at(w, mine / 2)->sum[q][4 * lane]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      }
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const float fw = __shfl_sync(0xffffffffu, f, 2 * w + (same >> (2 * w + 1) & 1u));
        sum.x = fmaf(fw, v[w].x, sum.x);
        sum.y = fmaf(fw, v[w].y, sum.y);
        sum.z = fmaf(fw, v[w].z, sum.z);
        sum.w = fmaf(fw, v[w].w, sum.w);
      }
      if (whole) {
        const float fp = exp2_of(prior - base);
        total += fp;
        if (fp > 0.0f) {
          sum.x = fmaf(fp, prior_out.x, sum.x);
          sum.y = fmaf(fp, prior_out.y, sum.y);
          sum.z = fmaf(fp, prior_out.z, sum.z);
          sum.w = fmaf(fp, prior_out.w, sum.w);
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        *reinterpret_cast<float4*>(a.out + out_row * D + 4 * lane) =
            make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
        __syncwarp();                                // (the log-sum may replace the prior's)
        if (a.lse && lane == 0) a.lse[out_row] = base * kLn2 + logf(total);
      } else {
        *reinterpret_cast<float4*>(piece + q * D + 4 * lane) = sum;
        if (lane == 0) {
          piece[kSegHeads * D + q] = best;
          piece[kSegHeads * D + kSegHeads + q] = total;
        }
      }
    }
    heads_before += n_g;
    if (begins && !whole && tid == 0) desc[blockIdx.x] = make_int4(one.b, one.seg, share.cta_of(one.last_unit), 0);
  }
}

// Joins the pieces of the segment that CTA blockIdx.x of the first launch began and did not end; one CTA
// a query head.  A warp takes every kJoinWarps-th piece, a lane four dimensions, eight pieces' loads at a time.
template <int kJoinWarps>
__global__ void __launch_bounds__(kJoinWarps * 32) aatc_paged_join_kernel(const DecodeArgs a, int n_ctas) {
  __shared__ float so[kJoinWarps][D];
  __shared__ float sm[kJoinWarps], sl[kJoinWarps];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, q = blockIdx.y, c0 = blockIdx.x;
  const int seg_blocks = (a.group + kSegHeads - 1) / kSegHeads;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int4 what = __ldcg(reinterpret_cast<const int4*>(a.ws + static_cast<size_t>(n_ctas) * 2 * kPiece) + c0);
  const int h = what.y / seg_blocks, head = h * a.group + (what.y % seg_blocks) * kSegHeads + q;
  if (what.x < 0 || head >= (h + 1) * a.group) return;
  const int n = what.z - c0 + 1;                                  // pieces 2 c0 + 1, 2 (c0 + 1), 2 (c0 + 2), ...
  const int64_t out_row = static_cast<int64_t>(what.x) * a.n_q + head;
  const float prior = a.prior_lse ? a.prior_lse[out_row] * kLog2e : -INFINITY;
  const float prior_out = a.prior_lse && tid < D ? a.prior_out[out_row * D + tid] : 0.0f;
  float top = -INFINITY, total = 0.0f;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kAtOnce = 8;
  for (int i0 = warp; i0 < n; i0 += kJoinWarps * kAtOnce) {
    float m[kAtOnce], l[kAtOnce];
    float4 o[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kJoinWarps;
      const float* piece = a.ws + (static_cast<size_t>(c0 + i) * 2 + (i == 0 ? 1 : 0)) * kPiece;
      m[k] = i < n ? __ldcg(piece + kSegHeads * D + q) : -INFINITY;
      l[k] = i < n ? __ldcg(piece + kSegHeads * D + kSegHeads + q) : 0.0f;
      o[k] = i < n ? __ldcg(reinterpret_cast<const float4*>(piece + q * D) + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    float next = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) next = fmaxf(next, m[k]);
    const float base = next == -INFINITY ? 0.0f : next, r = exp2_of(top - base);
    total *= r;
    sum.x *= r;
    sum.y *= r;
    sum.z *= r;
    sum.w *= r;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float f = exp2_of(m[k] - base);
      total = fmaf(f, l[k], total);
      sum.x = fmaf(f, o[k].x, sum.x);
      sum.y = fmaf(f, o[k].y, sum.y);
      sum.z = fmaf(f, o[k].z, sum.z);
      sum.w = fmaf(f, o[k].w, sum.w);
    }
    top = next;
  }
  *reinterpret_cast<float4*>(&so[warp][4 * lane]) = sum;
  if (lane == 0) {
    sm[warp] = top;
    sl[warp] = total;
  }
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
    s = fmaf(f, prior_out, s);
    l += f;
  }
  a.out[out_row * D + tid] = l == 0.0f ? 0.0f : s / l;
  if (a.lse && tid == 0) a.lse[out_row] = base * kLn2 + logf(l);   // (every thread has read the prior's)
}

// ---------------------------------------------------------------- page copies
constexpr int kCopyVecs = 4;        // 16-byte pieces of a thread, all loaded before the first is stored

// One CTA per 16 KB of a page (blockIdx.x), pair and layer.  Memory is the bound: 1203 pages of 128 KB x 4 layers in
// 189 us, 6.7 TB/s read and written, as a plain copy; one load at a time took 206.  Few pages are a matter of spreading
// them: 7 pages of 64 KB x 32 layers in 3.9 us, 9.6 with a CTA a page.
template <int N>
__global__ void __launch_bounds__(256) aatc_pages_copy_kernel(uint4* pages, int64_t page_vecs, int64_t layer_vecs,
                                                              const __grid_constant__ CopyPairs<N> pairs) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int2 pr = pairs.pair[blockIdx.y];
  const uint4* src = pages + blockIdx.z * layer_vecs + pr.x * page_vecs;
  uint4* dst = pages + blockIdx.z * layer_vecs + pr.y * page_vecs;
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * (256 * kCopyVecs) + threadIdx.x;
  uint4 x[kCopyVecs];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + 256 * k < page_vecs) x[k] = src[i0 + 256 * k];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + 256 * k < page_vecs) dst[i0 + 256 * k] = x[k];
}

// ---------------------------------------------------------------- gather
// A token's row is the keys of all kv-heads, then the values; one CTA per 16 KB of a sequence's rows, four pieces a
// thread, all loaded before the first is stored.  Memory is the bound: 6 prompts padded to 8192 tokens x 8 kv-heads in 37 us, 6.5
// TB/s read and written (42 with a CTA a token); 16 x 16 tokens in 2.5 us, two round trips.
__global__ void __launch_bounds__(256) aatc_paged_gather_kernel(const GatherArgs a) {
  constexpr int kVecs = D / 8;                                 // 16-byte pieces of a head
  const Pool& p = a.pool;
  const uint32_t row_vecs = 2 * p.n_kv * kVecs;
  const int r = blockIdx.y;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int n = a.lens ? a.lens[r] : INT32_MAX;
  const int32_t* row = p.table + static_cast<int64_t>(r) * p.table_stride;
  uint4 x[kCopyVecs];
  uint4* to[kCopyVecs];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * kCopyVecs + k) * 256 + threadIdx.x;
    const int64_t i_tok = i >> 32 ? i / row_vecs : static_cast<uint32_t>(i) / row_vecs;
    to[k] = nullptr;
    if (i_tok >= a.n_tokens) continue;
    const int c = static_cast<int>(i - i_tok * row_vecs), h = c / kVecs, t = a.first + static_cast<int>(i_tok);
    const bool key = h < p.n_kv;
    to[k] = static_cast<uint4*>(key ? a.k_out : a.v_out) +
            ((static_cast<int64_t>(r) * a.n_tokens + i_tok) * p.n_kv + (key ? h : h - p.n_kv)) * kVecs + c % kVecs;
    x[k] = make_uint4(0, 0, 0, 0);
    if (t >= n) continue;
    const int32_t id = row[t >> p.page_shift];
    if (id < 0 || id >= p.n_pages) {
      raise(p.err, kBadPage);
      continue;
    }
    x[k] = static_cast<const uint4*>(p.pages)[(((static_cast<int64_t>(id) * 2 * p.n_kv + h) << p.page_shift) +
                                               (t & ((1 << p.page_shift) - 1))) * kVecs + c % kVecs];
  }
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (to[k]) *to[k] = x[k];
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.lens && (n < 0 || n > static_cast<int64_t>(p.max_pages) << p.page_shift))
    raise(p.err, kBadRow);
}

}  // namespace

cudaError_t launch_append(int dtype, const AppendArgs& a, cudaStream_t st) {
  const int n_heads = a.n_q + (a.pool.pages ? 2 * a.pool.n_kv : 0), groups = (n_heads + kHeads - 1) / kHeads;
  const int64_t blocks = (static_cast<int64_t>(a.n_tokens) * groups + kJobs - 1) / kJobs;
  if (blocks > INT32_MAX) return cudaErrorNotSupported;
  const auto kernel = dtype == AATC_BF16 ? aatc_paged_append_kernel<__nv_bfloat16> : aatc_paged_append_kernel<__half>;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kAppendThreads), 0, st, a, groups);
}

size_t decode_workspace(int num_sms) {
  return static_cast<size_t>(std::max(1, num_sms)) * (2 * kPiece * sizeof(float) + sizeof(int4));
}

cudaError_t launch_decode(int dtype, const DecodeArgs& a, cudaStream_t st) {
  const int ctas = std::max(1, a.num_sms);
  const int64_t seqs_units = (static_cast<int64_t>(a.pool.max_pages) << a.pool.page_shift) / kUnit + 1 + kGap;
  const int n_seg = a.pool.n_kv * ((a.group + kSegHeads - 1) / kSegHeads);
  // tokens and units of the longest segment that the table's width and the window let be
  const int64_t room = static_cast<int64_t>(a.pool.max_pages) << a.pool.page_shift;
  const int64_t tokens_most = a.window > 0 ? std::min<int64_t>(room, a.window) : room, units_most = tokens_most / kUnit + 2;
  DecodeArgs args = a;
  args.whole = tokens_most < kWholeTokens && a.batch <= kChunk;
  const bool narrow = seqs_units * n_seg < ((1ll << 31) - (1 << 16)) / a.batch;
  const bool bf16 = dtype == AATC_BF16;
  const auto kernel = narrow ? (bf16 ? aatc_paged_decode_kernel<__nv_bfloat16, int> : aatc_paged_decode_kernel<__half, int>)
                             : (bf16 ? aatc_paged_decode_kernel<__nv_bfloat16, int64_t> : aatc_paged_decode_kernel<__half, int64_t>);
  CUtensorMap map;                  // [page][token of a head of keys or values][half][64]
  const uint64_t tokens = static_cast<uint64_t>(2) * a.pool.n_kv << a.pool.page_shift;
  cudaError_t e = make_tensor_map_halves(&map, a.pool.pages, tokens, a.pool.n_pages, kRow,
                                         std::min(kUnit, 1 << a.pool.page_shift));
  if (e != cudaSuccess) return e;
  e = ensure_smem_optin(reinterpret_cast<const void*>(kernel), kDecodeSmem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(ctas), dim3(kDecodeThreads), kDecodeSmem, st, args, map);
  if (e != cudaSuccess || args.whole) return e;
  // the segments of a sequence are equally long, so one has pieces in an n_seg-th of the CTAs in use, and two, at most
  const int64_t used = std::min<int64_t>(ctas, (units_most + kGap + kUnitsPerCta - 1) * n_seg * a.batch / kUnitsPerCta);
  const dim3 grid(ctas, std::min(a.group, kSegHeads));
  if (used / n_seg + 2 > kManyPieces) return launch_pdl(aatc_paged_join_kernel<16>, grid, dim3(16 * 32), 0, st, a, ctas);
  return launch_pdl(aatc_paged_join_kernel<4>, grid, dim3(4 * 32), 0, st, a, ctas);
}

template <int N>
static cudaError_t launch_copy_n(void* pages, size_t page_bytes, int n_layers, size_t layer_stride, const int32_t* pairs,
                                 int n, cudaStream_t st) {
  CopyPairs<N> cp;
  for (int i = 0; i < n; ++i) cp.pair[i] = make_int2(pairs[2 * i], pairs[2 * i + 1]);
  const int64_t vecs = static_cast<int64_t>(page_bytes / 16);
  const dim3 grid(static_cast<unsigned>((vecs + 256 * kCopyVecs - 1) / (256 * kCopyVecs)), n, n_layers);
  return launch_pdl(aatc_pages_copy_kernel<N>, grid, dim3(256), 0, st, static_cast<uint4*>(pages), vecs,
                    static_cast<int64_t>(layer_stride / 16), cp);
}

cudaError_t launch_copy(void* pages, size_t page_bytes, int n_layers, size_t layer_stride, const int32_t* pairs,
                        int n_pairs, cudaStream_t st) {
  // pairs of a launch: 4000 bytes of parameters, or 240 (host time of a copy of 7 pairs 2.7 us with these, 3.1 with those)
  constexpr int kMost = 500, kFew = 30;
  for (int i0 = 0; i0 < n_pairs; i0 += kMost) {
    const int n = std::min(kMost, n_pairs - i0);
    const cudaError_t e = (n <= kFew ? launch_copy_n<kFew> : launch_copy_n<kMost>)(pages, page_bytes, n_layers, layer_stride,
                                                                                  pairs + 2 * i0, n, st);
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
    const int64_t vecs = static_cast<int64_t>(a.n_tokens) * a.pool.n_kv * (2 * D / 8);
    const int64_t blocks = (vecs + 256 * kCopyVecs - 1) / (256 * kCopyVecs);
    if (blocks > INT32_MAX) return cudaErrorNotSupported;
    const cudaError_t e = launch_pdl(aatc_paged_gather_kernel, dim3(static_cast<unsigned>(blocks), s.n_rows), dim3(256), 0, st, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace paged
}  // namespace aatc
