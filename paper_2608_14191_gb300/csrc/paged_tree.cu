// Attention of the last tokens of every sequence over its pages (drafted trees, chains), and the weights that tokens get in it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "aatc_internal.h"
#include "paged.h"
#include "paged_device.cuh"
#include "ptx.cuh"

namespace aatc {
namespace paged {

namespace {

// Sequence b: its queries i0 .. i0 + n, the last n of its len tokens.  (Without starts a row of length 0 is a free slot: its query is
// none of a sequence's, and its results say so.)
struct Seq {
  int i0, n, len;
  __device__ int before() const { return len - n; }
};
__device__ __forceinline__ Seq seq_of(const TreeArgs& a, int b, bool tells) {
  Seq s;
  const int len = a.lens[b], most = a.pool.max_pages << a.pool.page_shift;
  s.len = min(max(len, 0), most);
  s.i0 = a.starts ? a.starts[b] : b;
  const int end = a.starts ? a.starts[b + 1] : b + (len != 0);
  const bool ok = len == s.len && s.i0 >= 0 && s.i0 <= end && end <= a.n_tokens && end - s.i0 <= len &&
                  (!a.mask || end - s.i0 <= static_cast<int64_t>(a.mask_words) * 32);
  s.n = ok ? end - s.i0 : 0;
  if (!ok && tells) raise(a.pool.err, kBadRow);
  return s;
}

// Whether query i of the sequence sees its token t.
__device__ __forceinline__ bool sees(const TreeArgs& a, const Seq& s, int i, int t) {
  const int j = t - s.before();
  if (j < 0) return true;
  if (t >= s.len) return false;
  return a.mask ? a.mask[static_cast<int64_t>(s.i0 + i) * a.mask_words + j / 32] >> j % 32 & 1 : j <= i;
}

// Token t of the table's row in head h: its key (kind 0) or value (1); null for a page outside the pool.
template <typename T>
__device__ __forceinline__ const T* token_at(const Pool& p, int b, int h, int kind, int t) {
  const int32_t id = p.table[static_cast<int64_t>(b) * p.table_stride + (t >> p.page_shift)];
  if (id < 0 || id >= p.n_pages) {
    raise(p.err, kBadPage);
    return nullptr;
  }
  const int64_t row = (((static_cast<int64_t>(id) * 2 + kind) * p.n_kv + h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
  return static_cast<const T*>(p.pages) + row * D;
}

// ---------------------------------------------------------------- attention
// out = sum over the tokens t that a query sees of p_t v_t, p = softmax(scale q k_t), in one pass over the keys and values:
// with a reference m near the greatest score so far, l = sum e^(s - m) and O = sum e^(s - m) v, both scaled when m moves.
//
// The rows of a sequence and kv-head are (query, head of the group), query by query, in blocks of 256: two TMEM lane
// blocks of 128, the slots.  A segment is a block of rows of one kv-head over the tokens that its queries see, in
// tiles of 128.  Where a block has more than 128 rows, both slots take every tile (a pair); else the slots take turns at
// the tiles, and their halves of the softmax are joined at the end.  Segments lie on a line, with a gap before each for what its
// begin and end cost, and every CTA takes an equal part of the line, whatever the lengths; what is left of a segment in several
// CTAs goes through the workspace and a second launch joins it.
//
// Roles: eight warps do the softmax, a thread a row; one warp issues the MMAs; one walks the line, tells the others of segments and
// tiles, and brings keys and values by TMA (a box per page) into a ring of 32 KB items.  Per tile and slot: S = Q K^T (tcgen05, fp32 in
// TMEM), the softmax with a lazy reference (O is rescaled only when a row's maximum is 2^8 past it), P in 16 bits over the first half
// of S, O += P V (P from TMEM, V as it lies).  While one slot's MMAs run, the other slot's softmax does.
//
// What bounds it (GB300): 64 queries x 32 heads over 131072 tokens x 8 kv-heads take 109 to 122 us, 4.9 to 4.4 TB/s, where the
// memory alone needs 79 and the same kernel without MMAs and softmax takes 94 to 100: a pair's tile costs 1.9 us of softmax and MMAs in
// turn, 1.5 of memory.  26 queries x 28 heads of 16 sequences over 8192 tokens (f16) 66 us; 37 ragged sequences with capped scores 73
// (61 without the cap's exponential and half a reciprocal a score): a segment's begin and end, some 7 us for queries, first tiles, results;
// 8 queries over 1001 tokens 13.4 us, of which 6 until the first tile is there and 3 the second launch.
//
// With sixteen softmax warps, two threads a row that tell each other maxima and sums, and with waits of the MMA warp out of line (see
// there), 119 us over 131072 tokens against 109 so; with either kept and spills to local memory, whose cache is what 227 KB of shared
// memory leave, more.
constexpr int kTile = 128;
constexpr int kSlotRows = 128;
constexpr int kBlockRows = 2 * kSlotRows;
constexpr int kItem = kTile * D * 2;             // bytes of a tile's keys or values
constexpr int kGroupStep = 2048, kHalfStep = 1024;   // of an item: groups of eight tokens, halves of the dimensions in a group
constexpr int kRing = 5;
constexpr int kInfos = 8;                        // tiles whose pages a softmax warp may still ask for: more than the ring holds
constexpr int kSegs = 4;
constexpr int kSoftmaxThreads = 256;
constexpr int kMmaWarp = 0, kLoadWarp = 1, kSoftmaxWarp = 4;   // (warps 2, 3 idle: a warp reaches the TMEM lanes of its number modulo 4)
constexpr int kTreeThreads = 384;
// What a segment costs beside its tiles, in units of the line.  With a cap a tile of a pair is two units, as the scores bound it; without
// one a tile is one unit, as its copies do.  Measured in us, sequences x drafted tokens over up to so many tokens:
//   capped, gaps (pairs' ones)       5 (6)    8 (8)    4 (4)    6 (8)   pairs of one unit, 3 (4)
//   37 x up to 48 over 4001, ragged   73.5     75.9     77.1     73.2     79.5
//   the same in f16                   74.5     76.3     78.0     73.8     80.5
//   37 x 48 over 1000, all alike      85.0     84.1     85.0     84.1     80.3
//   16 x 26 over 8192 (f16)          102.9    103.0    103.3    102.9    102.3
//   152 x 32 over 64                  74.5     74.9     74.9     74.9     74.4
//   8 x 200 over 3000                 51.9     51.2     52.9     51.3     51.7
//   3 x 16 over 20000                 32.8     33.6     33.0     32.5     32.5
//   not capped, a gap of                 6        8        3        5        7
//   the first of these                61.1     63.4     70.0     62.4     62.9
//   16 x 26 over 8192 (f16)           66.2     68.2     68.6     66.8     66.5
//   8 x 200 over 3000                 41.7     45.0     43.3     42.4     42.3
//   3 x 16 over 20000                 29.8     30.6     30.4     30.1     30.1
//   1 x 64 over 131072               113.8    112.9    115.3    113.8    115.0
// (the other two within 1 %).
constexpr int kTreeGap = 6, kTreeGapCapped = 5, kTreeGapCappedPair = 6;
constexpr int kTreeUnits = 2;                    // of a CTA, at least: every part between a segment's first and last has a tile then
constexpr uint32_t kColS = 0, kColO = 256;       // TMEM: S (and P) of the slots, then O
constexpr size_t kTreeSmem = 2 * kItem + kRing * kItem;
constexpr int kTreePiece = kBlockRows * (D + 2); // floats: sums [256][128], references [256], totals [256]

// Workspace: pieces [2 n_ctas] (CTA c's share begins inside a segment: piece 2 c; ends inside one that it began: 2 c + 1), then per
// CTA two int4 of the segment that it began and did not end: (last CTA with a part of it, or -1: none; kv-head; first row; rows) and
// (the sequence's first query, -, -, -).

using Pos = int64_t;

struct Share {
  Pos each;
  int n_ctas, longer;               // CTAs that get anything; the first of them get one more
  __device__ Pos begin(int c) const { return c * each + min(c, longer); }
  __device__ int cta_of(Pos at) const {
    const Pos big = longer * (each + 1);
    return static_cast<int>(at < big ? quotient(at, each + 1) : longer + quotient(at - big, each));
  }
};

// A CTA's share [x, x_end) of a line, which begins `off` units into sequence b (x == x_end: nothing).
struct Begin {
  Share share;
  Pos x, x_end, off;
  int b;
};
// Measures the line and finds it, for a converged warp.  A lane sums up the same number of sequences each, then as many of the one lane
// in whose sum the share begins, and so on; units(i, tells): of sequence i (tells: flag what does not fit).
template <typename Units>
__device__ __forceinline__ Begin begin_of(int batch, int units_per_cta, Units units) {
  const int lane = threadIdx.x % 32;
  Begin at = {};
  int count = batch;
  for (bool first = true; first || count > 1; first = false) {
    const int per = (count + 31) / 32, from = at.b + lane * per;
    Pos mine = 0;
#pragma unroll 2
    for (int i = from; i < min(from + per, at.b + count); ++i) mine += units(i, first && blockIdx.x == 0);
    Pos upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Pos y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (first) {
      const Pos total = __shfl_sync(0xffffffffu, upto, 31);
      at.share.n_ctas = static_cast<int>(min(static_cast<Pos>(gridDim.x), total / units_per_cta));
      if (static_cast<int>(blockIdx.x) >= at.share.n_ctas) return at;
      at.share.each = quotient(total, static_cast<Pos>(at.share.n_ctas));
      at.share.longer = static_cast<int>(total - at.share.each * at.share.n_ctas);
      at.off = at.x = at.share.begin(blockIdx.x);
      at.x_end = at.share.begin(blockIdx.x + 1);
    }
    const uint32_t past = __ballot_sync(0xffffffffu, upto > at.off);
    if (!past) {                                     // (lengths that changed between two reads of them)
      at.x = at.x_end;
      return at;
    }
    const int lane_of = __ffs(past) - 1;
    at.off -= __shfl_sync(0xffffffffu, upto - mine, lane_of);
    count = min(per, at.b + count - __shfl_sync(0xffffffffu, from, lane_of));
    at.b = __shfl_sync(0xffffffffu, from, lane_of);
  }
  return at;
}

// Tokens that the rows row0 .. row0 + rows see, at most, and the line's units of them.
__device__ __forceinline__ int rows_of(const TreeArgs& a, const Seq& s, int block) {
  return min(kBlockRows, s.n * a.group - block * kBlockRows);
}
__device__ __forceinline__ int seen_to(const TreeArgs& a, const Seq& s, int block) {
  return a.mask ? s.len : min(s.len, s.before() + (block * kBlockRows + rows_of(a, s, block) - 1) / a.group + 1);
}
__device__ __forceinline__ int tiles_to(int tokens) { return tokens / kTile + (tokens % kTile > 0); }
__device__ __forceinline__ int blocks_of(const TreeArgs& a, const Seq& s) {
  const int rows = s.n * a.group;
  return rows / kBlockRows + (rows % kBlockRows > 0);
}
// A tile's units, and a segment's beside its tiles.
template <bool kCap>
__device__ __forceinline__ int weight_of(int rows) {
  return kCap && rows > kSlotRows ? 2 : 1;
}
template <bool kCap>
__device__ __forceinline__ int gap_of(int rows) {
  return !kCap ? kTreeGap : rows > kSlotRows ? kTreeGapCappedPair : kTreeGapCapped;
}
template <bool kCap>
__device__ __forceinline__ Pos units_of(const TreeArgs& a, const Seq& s) {
  const int blocks = blocks_of(a, s);
  auto units = [&](int tokens, int rows) { return static_cast<Pos>(tiles_to(tokens)) * weight_of<kCap>(rows) + gap_of<kCap>(rows); };
  Pos sum = 0;
  if (a.mask) {                                      // (all blocks but the last one are full)
    if (blocks > 0) sum = (blocks - 1) * units(s.len, kBlockRows) + units(s.len, rows_of(a, s, blocks - 1));
  } else {
    for (int i = 0; i < blocks; ++i) sum += units(seen_to(a, s, i), rows_of(a, s, i));
  }
  return sum * a.pool.n_kv;
}

// What the walking warp tells of a CTA's part of a segment: rows row0 .. row0 + rows of sequence b's n queries in kv-head h, its
// tiles t0 .. t1 of `tiles`; rows == 0: there is no more.
struct __align__(16) Segment {
  int b, h, i0, n;
  int before, hi, row0, rows;
  int t0, t1, tiles, last_cta;      // last_cta: the last CTA with a part of it
};

template <typename T>
struct Half16;
template <>
struct Half16<__nv_bfloat16> {
  static constexpr uint32_t kFormat = 1;
  static constexpr float kShift = 0.0f;          // log2 of the scale on the weights
  static constexpr float kLag = 8.0f;            // log2 of how far a maximum may be past the reference
  static constexpr uint32_t kLeast = 0x0D800D80u;  // 2^-100, twice
  // two weights, rounded, each at least that of `least`
  static __device__ __forceinline__ uint32_t weights(float p, float q, uint32_t least) {
    const __nv_bfloat162 h = __hmax2_nan(__floats2bfloat162_rn(p, q), *reinterpret_cast<const __nv_bfloat162*>(&least));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <>
struct Half16<__half> {
  static constexpr uint32_t kFormat = 0;
  // Weights up to 2^8 of the reference times 2^7 are below the largest number; 11 bits are left of one of 2^-21 of it, and the
  // least is 2^-31: a tail of 131072 such tokens is 2^-14 of a result, an eighth of its rounding.  A lag of 5 (2^10) would leave
  // 2^-34, but rescales more often: 74 us for 66 (16 x 26 queries of 28 heads over 8192 tokens).  So a part of a segment that has
  // more tokens has a lag that is as much smaller, down to 1 for 2^24 tokens, where the least is 2^-38.
  static constexpr float kShift = 7.0f, kLag = 8.0f;
  static constexpr int kLagTiles = 10, kLagMore = 7;       // log2 of the tiles that kLag is for; that it gives up at most
  static constexpr uint32_t kLeast = 0x00010001u;  // 2^-24, twice
  static __device__ __forceinline__ uint32_t weights(float p, float q, uint32_t least) {
    const __half2 h = __hmax2_nan(__floats2half2_rn(p, q), *reinterpret_cast<const __half2*>(&least));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// Instruction descriptor: 16-bit operands of one type, fp32 sums, 128 x 128; values come with their dimensions along the rows
// in memory (the transposed form of operand B).
template <typename T>
__host__ __device__ constexpr uint32_t tree_idesc(bool values) {
  return (1u << 4) | (Half16<T>::kFormat << 7) | (Half16<T>::kFormat << 10) | (values ? 1u << 16 : 0u) | (16u << 17) | (8u << 24);
}
// Shared-memory descriptor of rows of 128 bytes, swizzled: `lead`, `stride`: bytes between blocks along the rows' direction
// and between groups of eight rows.
__device__ __forceinline__ uint64_t smem_desc(uint32_t at, uint32_t lead, uint32_t stride) {
  return static_cast<uint64_t>((at & 0x3FFFFu) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 |
         static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// Caps up to here come from cap - 2 cap / (e^(2 s / cap) + 1), whose error is 2^-21 of the cap (3.1e-5 at this one), past it from a
// form whose error is 4e-7 of the score (37 ragged sequences 73 us with the first, 77 with the second; weights of 32 queries over
// 3 x 32768 tokens 70 and 66).  They are kernels of their own: both in one cost the first 4 %.
constexpr float kNearCap = 64.0f;
constexpr int kNone = 0, kNear = 1, kFar = 2;
int cap_kind(float cap) { return !(cap > 0.0f) ? kNone : cap <= kNearCap ? kNear : kFar; }

// Bits j .. j + 127 of what query i of the sequence sees of its drafted tokens (ones before them, zeros behind).
__device__ __forceinline__ void seen_bits(const TreeArgs& a, const Segment& s, int i, int j, uint32_t (&vis)[4]) {
#pragma unroll
  for (int y = 0; y < 4; ++y) vis[y] = 0xFFFFFFFFu;
  if (j <= -128) return;
  const int left = (a.mask ? s.n : i + 1) - j;       // drafted tokens from there on are not seen
  if (a.mask && left > 0) {
    const int k = j >> 5;                            // (down)
    const int32_t* row = a.mask + static_cast<int64_t>(s.i0 + i) * a.mask_words + k;
    uint32_t w[5];
#pragma unroll
    for (int y = 0; y < 5; ++y) w[y] = k + y < 0 ? 0xFFFFFFFFu : k + y < a.mask_words ? row[y] : 0u;
#pragma unroll
    for (int y = 0; y < 4; ++y) vis[y] = __funnelshift_r(w[y], w[y + 1], j & 31);
  }
#pragma unroll
  for (int y = 0; y < 4; ++y)
    if (left < 32 * y + 32) vis[y] = left <= 32 * y ? 0u : vis[y] & ((1u << (left - 32 * y)) - 1u);
}

// Bit 15 or 31 is set where the lower or upper of two 16-bit values has an exponent of all ones (infinite, or NaN).
__device__ __forceinline__ uint32_t not_finite(uint32_t w, uint32_t exponent, uint32_t least) { return (w & exponent) + least; }
__device__ __forceinline__ float least_of(float a, float b) {   // NaN where one is
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^x for a factor on sums that may hold an infinite value: at least the least number above 0, so that the value stays infinite and
// does not turn into NaN.  (Finite sums lose 2^-126 and more: next to nothing is left of them either way.)
__device__ __forceinline__ float factor_of(float x) {
  const float f = exp2_of(x), least = __uint_as_float(1u);
  return f < least ? least : f;                      // (NaN stays)
}

// Named barriers: of all softmax threads, of a slot's.
__device__ __forceinline__ void both_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void slot_sync(int slot) { asm volatile("bar.sync %0, 128;" ::"r"(2 + slot) : "memory"); }
// Whether `ok` holds for all softmax threads, which meet here.
__device__ __forceinline__ bool both_agree(bool ok) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(all)
               : "r"(static_cast<uint32_t>(ok))
               : "memory");
  return all != 0;
}

struct TreeSync {
  uint64_t kv_full[kRing], kv_free[kRing], s_full[2], p_full[2], o_full[2], q_full, seg_full[kSegs], seg_free[kSegs],
      info_full[kInfos];
  Segment seg[kSegs];
  uint32_t bad[kInfos];             // a tile's groups of eight tokens whose page is none of the pool's
  uint32_t special[2][3][4];        // [slot][turn]: tokens of a tile with infinities or NaN among their values
  uint32_t tmem;
  int abort;
};

// The long way of a wait, out of line: the code of a call that is short is fetched once, at some 1 ns a byte.
__device__ __noinline__ bool wait_long(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* err) {
  if (ptx::mbar_wait_bounded(bar, parity, abort_flag)) return true;
  if (!*abort_flag) raise(err, kTimeout);
  *abort_flag = 1;
  return false;
}

template <typename T, int kCap>
__global__ void __launch_bounds__(kTreeThreads, 1)
    aatc_paged_tree_kernel(const TreeArgs a, const __grid_constant__ CUtensorMap map) {
  extern __shared__ __align__(1024) unsigned char smem[];        // queries of the slots, then the ring
  __shared__ TreeSync sy;
  const Pool& p = a.pool;
  const int tid = threadIdx.x, warp = ptx::warp_uniform(tid / 32), lane = tid % 32;
  unsigned char* ring = smem + 2 * kItem;
  int4* desc = reinterpret_cast<int4*>(a.ws + static_cast<size_t>(gridDim.x) * 2 * kTreePiece);
  volatile int* abort_flag = &sy.abort;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return ptx::mbar_try_wait(bar, parity) || wait_long(bar, parity, abort_flag, p.err); };
  constexpr int kBarriers = 2 * kRing + 7 + 2 * kSegs + kInfos;
  static_assert(offsetof(TreeSync, kv_full) == 0 && offsetof(TreeSync, info_full) == (kBarriers - kInfos) * sizeof(uint64_t),
                "every barrier is set up");
  if (warp == kLoadWarp) {
    for (int i = lane; i < kBarriers; i += 32) {
      uint64_t* bar = sy.kv_full + i;
      ptx::mbar_init(bar, bar >= sy.p_full && bar < sy.p_full + 2 ? 4
                          : bar == &sy.q_full ? kSoftmaxThreads / 32
                          : bar >= sy.seg_free && bar < sy.seg_free + kSegs ? kSoftmaxThreads / 32 + 1 : 1);
    }
    if (lane == 0) {
      sy.abort = 0;
      ptx::prefetch_tmap(&map);
    }
    ptx::fence_mbar_init();
  }
  if (warp == 2) {
    ptx::tmem_alloc(&sy.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const uint32_t tmem = sy.tmem;

  if (warp == kLoadWarp) {
    if (lane == 0) desc[2 * blockIdx.x] = make_int4(-1, 0, 0, 0);
    Begin at = begin_of(a.batch, kTreeUnits, [&](int i, bool tells) { return units_of<kCap != kNone>(a, seq_of(a, i, tells)); });
    Pos &x = at.x, &off = at.off;
    const Pos x_end = at.x_end;
    int& b = at.b;
    const Share& share = at.share;
    // ---- the walk: segments and tiles of this CTA's share
    int seg_i = 0, item = 0, tile_i = 0;
    uint32_t free_round = 0;                         // bit s: parity of the next wait for seg_free[s]
    auto stopped = [&]() { return __any_sync(0xffffffffu, *abort_flag) != 0; };
    auto tell = [&](const Segment& s) {
      const int at = seg_i % kSegs;
      if (seg_i >= kSegs) {
        wait(&sy.seg_free[at], free_round >> at & 1u);
        free_round ^= 1u << at;
      }
      if (stopped()) return;
      if (lane == 0) {
        sy.seg[at] = s;
        ptx::mbar_arrive(&sy.seg_full[at]);
      }
      ++seg_i;
      __syncwarp();
    };
    Seq s = {};
    if (x < x_end) s = seq_of(a, b, false);
    int block = 0, h = 0, hi = 0, tiles = 0, each = 1, gap = 0;  // (each: units of a tile)
    Pos units = 0;                                               // a segment's
    auto set_block = [&]() {
      hi = seen_to(a, s, block);
      tiles = tiles_to(hi);
      each = weight_of<kCap != kNone>(rows_of(a, s, block));
      gap = gap_of<kCap != kNone>(rows_of(a, s, block));
      units = static_cast<Pos>(tiles) * each + gap;
    };
    int n_blocks = blocks_of(a, s);
    if (n_blocks > 0) set_block();
    while (block + 1 < n_blocks && off >= units * p.n_kv) {
      off -= units * p.n_kv;
      ++block;
      set_block();
    }
    while (h + 1 < p.n_kv && off >= units) {
      off -= units;
      ++h;
    }
    // a tile is the CTA's in whose share it begins: x is where the next one does
    int t = off <= gap ? 0 : static_cast<int>((off - gap + each - 1) / each);
    x += gap + static_cast<Pos>(t) * each - off;
    const int shift = p.page_shift, page = 1 << shift;
    const int rows_box = min(page, kTile), n_boxes = kTile / rows_box;           // lane i brings box i of a tile
    const uint32_t box_bytes = rows_box * D * 2;
    while (n_blocks > 0 && x < x_end && b < a.batch) {
      const int t0 = t, t1 = static_cast<int>(min(static_cast<Pos>(tiles), t + (x_end - x + each - 1) / each));
      Segment g;
      g.b = b;
      g.h = h;
      g.i0 = s.i0;
      g.n = s.n;
      g.before = s.before();
      g.hi = hi;
      g.row0 = block * kBlockRows;
      g.rows = rows_of(a, s, block);
      g.t0 = t0;
      g.t1 = t1;
      g.tiles = tiles;
      g.last_cta = t1 < tiles ? min(share.cta_of(x + static_cast<Pos>(tiles - 1 - t) * each), share.n_ctas - 1) : blockIdx.x;
      if (t < t1) tell(g);                           // (none where the share begins within the last tile)
      const int32_t* row = p.table + static_cast<int64_t>(b) * p.table_stride;
      auto id_of = [&](int tile) {                   // the page of this lane's box
        const int tok = tile * kTile + lane * rows_box;
        return lane < n_boxes && tok < hi ? row[tok >> shift] : 0;
      };
      int id = t < t1 ? id_of(t) : 0;
      for (; t < t1; ++t) {
        const int tok = t * kTile + lane * rows_box;
        const bool live = lane < n_boxes && tok < hi, ok = live && static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages);
        const int now = id;
        if (t + 1 < t1) id = id_of(t + 1);
        if (live && !ok) raise(p.err, kBadPage);
        const uint32_t n_ok = __popc(__ballot_sync(0xffffffffu, ok));
        uint32_t bad = live && !ok ? (rows_box >= kTile ? 0xFFFFu : ((1u << rows_box / 8) - 1u) << lane * (rows_box / 8)) : 0u;
        bad = __reduce_or_sync(0xffffffffu, bad);
        if (lane == 0) {
          sy.bad[tile_i % kInfos] = bad;
          ptx::mbar_arrive(&sy.info_full[tile_i % kInfos]);
        }
        ++tile_i;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind, ++item) {
          const int at = item % kRing;
          if (item >= kRing) wait(&sy.kv_free[at], (item / kRing - 1) & 1);
          if (stopped()) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(&sy.kv_full[at], n_ok * box_bytes);
          __syncwarp();
          if (ok)
            ptx::tma_load_5d(ring + at * kItem + lane * box_bytes, &map, &sy.kv_full[at], 0, 0, 0,
                             (((kind * p.n_kv + h) << shift) + (tok & (page - 1))) / 8, now);
        }
        if (stopped()) break;
      }
      if (stopped()) break;
      x += static_cast<Pos>(t1 - t0) * each;
      if (t1 < tiles) break;                         // (the share ends inside)
      t = 0;
      if (++h == p.n_kv) {
        h = 0;
        if (++block == n_blocks) {
          block = 0;
          do {
            ++b;
            if (b >= a.batch) break;
            s = seq_of(a, b, false);
            n_blocks = blocks_of(a, s);
          } while (n_blocks == 0);
          if (b >= a.batch) break;
        }
        set_block();
      }
      x += gap;                                      // (the next segment's)
    }
    Segment none = {};
    tell(none);
  } else if (warp == kMmaWarp) {
    // ---- MMAs, issued by the converged warp
    auto wait_here = [&](uint64_t* bar, uint32_t parity) {     // (not a call: over one nothing stays in uniform registers)
      if (ptx::mbar_wait_bounded(bar, parity, abort_flag)) return true;
      if (!*abort_flag) raise(p.err, kTimeout);
      *abort_flag = 1;
      return false;
    };
    const uint32_t el = ptx::elect_one(), tm = __reduce_max_sync(0xffffffffu, tmem);
    const uint64_t q_desc = smem_desc(ptx::smem_u32(smem), 16, 1024);
    const uint64_t k_desc = smem_desc(ptx::smem_u32(ring), 16, kGroupStep);
    const uint64_t v_desc = smem_desc(ptx::smem_u32(ring), kHalfStep, kGroupStep);
    // Places in the ring and parities by counting, and conditions by votes: then what the MMAs take stays in uniform registers, else
    // it is moved there for each of them (some 90 cycles an MMA, where it computes for 64).
    int k_at = 0, v_at = 1;                          // the next keys' and values' places in the ring
    uint32_t k_parity = 0, v_parity = 0, p_parity = 0;
    auto ahead = [](int& at, uint32_t& parity) {     // two items on
      at += 2;
      if (at >= kRing) {
        at -= kRing;
        parity ^= 1;
      }
    };
    for (int seg_i = 0;; ++seg_i) {
      const bool there = wait_here(&sy.seg_full[seg_i % kSegs], seg_i / kSegs & 1) && !*abort_flag;
      if (!__all_sync(0xffffffffu, there)) break;
      const Segment& g = sy.seg[seg_i % kSegs];
      const int rows = g.rows, n_tiles = g.t1 - g.t0;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sy.seg_free[seg_i % kSegs]);
      if (__any_sync(0xffffffffu, rows == 0)) break;
      const bool pair = __any_sync(0xffffffffu, rows > kSlotRows);
      wait_here(&sy.q_full, seg_i & 1);
      ptx::tc_fence_after();
      // step 2 t + slot of a pair, or t: tile t in slot t % 2
      const int steps = pair ? 2 * n_tiles : n_tiles;
      for (int step = -2; __any_sync(0xffffffffu, step < steps); ++step) {
        const uint32_t slot = step & 1, cols = 128 * slot;
        const bool last_use = !pair || slot;         // of the keys or values
        if (step >= 0) {                             // O += P V
          wait_here(&sy.kv_full[v_at], v_parity);
          wait_here(&sy.p_full[slot], p_parity >> slot & 1u);
          p_parity ^= 1u << slot;
          ptx::tc_fence_after();
          const uint64_t vd = v_desc + static_cast<uint64_t>(v_at) * (kItem >> 4);
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            ptx::umma_f16_ta_w(tm + kColO + cols, tm + kColS + cols + 8 * kk, vd + ((2 * kk * kGroupStep) >> 4), tree_idesc<T>(true), 1u, el);
          if (last_use) {
            ptx::umma_commit_w(&sy.kv_free[v_at], el);
            ahead(v_at, v_parity);
          }
          if (__any_sync(0xffffffffu, step + 2 >= steps)) ptx::umma_commit_w(&sy.o_full[slot], el);
        }
        if (__any_sync(0xffffffffu, step + 2 < steps)) {         // S = Q K^T of the step after the next
          wait_here(&sy.kv_full[k_at], k_parity);
          ptx::tc_fence_after();
          const uint64_t qd = q_desc + (pair && slot ? kItem >> 4 : 0), kd = k_desc + static_cast<uint64_t>(k_at) * (kItem >> 4);
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            ptx::umma_bf16_w(tm + kColS + cols, qd + (((kk >> 2) * (kItem / 2) + (kk & 3) * 32) >> 4),
                             kd + (((kk >> 2) * kHalfStep + (kk & 3) * 32) >> 4), tree_idesc<T>(false), kk > 0 ? 1u : 0u, el);
          ptx::umma_commit_w(&sy.s_full[slot], el);
          if (last_use) {
            ptx::umma_commit_w(&sy.kv_free[k_at], el);
            ahead(k_at, k_parity);
          }
        }
      }
    }
  } else if (warp >= kSoftmaxWarp) {
    // ---- softmax: warp w has rows 32 (w % 4) .. + 31 of slot w / 4, a thread a row
    const int tid = threadIdx.x - 32 * kSoftmaxWarp, warp = ptx::warp_uniform(tid / 32), slot = warp / 4, r = tid % kSlotRows;
    const uint32_t lanes = static_cast<uint32_t>(32 * (warp % 4)) << 16;
    const uint32_t col_s = tmem + lanes + kColS + 128 * slot, col_o = tmem + lanes + kColO;
    // scores after c, which is above 0, ascend with S: other scales are done to S first
    const bool in_place = !(a.scale > 0.0f);
    const float c = in_place ? 1.0f : a.scale * kLog2e;
    const uint64_t c2 = ptx::f2_pack(c, c);
    const float cap_in = (kCap ? 2.0f * a.scale / a.cap : a.scale) * kLog2e, cap_out = a.cap * kLog2e;
    constexpr uint32_t kExponent = Half16<T>::kFormat ? 0x7F807F80u : 0x7C007C00u, kOne = Half16<T>::kFormat ? 0x00800080u : 0x04000400u;
    const float far_in = kCap ? a.scale / a.cap : 0.0f, unit = a.scale * kLog2e;
    // Near caps: cap tanh y = cap - 2 cap / (e^(2 y) + 1), two scores with one reciprocal (e^(2 y) up to 2^60, where the cap is reached).
    auto capped_two = [&](uint32_t& s0, uint32_t& s1) {
      const float z0 = exp2_of(least_of(__uint_as_float(s0) * cap_in, 60.0f)) + 1.0f, z1 = exp2_of(least_of(__uint_as_float(s1) * cap_in, 60.0f)) + 1.0f;
      const float f = -2.0f * cap_out * reciprocal(z0 * z1);
      s0 = __float_as_uint(fmaf(f, z1, cap_out));
      s1 = __float_as_uint(fmaf(f, z0, cap_out));
    };
    int item0 = 0, tile0 = 0;
    uint32_t s_parity = 0, o_parity = 0;             // (of the slot's S; bit i: of slot i's O)
    bool there = wait(&sy.seg_full[0], 0);
    for (int seg_i = 0;; ++seg_i) {
      // (every thread is past the last segment's results)
      if (!both_agree(there && !*abort_flag)) break;
      const Segment& g = sy.seg[seg_i % kSegs];      // (read where it is needed)
      if (g.rows == 0) break;
      const bool pair = g.rows > kSlotRows;
      const int n_tiles = g.t1 - g.t0;
      // ---- queries to shared memory (zeros behind the last row), O = 0
      {
        const int piece = tid % 16, by = 16 / a.group, by_head = 16 - by * a.group;
        int query = quotient(g.row0 + tid / 16, a.group), head = g.row0 + tid / 16 - query * a.group;
#pragma unroll 1
        for (int row = tid / 16; row < (pair ? kBlockRows : kSlotRows); row += 16) {
          const bool in = row < g.rows;
          const T* from = static_cast<const T*>(a.q.x);
          if (in) from += (g.i0 + query) * a.q.token_stride + (g.h * a.group + head) * a.q.head_stride + 8 * piece;
          ptx::cp_async_16(smem + row / kSlotRows * kItem + piece / 8 * (kItem / 2) + row % kSlotRows * 128 + ((piece % 8) ^ (row % 8)) * 16,
                           from, in ? 16 : 0);
          query += by;
          head += by_head;
          if (head >= a.group) {
            head -= a.group;
            ++query;
          }
        }
        uint32_t zero[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) ptx::tmem_st16(col_o + 128 * slot + 16 * i, zero);
        ptx::tmem_wait_st();
        ptx::cp_async_wait_all();
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sy.q_full);
      }
      const int my_row = pair ? slot * kSlotRows + r : r;
      const int node = min(quotient(g.row0 + min(my_row, g.rows - 1), a.group), g.n - 1);
      const bool idle = my_row - lane >= g.rows;
      float m = -INFINITY;
      uint64_t l2 = ptx::f2_pack(0.0f, 0.0f);
      bool first_step = true;
      float shift = Half16<T>::kShift, lag = Half16<T>::kLag;
      if constexpr (Half16<T>::kFormat == 0) {
        const int more = min(max(32 - __clz(n_tiles - 1) - Half16<T>::kLagTiles, 0), Half16<T>::kLagMore);
        shift += more;
        lag -= more;
      }
      auto rescale = [&](float f) {                  // O *= f (it is complete up to the tile before: its MMAs came before those of S)
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          uint32_t o[16];
          ptx::tmem_ld_16raw(col_o + 128 * slot + 16 * i, o);
          ptx::tmem_ld_wait();
          ptx::tmem_regs_ready(o);
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
          ptx::tmem_st16(col_o + 128 * slot + 16 * i, o);
        }
      };
      for (int k = pair ? 0 : slot; k < n_tiles; k += pair ? 1 : 2) {
        const int T0 = (g.t0 + k) * kTile, info = (tile0 + k) % kInfos;
        wait(&sy.info_full[info], (tile0 + k) / kInfos & 1);
        const uint32_t bad = sy.bad[info];
        const bool edge = g.before - T0 < kTile || bad;      // (T0 + kTile may be 2^31)
        // Tiles that are under way together have turns of their own: a slot that begins a tile is done with the one before the last, but
        // of a pair the other slot, which reads what the first one found, may have come to that one only.
        const int turn = pair ? (tile0 + k) % 3 : (tile0 + k) / 2 & 1;
        uint32_t vis[4] = {0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu};   // which of the tile's tokens the row sees
        if (edge) {
          seen_bits(a, g, node, T0 - g.before, vis);
          if (bad) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (bad >> j & 1u) vis[j / 4] &= ~(0xFFu << 8 * (j % 4));
          }
          // values of tokens that nobody sees, and those with infinities or NaN: their weight may be 0, but 0 x NaN is not;
          // both are cleared, and the latter's products summed apart
          if (!pair || slot == 0) {
            const int it = item0 + 2 * k + 1, tok = T0 + r;
            wait(&sy.kv_full[it % kRing], it / kRing & 1);
            unsigned char* v = ring + it % kRing * kItem + r / 8 * kGroupStep + r % 8 * 128;
            const bool dead = tok >= g.hi || (bad >> r / 8 & 1u);
            bool clear = dead;
            if (!dead) {
              uint32_t found = 0;
#pragma unroll 4
              for (int i = 0; i < 16; ++i) {
                const uint4 y = *reinterpret_cast<const uint4*>(v + i / 8 * kHalfStep + ((i % 8) ^ (r % 8)) * 16);
                found |= not_finite(y.x, kExponent, kOne) | not_finite(y.y, kExponent, kOne) | not_finite(y.z, kExponent, kOne) |
                         not_finite(y.w, kExponent, kOne);
              }
              clear = found & 0x80008000u;
            }
            if (clear) {
#pragma unroll 1
              for (int i = 0; i < 16; ++i) *reinterpret_cast<uint4*>(v + i / 8 * kHalfStep + i % 8 * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            const uint32_t which = __ballot_sync(0xffffffffu, clear && !dead);
            if (lane == 0) sy.special[slot][turn][warp % 4] = which;
            ptx::fence_proxy_async_smem();
          }
          if (pair) both_sync();
          else slot_sync(slot);
        }
        wait(&sy.s_full[slot], s_parity);
        s_parity ^= 1;
        ptx::tc_fence_after();
        // Most tiles: the weights with the last reference straight away, in registers; they hold unless a maximum is far past it.
        // (A warp without rows leaves its lanes of P as they are: they come into no other row.)
        bool done = idle;
        constexpr int kN = 32;                       // scores at once
        auto greatest = [](const uint32_t (&x)[kN]) {
          float t[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) t[j] = fmaxf(__uint_as_float(x[j]), __uint_as_float(x[j + 4]));
#pragma unroll
          for (int j = 8; j < kN; j += 8)
#pragma unroll
            for (int y = 0; y < 4; ++y) t[y] = ptx::fmax3(t[y], __uint_as_float(x[j + y]), __uint_as_float(x[j + y + 4]));
          return fmaxf(ptx::fmax3(t[0], t[1], t[2]), t[3]);
        };
        if (idle) {
          // (nothing)
        } else if constexpr (kCap) {
          // 32 scores at once, each with the reference as it is by then: capped ones cost too much to be made twice (37 ragged sequences
          // 73 us; 81 with all 128 in registers as below).  References are whole, so that the weights of the tile that are there
          // already move with one exactly (down to the type's least).  With 0 for a reference, which bf16 has the range for up to a
          // cap of 69, it is 69 us, but values of 2^29 overflow next to scores at that cap.
          const uint32_t least = edge ? 0u : Half16<T>::kLeast;
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            uint32_t x[32], w[16];
            ptx::tmem_ld_32raw(col_s + 32 * i, x);
            const uint32_t see = i < 2 ? (i == 0 ? vis[0] : vis[1]) : (i == 2 ? vis[2] : vis[3]);
            ptx::tmem_ld_wait();
            ptx::tmem_regs_ready(x);
            if (edge) {                              // (what is not seen may be NaN, and shares a reciprocal)
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(see >> j & 1u)) x[j] = 0u;
            }
            if constexpr (kCap == kNear) {
#pragma unroll
              for (int j = 0; j < 32; j += 2) capped_two(x[j], x[j + 1]);
            } else {
              cap_far(x, unit, far_in, cap_out);
            }
            if (edge) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(see >> j & 1u)) x[j] = 0xFF800000u;
            }
            const float top = greatest(x);
            uint64_t sum;
#pragma unroll 1
            for (;;) {                               // (twice where a score is far past the reference)
              const float base = m == -INFINITY ? 0.0f : shift - m;
              const uint64_t base2 = ptx::f2_pack(base, base);
              sum = l2;
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                float e0, e1;
                ptx::f2_unpack(ptx::f2_add(ptx::f2_pack(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), base2), e0, e1);
                e0 = exp2_of(e0);
                e1 = exp2_of(e1);
                sum = ptx::f2_add(sum, ptx::f2_pack(e0, e1));
                w[j / 2] = Half16<T>::weights(e0, e1, least);
              }
              const bool need = top > m + lag;
              if (!__any_sync(0xffffffffu, need)) break;
              const float next = need ? floorf(top) : m, f = need ? factor_of(m - next) : 1.0f;
              if (!first_step) rescale(f);
              ptx::tmem_wait_st();
#pragma unroll 1
              for (int e = 0; e < i; ++e) {
                ptx::tmem_ld_16raw(col_s + 16 * e, w);
                ptx::tmem_ld_wait();
                ptx::tmem_regs_ready(w);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  const float2 two = widen(T(), w[j]);
                  w[j] = Half16<T>::weights(two.x * f, two.y * f, least);
                }
                ptx::tmem_st16(col_s + 16 * e, w);
              }
              l2 = ptx::f2_mul(l2, ptx::f2_pack(f, f));
              m = next;
            }
            l2 = sum;
            ptx::tmem_st16(col_s + 16 * i, w);
          }
          ptx::tmem_wait_st();
          first_step = false;
          done = true;
        } else if (!first_step && !edge && !in_place) {
          uint32_t w[4][16];
          float top = -INFINITY;
          const float base = m == -INFINITY ? 0.0f : shift - m;
          const uint64_t base2 = ptx::f2_pack(base, base);
          uint64_t sum = l2;
#pragma unroll
          for (int i = 0; i < kTile / kN; ++i) {
            uint32_t x[kN];
            ptx::tmem_ld_32raw(col_s + kN * i, x);
            ptx::tmem_ld_wait();
            ptx::tmem_regs_ready(x);
            top = fmaxf(top, greatest(x));
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
              float e0, e1;
              ptx::f2_unpack(ptx::f2_fma(ptx::f2_pack(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), c2, base2), e0, e1);
              e0 = exp2_of(e0);
              e1 = exp2_of(e1);
              sum = ptx::f2_add(sum, ptx::f2_pack(e0, e1));
              w[kN * i / 32][kN * i % 32 / 2 + j / 2] = Half16<T>::weights(e0, e1, Half16<T>::kLeast);
            }
          }
          if (!__any_sync(0xffffffffu, top * c > m + lag)) {
            l2 = sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) ptx::tmem_st16(col_s + 16 * i, w[i]);
            ptx::tmem_wait_st();
            done = true;
          }
        }
        if (!kCap && !done) {
          float top = -INFINITY;
#pragma unroll 1
          for (int i = 0; i < kTile / kN; ++i) {
            uint32_t x[kN];
            ptx::tmem_ld_32raw(col_s + kN * i, x);
            ptx::tmem_ld_wait();
            ptx::tmem_regs_ready(x);
            if (in_place) {
#pragma unroll
              for (int j = 0; j < kN; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * cap_in);
            }
            if (edge) {
              const int word = kN * i / 32;
              const uint32_t see = (word < 2 ? (word == 0 ? vis[0] : vis[1]) : (word == 2 ? vis[2] : vis[3])) >> kN * i % 32;
#pragma unroll
              for (int j = 0; j < kN; ++j)
                if (!(see >> j & 1u)) x[j] = 0xFF800000u;
            }
            if (edge || in_place) {
              ptx::tmem_st32(col_s + kN * i, x);
            }
            top = fmaxf(top, greatest(x));
          }
          ptx::tmem_wait_st();
          top *= c;
          const bool need = top > m + lag;
          if (__any_sync(0xffffffffu, need)) {
            const float f = need ? factor_of(m - top) : 1.0f;
            if (!first_step) rescale(f);
            l2 = ptx::f2_mul(l2, ptx::f2_pack(f, f));
            if (need) m = top;
          }
          first_step = false;
          const float base = m == -INFINITY ? 0.0f : shift - m;
          const uint64_t base2 = ptx::f2_pack(base, base);
          const uint32_t least = edge ? 0u : Half16<T>::kLeast;     // where all tokens are seen none is 0: times infinity it would be NaN
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            uint32_t x[16], w[8];
            ptx::tmem_ld_16raw(col_s + 16 * i, x);
            ptx::tmem_ld_wait();
            ptx::tmem_regs_ready(x);
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              float e0, e1;
              ptx::f2_unpack(ptx::f2_fma(ptx::f2_pack(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), c2, base2), e0, e1);
              e0 = exp2_of(e0);
              e1 = exp2_of(e1);
              l2 = ptx::f2_add(l2, ptx::f2_pack(e0, e1));
              w[j / 2] = Half16<T>::weights(e0, e1, least);
            }
            ptx::tmem_st8(col_s + 8 * i, w);
          }
          ptx::tmem_wait_st();
        }
        if (edge && !idle) {
          const uint32_t* some = sy.special[pair ? 0 : slot][turn];
          if (some[0] | some[1] | some[2] | some[3]) {
            // (rare) O += p v of tokens whose values were cleared, in the rows that see them
#pragma unroll 1
            for (int j = 0; j < kTile; ++j) {
              if (!(some[j / 32] >> j % 32 & 1u)) continue;
              uint32_t w2;
              ptx::tmem_ld_1raw(col_s + j / 2, w2);
              ptx::tmem_ld_wait();
              asm volatile("" : "+r"(w2)::"memory");
              const float2 two = widen(T(), w2);
              const float w = fmaxf(j % 2 ? two.y : two.x, 7.8886e-31f);         // (2^-100: not 0 where it is seen)
              const Seq s = {g.i0, g.n, g.before + g.n};
              const bool seen = sees(a, s, node, T0 + j);
              const T* v = token_at<T>(p, g.b, g.h, 1, T0 + j);
#pragma unroll 1
              for (int i = 0; i < D; i += 16) {
                uint32_t o[16];
                ptx::tmem_ld_16raw(col_o + 128 * slot + i, o);
                ptx::tmem_ld_wait();
                ptx::tmem_regs_ready(o);
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                  const float with = fmaf(w, v ? static_cast<float>(v[i + y]) : 0.0f, __uint_as_float(o[y]));
                  if (seen) o[y] = __float_as_uint(with);
                }
                ptx::tmem_st16(col_o + 128 * slot + i, o);
                ptx::tmem_wait_st();
              }
            }
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sy.p_full[slot]);
      }
      item0 += 2 * n_tiles;
      tile0 += n_tiles;
      // ---- the next segment's queries and masks come to L2 while this one ends
      there = wait(&sy.seg_full[(seg_i + 1) % kSegs], (seg_i + 1) / kSegs & 1);
      if (there) {
        const Segment& next = sy.seg[(seg_i + 1) % kSegs];
        if (tid < next.rows) {
          const int R = next.row0 + tid, query = quotient(R, a.group), head = next.h * a.group + R - query * a.group;
          const T* from = static_cast<const T*>(a.q.x) + (next.i0 + query) * a.q.token_stride + head * a.q.head_stride;
          asm volatile("prefetch.global.L2 [%0];" ::"l"(from));
          asm volatile("prefetch.global.L2 [%0];" ::"l"(from + 64));
          if (a.mask) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.mask + static_cast<int64_t>(next.i0 + query) * a.mask_words));
        }
      }
      // ---- results: in a pair a slot's own rows; else both slots' parts of the softmax, half of the dimensions by each
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (pair || i < n_tiles) {
          wait(&sy.o_full[i], o_parity >> i & 1u);
          o_parity ^= 1u << i;
        }
      }
      ptx::tc_fence_after();
      float l, l_hi, f0 = 1.0f, f1 = 0.0f;
      ptx::f2_unpack(l2, l, l_hi);
      l += l_hi;
      if (l != l) m = INFINITY;                      // (NaN among the scores: also where there is no other, and m would be -infinity)
      if (!pair) {
        float2* ml = reinterpret_cast<float2*>(smem + kItem);    // (the second slot's queries, which nobody reads) [slot][row]
        ml[slot * kSlotRows + r] = make_float2(m, l);
        both_sync();
        const float2 of0 = ml[r], of1 = ml[kSlotRows + r];
        const float best = fmaxf(of0.x, of1.x), base = best == -INFINITY ? 0.0f : best;
        f0 = of0.y == 0.0f ? 0.0f : factor_of(of0.x - base);     // (a sum of 0: a part of nothing)
        f1 = of1.y == 0.0f ? 0.0f : factor_of(of1.x - base);
        l = fmaf(of0.y, f0, of1.y * f1);
        m = best;
      }
      const bool whole = g.t0 == 0 && g.t1 == g.tiles, begins = g.t0 == 0;
      const float m_out = m == -INFINITY ? -INFINITY : m - shift;
      const bool in = my_row < g.rows;
      const int R = g.row0 + my_row, query = in ? quotient(R, a.group) : 0, head = g.h * a.group + R - query * a.group;
      const int64_t out_row = static_cast<int64_t>(g.i0 + query) * a.n_q + head;
      float* piece = a.ws + (static_cast<size_t>(blockIdx.x) * 2 + begins) * kTreePiece;
      const float inv = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
      // A warp's rows of so many dimensions go through shared memory (where the queries were), so that neighbouring lanes write
      // neighbouring pieces: 256 or 128 bytes of a row, their 16-byte pieces permuted by the row's number.
      const int dims = (pair ? D : D / 2) / (whole ? 1 : 2), pieces = dims * (whole ? 2 : 4) / 16;   // of a pass; of a row
      unsigned char* stage = smem + (pair ? 8192 : 4096) * warp;
      const int d0 = pair ? 0 : D / 2 * slot, d1 = pair ? D : d0 + D / 2;
#pragma unroll 1
      for (int d = d0; d < d1 && !idle; d += dims) {
#pragma unroll 1
        for (int e = 0; e < dims; e += 16) {
          uint32_t o[16], y[16];
          ptx::tmem_ld_16raw(col_o + (pair ? 128 * slot : 0) + d + e, o);
          if (!pair) ptx::tmem_ld_16raw(col_o + 128 + d + e, y);
          ptx::tmem_ld_wait();
          ptx::tmem_regs_ready(o);
          if (!pair) {
            ptx::tmem_regs_ready(y);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float both = f0 == 0.0f ? 0.0f : f0 * __uint_as_float(o[i]);
              if (f1 != 0.0f) both = fmaf(f1, __uint_as_float(y[i]), both);
              o[i] = __float_as_uint(both);
            }
          }
          if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float lo = __uint_as_float(o[2 * i]), hi = __uint_as_float(o[2 * i + 1]);
              o[i] = narrow(T(), l == 0.0f ? 0.0f : lo * inv, l == 0.0f ? 0.0f : hi * inv);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i == 2 && whole) break;
            const int at = (whole ? e / 8 : e / 4) + i;
            *reinterpret_cast<uint4*>(stage + (lane * pieces + (at ^ (lane & 7))) * 16) =
                make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          }
        }
        __syncwarp();
        const int shift = pair ? 4 : 3;              // pieces: 16 or 8
#pragma unroll 2
        for (int i = lane; i < 32 * pieces; i += 32) {
          const int row = i >> shift, at = i & (pieces - 1);
          const uint4 y = *reinterpret_cast<const uint4*>(stage + (row * pieces + (at ^ (row & 7))) * 16);
          const int of = my_row - lane + row;
          const int64_t to = __shfl_sync(0xffffffffu, out_row, row);
          if (of < g.rows) {
            if (whole) *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + to * D + d + 8 * at) = y;
            else *reinterpret_cast<uint4*>(piece + of * D + d + 4 * at) = y;
          }
        }
        __syncwarp();
      }
      if (in && (pair || slot == 0)) {
        if (!whole) {
          piece[kBlockRows * D + my_row] = m_out;
          piece[kBlockRows * (D + 1) + my_row] = l;
        } else if (a.lse) {
          a.lse[out_row] = (m == -INFINITY ? 0.0f : m_out * kLn2) + logf(l);
        }
      }
      if (tid == 0 && begins && !whole) {
        desc[2 * blockIdx.x] = make_int4(g.last_cta, g.h, g.row0, g.rows);
        desc[2 * blockIdx.x + 1] = make_int4(g.i0, 0, 0, 0);
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sy.seg_free[seg_i % kSegs]);
    }
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (sy.abort) {                                    // copies under way write to this CTA's memory: wait them out
    if (tid == 0) {
      const uint64_t t0 = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - t0 < 100000000ull) __nanosleep(1000000);
    }
    __syncthreads();
  }
  if (warp == 2) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// Joins the pieces of the segment that CTA blockIdx.x of the first launch began and did not end; a warp a row, a lane four dimensions.
// And writes the results of free slots: a lane looks at a row of the table, its warp writes.
constexpr int kJoinRows = 8;
template <typename T>
__global__ void __launch_bounds__(kJoinRows * 32) aatc_paged_tree_join_kernel(const TreeArgs a, int n_ctas) {
  const int c0 = blockIdx.x, row = blockIdx.y * kJoinRows + threadIdx.x / 32, lane = threadIdx.x % 32;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (!a.starts && blockIdx.y == 0) {
    for (int64_t b0 = 32ll * (c0 * kJoinRows + threadIdx.x / 32); b0 < a.batch; b0 += 32ll * kJoinRows * gridDim.x) {
      for (uint32_t free = __ballot_sync(0xffffffffu, b0 + lane < a.batch && a.lens[b0 + lane] == 0); free; free &= free - 1) {
        const int64_t first = (b0 + __ffs(free) - 1) * a.n_q;
        uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + first * D);
        for (int i = lane; i < a.n_q * (D / 8); i += 32) out[i] = make_uint4(0u, 0u, 0u, 0u);
        for (int i = lane; a.lse && i < a.n_q; i += 32) a.lse[first + i] = -INFINITY;
      }
    }
  }
  const int4* desc = reinterpret_cast<const int4*>(a.ws + static_cast<size_t>(n_ctas) * 2 * kTreePiece) + 2 * c0;
  const int4 what = __ldcg(desc);                    // last CTA, kv-head, first row, rows
  if (what.x < 0 || row >= what.w) return;
  const int i0 = __ldcg(desc + 1).x, n = what.x - c0 + 1;        // pieces 2 c0 + 1, 2 (c0 + 1), 2 (c0 + 2), ...
  float top = -INFINITY, total = 0.0f;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kAtOnce = 4;
  for (int k0 = 0; k0 < n; k0 += kAtOnce) {
    float m[kAtOnce], l[kAtOnce];
    float4 o[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = k0 + k;
      const float* piece = a.ws + (static_cast<size_t>(c0 + i) * 2 + (i == 0 ? 1 : 0)) * kTreePiece;
      m[k] = i < n ? __ldcg(piece + kBlockRows * D + row) : -INFINITY;
      l[k] = i < n ? __ldcg(piece + kBlockRows * (D + 1) + row) : 0.0f;
      o[k] = i < n ? __ldcg(reinterpret_cast<const float4*>(piece + row * D) + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    float next = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) next = fmaxf(next, m[k]);
    const float base = next == -INFINITY ? 0.0f : next, r = factor_of(top - base);
    total *= r;
    sum.x *= r;
    sum.y *= r;
    sum.z *= r;
    sum.w *= r;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (l[k] == 0.0f) continue;                    // (a piece of nothing)
      const float f = factor_of(m[k] - base);
      total = fmaf(f, l[k], total);
      sum.x = fmaf(f, o[k].x, sum.x);
      sum.y = fmaf(f, o[k].y, sum.y);
      sum.z = fmaf(f, o[k].z, sum.z);
      sum.w = fmaf(f, o[k].w, sum.w);
    }
    top = next;
  }
  const int R = what.z + row, query = quotient(R, a.group), head = what.y * a.group + R - query * a.group;
  const int64_t out_row = static_cast<int64_t>(i0 + query) * a.n_q + head;
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  if (total == 0.0f) sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  reinterpret_cast<uint2*>(static_cast<T*>(a.out) + out_row * D)[lane] =
      make_uint2(narrow(T(), sum.x * inv, sum.y * inv), narrow(T(), sum.z * inv, sum.w * inv));
  if (a.lse && lane == 0) a.lse[out_row] = (top == -INFINITY ? 0.0f : top * kLn2) + logf(total);
}

// ---------------------------------------------------------------- weights
// The scores the other way round: S^T = K Q^T, a tile of 128 tokens in the TMEM lanes, the rows (query, head of the group) of a
// kv-head in the columns, so that a thread has a token and sums exp(s - lse) over its columns; nothing goes from thread to
// thread, and the work is in proportion to the rows (32 at least).  Keys are the floor: 256 bytes a token and kv-head, once for 256 rows.
// One query of each of 16 ragged sequences (8192 tokens at most, 8 kv-heads) 11 to 14 us, of which the keys need 7; 32 queries x 7 heads over
// 3 x 32768 tokens x 4 kv-heads (f16) 31 us, the keys 15: 88 million exponentials, whose unit is busy 27 % of the time, and for every
// tile and warp 224 columns that come from TMEM 16 at a time; one query over 1001 tokens 5.3 us, a launch and the way of the first tile.
// Segments are a sequence's kv-heads, in equal parts of a line over the CTAs as in the attention; more than 256 rows of them
// take the CTA's tiles again.  Roles: eight warps sum, four a TMEM buffer, which take turns at the tiles; one warp issues the
// MMAs; one walks the line and brings the keys.
constexpr int kSumRows = 256;                    // columns of a TMEM buffer
constexpr int kSumGap = 2;                       // as kTreeGap (1: 12.1 us for the 16 ragged sequences, 11.3 with 2)
constexpr size_t kSumSmem = static_cast<size_t>(kSumRows) * D * 2 + kRing * kItem;

__device__ __forceinline__ Pos sum_tiles(const TreeArgs& a, const Seq& s) {
  return s.n == 0 && a.decay == 1.0f ? 0 : tiles_to(min(s.len, a.width));
}

// rows == 0: there is no more; rows < 0: no queries, the weights are decayed only.
struct __align__(16) SumSegment {
  int b, h, i0, n;
  int before, hi, row0, rows;
  int t0, t1, first;                // first: the old weights are decayed
};

struct SumSync {
  uint64_t k_full[kRing], k_free[kRing], s_full[2], s_free[2], q_full, seg_full[kSegs], seg_free[kSegs], info_full[kInfos];
  SumSegment seg[kSegs];
  uint32_t bad[kInfos];
  float lse[kSumRows];              // times -log2(e); -infinity: gives nothing
  uint32_t tmem;
  int abort;
};

template <typename T, bool kFarCap>
__global__ void __launch_bounds__(320, 1) aatc_paged_weights_kernel(const TreeArgs a, const __grid_constant__ CUtensorMap map) {
  extern __shared__ __align__(1024) unsigned char smem[];        // queries, then the ring
  __shared__ SumSync sy;
  const Pool& p = a.pool;
  const int tid = threadIdx.x, warp = ptx::warp_uniform(tid / 32), lane = tid % 32;
  unsigned char* ring = smem + kSumRows * D * 2;
  volatile int* abort_flag = &sy.abort;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return ptx::mbar_try_wait(bar, parity) || wait_long(bar, parity, abort_flag, p.err); };
  auto stopped = [&]() { return __any_sync(0xffffffffu, *abort_flag) != 0; };
  constexpr int kBarriers = 2 * kRing + 5 + 2 * kSegs + kInfos, kWarps = 8;
  static_assert(offsetof(SumSync, k_full) == 0 && offsetof(SumSync, info_full) == (kBarriers - kInfos) * sizeof(uint64_t),
                "every barrier is set up");
  if (warp == kWarps + 1) {
    for (int i = lane; i < kBarriers; i += 32) {
      uint64_t* bar = sy.k_full + i;
      ptx::mbar_init(bar, bar >= sy.s_free && bar < sy.s_free + 2 ? kWarps / 2
                          : bar == &sy.q_full ? kWarps
                          : bar >= sy.seg_free && bar < sy.seg_free + kSegs ? kWarps + 1 : 1);
    }
    if (lane == 0) {
      sy.abort = 0;
      ptx::prefetch_tmap(&map);
    }
    ptx::fence_mbar_init();
  }
  if (warp == 0) {
    ptx::tmem_alloc(&sy.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const uint32_t tmem = sy.tmem;

  if (warp == kWarps + 1) {
    // ---- the walk
    auto fit = [&](const Seq& s, bool tells) {
      if (tells && s.len > a.width) raise(p.err, kBadRow);
      const Pos tiles = sum_tiles(a, s);
      return tiles > 0 ? (tiles + kSumGap) * p.n_kv : 0;
    };
    Begin at = begin_of(a.batch, 1, [&](int i, bool tells) { return fit(seq_of(a, i, tells), tells); });
    int seg_i = 0, item = 0, tile_i = 0;
    uint32_t free_round = 0;
    auto tell = [&](const SumSegment& s) {
      const int to = seg_i % kSegs;
      if (seg_i >= kSegs) {
        wait(&sy.seg_free[to], free_round >> to & 1u);
        free_round ^= 1u << to;
      }
      if (stopped()) return;
      if (lane == 0) {
        sy.seg[to] = s;
        ptx::mbar_arrive(&sy.seg_full[to]);
      }
      ++seg_i;
      __syncwarp();
    };
    const int shift = p.page_shift, page = 1 << shift, rows_box = min(page, kTile), n_boxes = kTile / rows_box;
    const uint32_t box_bytes = rows_box * D * 2;
    Pos x = at.x, off = at.off;
    int b = at.b, h = 0;
    while (x < at.x_end && b < a.batch && !stopped()) {
      const Seq s = seq_of(a, b, false);
      const int tiles = static_cast<int>(sum_tiles(a, s)), hi = min(s.len, a.width);
      const Pos each = tiles + kSumGap;              // (a gap, then the tiles)
      if (tiles == 0) {
        ++b;
        continue;
      }
      while (h + 1 < p.n_kv && off >= each) {
        off -= each;
        ++h;
      }
      const int t0 = static_cast<int>(max(static_cast<Pos>(0), off - kSumGap));
      x += max(static_cast<Pos>(0), kSumGap - off);  // the gap's rest
      off = 0;
      const int t1 = static_cast<int>(min(static_cast<Pos>(tiles), t0 + max(static_cast<Pos>(0), at.x_end - x)));
      const int rows = s.n * a.group;
      for (int row0 = 0; t0 < t1 && (row0 < rows || row0 == 0); row0 += kSumRows) {
        SumSegment g;
        g.b = b;
        g.h = h;
        g.i0 = s.i0;
        g.n = s.n;
        g.before = s.before();
        g.hi = hi;
        g.row0 = row0;
        g.rows = rows == 0 ? -1 : min(kSumRows, rows - row0);
        g.t0 = t0;
        g.t1 = t1;
        g.first = row0 == 0;
        tell(g);
        if (rows == 0) break;
        const int32_t* row = p.table + static_cast<int64_t>(b) * p.table_stride;
        auto id_of = [&](int tile) {                 // the page of this lane's box
          const int tok = tile * kTile + lane * rows_box;
          return lane < n_boxes && tok < hi ? row[tok >> shift] : 0;
        };
        int id = id_of(t0);
        for (int t = t0; t < t1; ++t, ++item) {
          const int tok = t * kTile + lane * rows_box;
          const bool live = lane < n_boxes && tok < hi, ok = live && static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages);
          const int now = id;
          if (t + 1 < t1) id = id_of(t + 1);
          if (live && !ok) raise(p.err, kBadPage);
          const uint32_t n_ok = __popc(__ballot_sync(0xffffffffu, ok));
          uint32_t bad = live && !ok ? (rows_box >= kTile ? 0xFFFFu : ((1u << rows_box / 8) - 1u) << lane * (rows_box / 8)) : 0u;
          bad = __reduce_or_sync(0xffffffffu, bad);
          if (lane == 0) {
            sy.bad[tile_i % kInfos] = bad;
            ptx::mbar_arrive(&sy.info_full[tile_i % kInfos]);
          }
          ++tile_i;
          const int to = item % kRing;
          if (item >= kRing) wait(&sy.k_free[to], (item / kRing - 1) & 1);
          if (stopped()) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(&sy.k_full[to], n_ok * box_bytes);
          __syncwarp();
          if (ok)
            ptx::tma_load_5d(ring + to * kItem + lane * box_bytes, &map, &sy.k_full[to], 0, 0, 0, ((h << shift) + (tok & (page - 1))) / 8, now);
        }
        if (stopped()) break;
      }
      x += t1 - t0;
      if (t1 < tiles) break;                         // (the share ends inside)
      if (++h == p.n_kv) {
        h = 0;
        ++b;
      }
    }
    SumSegment none = {};
    tell(none);
  } else if (warp == kWarps) {
    // ---- MMAs, issued by the converged warp; the waits are not calls, over which nothing would stay in uniform registers
    auto wait_here = [&](uint64_t* bar, uint32_t parity) {
      if (ptx::mbar_wait_bounded(bar, parity, abort_flag)) return true;
      if (!*abort_flag) raise(p.err, kTimeout);
      *abort_flag = 1;
      return false;
    };
    const uint32_t el = ptx::elect_one(), tm = ptx::warp_uniform(tmem);
    const uint64_t q_desc = smem_desc(ptx::smem_u32(smem), 16, 1024), k_desc = smem_desc(ptx::smem_u32(ring), 16, kGroupStep);
    int k_at = 0;
    uint32_t k_parity = 0, free_parity = 3, q_parity = 0;         // (the buffers are free at first)
    for (int seg_i = 0;; ++seg_i) {
      const bool there = wait_here(&sy.seg_full[seg_i % kSegs], seg_i / kSegs & 1) && !*abort_flag;
      if (!__all_sync(0xffffffffu, there)) break;
      const SumSegment& g = sy.seg[seg_i % kSegs];
      const int rows = g.rows, n_tiles = g.t1 - g.t0;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sy.seg_free[seg_i % kSegs]);
      if (__any_sync(0xffffffffu, rows == 0)) break;
      if (__any_sync(0xffffffffu, rows < 0)) continue;
      // fp32 sums, 128 tokens x the rows up to a multiple of 32
      const uint32_t idesc = (1u << 4) | (Half16<T>::kFormat << 7) | (Half16<T>::kFormat << 10) | ((rows + 31) / 32 * 4 << 17) | (8u << 24);
      wait_here(&sy.q_full, q_parity);
      q_parity ^= 1;
      ptx::tc_fence_after();
      for (int t = 0; __any_sync(0xffffffffu, t < n_tiles); ++t) {
        const uint32_t buf = t & 1;
        wait_here(&sy.k_full[k_at], k_parity);
        wait_here(&sy.s_free[buf], free_parity >> buf & 1u);
        free_parity ^= 1u << buf;
        ptx::tc_fence_after();
        const uint64_t kd = k_desc + static_cast<uint64_t>(k_at) * (kItem >> 4);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          ptx::umma_bf16_w(tm + kSumRows * buf, kd + (((kk >> 2) * kHalfStep + (kk & 3) * 32) >> 4),
                           q_desc + (((kk >> 2) * (kSumRows * 128) + (kk & 3) * 32) >> 4), idesc, kk > 0 ? 1u : 0u, el);
        ptx::umma_commit_w(&sy.s_full[buf], el);
        ptx::umma_commit_w(&sy.k_free[k_at], el);
        if (++k_at == kRing) {
          k_at = 0;
          k_parity ^= 1;
        }
      }
    }
  } else {
    // ---- sums: warp w has tokens 32 (w % 4) .. + 31 of tiles w / 4, w / 4 + 2, ...
    const int buf = warp / 4, r = tid % kTile;
    const uint32_t col = tmem + (static_cast<uint32_t>(32 * (warp % 4)) << 16) + kSumRows * buf;
    const bool cap = kFarCap || a.cap > 0.0f;
    const float cap_in = cap ? 2.0f * a.unit / a.cap : 0.0f, far_in = cap ? a.unit * kLn2 / a.cap : 0.0f, cap_out = a.cap * kLog2e;
    const uint64_t unit2 = cap ? ptx::f2_pack(1.0f, 1.0f) : ptx::f2_pack(a.unit, a.odd_unit);
    int tile0 = 0;
    uint32_t s_parity = 0;
    for (int seg_i = 0;; ++seg_i) {
      const bool there = wait(&sy.seg_full[seg_i % kSegs], seg_i / kSegs & 1);
      // (every thread is past the last segment's tiles)
      if (!both_agree(there && !*abort_flag)) break;
      const SumSegment& g = sy.seg[seg_i % kSegs];
      if (g.rows == 0) break;
      const int n_tiles = g.t1 - g.t0, columns = (g.rows + 31) / 32 * 32;
      float* const to = a.weights + (static_cast<int64_t>(g.b) * p.n_kv + g.h) * a.width;
      if (g.rows > 0) {
        // ---- queries and log-sums to shared memory; behind the last row the last query's once more, with no weight (zeros would make
        // NaN of infinite keys, where the rows make weights of 0)
        const int piece = tid % 16, by = 16 / a.group, by_head = 16 - by * a.group;
        int query = quotient(g.row0 + tid / 16, a.group), head = g.row0 + tid / 16 - query * a.group;
        const int last_query = quotient(g.row0 + g.rows - 1, a.group), last_head = g.row0 + g.rows - 1 - last_query * a.group;
#pragma unroll 1
        for (int row = tid / 16; row < columns; row += 16) {
          const bool in = row < g.rows;
          const T* from = static_cast<const T*>(a.q.x) + (g.i0 + (in ? query : last_query)) * a.q.token_stride +
                          (g.h * a.group + (in ? head : last_head)) * a.q.head_stride + 8 * piece;
          ptx::cp_async_16(smem + piece / 8 * (kSumRows * 128) + row * 128 + ((piece % 8) ^ (row % 8)) * 16, from, 16);
          query += by;
          head += by_head;
          if (head >= a.group) {
            head -= a.group;
            ++query;
          }
        }
        float e = -INFINITY;
        if (tid < g.rows) {
          const int R = g.row0 + tid, of = quotient(R, a.group);
          e = a.lse[static_cast<int64_t>(g.i0 + of) * a.n_q + g.h * a.group + R - of * a.group] * -kLog2e;
          if (e == INFINITY) e = -INFINITY;          // (its query sees nothing)
        }
        sy.lse[tid] = e;
        ptx::cp_async_wait_all();
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sy.q_full);
        both_sync();
      }
      if (g.rows < 0) {                              // no queries
        const int64_t end = min(static_cast<int64_t>(g.t1) * kTile, static_cast<int64_t>(g.hi));
#pragma unroll 8
        for (int64_t tok = static_cast<int64_t>(g.t0) * kTile + tid; tok < end; tok += 2 * kTile)
          to[tok] = a.decay == 0.0f ? 0.0f : to[tok] * a.decay;
      }
      for (int k = buf; k < n_tiles && g.rows > 0; k += 2) {
        const int tok = (g.t0 + k) * kTile + r;
        const bool in = tok < g.hi;
        float w = 0.0f;
        if (in && !(g.first && a.decay == 0.0f)) w = to[tok];
        if (g.first) w = a.decay == 0.0f ? 0.0f : w * a.decay;
        {
          const int info = (tile0 + k) % kInfos;
          wait(&sy.info_full[info], (tile0 + k) / kInfos & 1);
          const bool bad = sy.bad[info] >> r / 8 & 1u;
          // whether there may be a query that does not see all of the tile's tokens (of a chain, every one sees the first drafted one)
          const int last = min(tok - r + (kTile - 1), g.hi - 1);
          const bool edge = last - g.before >= (a.mask ? 0 : 1);
          wait(&sy.s_full[buf], s_parity);
          s_parity ^= 1;
          ptx::tc_fence_after();
          uint64_t sum0 = ptx::f2_pack(0.0f, 0.0f), sum1 = sum0;
          // exp(s - lse) of 4 columns from j on
          auto add = [&](const uint32_t* x, int j, auto is_edge, uint32_t vis) {
            const float4 e = *reinterpret_cast<const float4*>(&sy.lse[j]);               // (negated)
            float y[4];
            const uint64_t lo = ptx::f2_pack(__uint_as_float(x[0]), __uint_as_float(x[1])), hi = ptx::f2_pack(__uint_as_float(x[2]), __uint_as_float(x[3]));
            ptx::f2_unpack(ptx::f2_fma(lo, unit2, ptx::f2_pack(e.x, e.y)), y[0], y[1]);
            ptx::f2_unpack(ptx::f2_fma(hi, unit2, ptx::f2_pack(e.z, e.w)), y[2], y[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              y[i] = exp2_of(y[i]);
              if constexpr (decltype(is_edge)::value) y[i] = vis >> i & 1u ? y[i] : 0.0f;
            }
            sum0 = ptx::f2_add(sum0, ptx::f2_pack(y[0], y[1]));
            sum1 = ptx::f2_add(sum1, ptx::f2_pack(y[2], y[3]));
          };
          if (edge || cap) {
            // Of a chain, token j of the drafted ones is seen from its own query's columns on; of a tree, by the queries whose
            // bit it is, four queries' words at a time.
            const int drafted = tok - g.before, from = edge && !a.mask ? max(0, drafted) * a.group - g.row0 : 0;
            const bool masked = edge && a.mask && drafted >= 0 && drafted < g.n;
            const int32_t* word = masked ? a.mask + static_cast<int64_t>(g.i0) * a.mask_words + drafted / 32 : nullptr;
#pragma unroll 1
            for (int j0 = 0; j0 < columns; j0 += 16) {
              uint32_t x[16], vis = 0xFFFFu;
              ptx::tmem_ld_16raw(col + j0, x);
              if (masked) {
                vis = 0;
                const int R = g.row0 + j0, last = min(g.n - 1, quotient(R + 15, a.group));
                for (int i = quotient(R, a.group); i <= last; i += 4) {
                  uint32_t w[4];
#pragma unroll
                  for (int y = 0; y < 4; ++y) w[y] = i + y <= last ? word[static_cast<int64_t>(i + y) * a.mask_words] : 0u;
#pragma unroll
                  for (int y = 0; y < 4; ++y) {
                    const int lo = max((i + y) * a.group - R, 0), hi = min((i + y + 1) * a.group - R, 16);
                    if (i + y <= last && (w[y] >> drafted % 32 & 1u)) vis |= (1u << hi) - (1u << lo);
                  }
                }
              } else if (from > j0) {
                vis = from - j0 >= 16 ? 0u : 0xFFFFu << (from - j0);
              }
              ptx::tmem_ld_wait();
              ptx::tmem_regs_ready(x);
              if constexpr (kFarCap) {
                cap_far(x, a.unit, far_in, cap_out);
              } else if (cap) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                  x[j] = __float_as_uint(fmaf(-2.0f * cap_out, reciprocal(exp2_of(__uint_as_float(x[j]) * cap_in) + 1.0f), cap_out));
              }
#pragma unroll
              for (int j = 0; j < 16; j += 4) add(x + j, j0 + j, std::true_type(), vis >> j);
            }
          } else {
            // 16 columns at a time, the next ones on their way
            uint32_t x0[16], x1[16];
            ptx::tmem_ld_16raw(col, x0);
#pragma unroll 1
            for (int j0 = 0; j0 < columns; j0 += 32) {
              ptx::tmem_ld_wait();
              ptx::tmem_regs_ready(x0);
              ptx::tmem_ld_16raw(col + j0 + 16, x1);
#pragma unroll
              for (int j = 0; j < 16; j += 4) add(x0 + j, j0 + j, std::false_type(), 0u);
              ptx::tmem_ld_wait();
              ptx::tmem_regs_ready(x1);
              if (j0 + 32 < columns) ptx::tmem_ld_16raw(col + j0 + 32, x0);
#pragma unroll
              for (int j = 0; j < 16; j += 4) add(x1 + j, j0 + 16 + j, std::false_type(), 0u);
            }
          }
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&sy.s_free[buf]);
          float lo, hi;
          ptx::f2_unpack(ptx::f2_add(sum0, sum1), lo, hi);
          if (!bad) w += lo + hi;
        }
        if (in) to[tok] = w;
      }
      if (g.rows > 0) tile0 += n_tiles;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sy.seg_free[seg_i % kSegs]);
    }
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (sy.abort) {                                    // copies under way write to this CTA's memory: wait them out
    if (tid == 0) {
      const uint64_t t0 = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - t0 < 100000000ull) __nanosleep(1000000);
    }
    __syncthreads();
  }
  if (warp == 0) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
}

}  // namespace

size_t tree_workspace(int num_sms) {
  return static_cast<size_t>(std::max(1, num_sms)) * (2 * kTreePiece * sizeof(float) + 2 * sizeof(int4));
}

// The pages in boxes of a page, or of a tile where that is smaller.
static cudaError_t tile_map(CUtensorMap* map, const Pool& p) {
  const uint64_t tokens = static_cast<uint64_t>(2) * p.n_kv << p.page_shift;
  return make_tensor_map_groups(map, p.pages, tokens, p.n_pages, std::min(1 << p.page_shift, kTile));
}

cudaError_t launch_tree(int dtype, const TreeArgs& a, cudaStream_t st) {
  const int ctas = std::max(1, a.num_sms);
  const bool bf16 = dtype == AATC_BF16;
  constexpr decltype(&aatc_paged_tree_kernel<__half, kNone>) kernels[2][3] = {
      {aatc_paged_tree_kernel<__half, kNone>, aatc_paged_tree_kernel<__half, kNear>, aatc_paged_tree_kernel<__half, kFar>},
      {aatc_paged_tree_kernel<__nv_bfloat16, kNone>, aatc_paged_tree_kernel<__nv_bfloat16, kNear>, aatc_paged_tree_kernel<__nv_bfloat16, kFar>}};
  const auto kernel = kernels[bf16][cap_kind(a.cap)];
  CUtensorMap map;
  cudaError_t e = tile_map(&map, a.pool);
  if (e != cudaSuccess) return e;
  e = ensure_smem_optin(reinterpret_cast<const void*>(kernel), kTreeSmem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(ctas), dim3(kTreeThreads), kTreeSmem, st, a, map);
  if (e != cudaSuccess) return e;
  const int rows = static_cast<int>(std::min<int64_t>(kBlockRows, static_cast<int64_t>(a.n_tokens) * a.group));
  return launch_pdl(bf16 ? aatc_paged_tree_join_kernel<__nv_bfloat16> : aatc_paged_tree_join_kernel<__half>,
                    dim3(ctas, (rows + kJoinRows - 1) / kJoinRows), dim3(kJoinRows * 32), 0, st, a, ctas);
}

cudaError_t launch_weights(int dtype, const TreeArgs& a, cudaStream_t st) {
  const bool far = cap_kind(a.cap) == kFar;
  const auto kernel = dtype == AATC_BF16 ? (far ? aatc_paged_weights_kernel<__nv_bfloat16, true> : aatc_paged_weights_kernel<__nv_bfloat16, false>)
                                         : (far ? aatc_paged_weights_kernel<__half, true> : aatc_paged_weights_kernel<__half, false>);
  CUtensorMap map;
  cudaError_t e = tile_map(&map, a.pool);
  if (e != cudaSuccess) return e;
  e = ensure_smem_optin(reinterpret_cast<const void*>(kernel), kSumSmem);
  if (e != cudaSuccess) return e;
  // The tensor cores cut their sums off, toward 0: sums of 128 products come out low by 1.35 (bf16) or 2.4 (f16) times 2^-24 of
  // their value on average (measured, 1 to 2.5 over scores of several spreads), which a weight would show.  The unit makes up for
  // it.  As one unit rounds by as much, odd columns have another one, so that both are right on average (a unit's rest, multiplied
  // and added on its own, is mostly less than half a step of the sum, and lost).  A single column has its unit's 2^-25 of a score.
  const double low = (dtype == AATC_BF16 ? 1.35 : 2.4) / (1 << 24), unit = static_cast<double>(a.scale) * 1.4426950408889634 * (1.0 + low);
  TreeArgs args = a;
  args.unit = static_cast<float>(unit);
  args.odd_unit = static_cast<float>(2.0 * unit - args.unit);
  return launch_pdl(kernel, dim3(std::max(1, a.num_sms)), dim3(320), kSumSmem, st, args, map);
}

}  // namespace paged
}  // namespace aatc
