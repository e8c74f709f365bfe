// The choice of the tokens that a sequence keeps, and their move in the pages.
#include <cooperative_groups.h>

#include <algorithm>

#include "aatc_internal.h"
#include "paged.h"
#include "paged_device.cuh"
#include "ptx.cuh"

namespace aatc {
namespace paged {

namespace {

// Weights as unsigned numbers in the same order; -0 and 0 are equal, a NaN is above everything.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (w != w) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The row of a sequence and head is dealt out in equal runs over the CTAs of a cluster, each of which keeps the ranks of
// its tokens in shared memory, read once.  The rank of the last token that is kept comes digit by digit from the top: the tokens whose
// upper digits are those found are counted by their next digit, and the first digit at which the counts from above pass the places
// left is the next one found.  There are three rounds, of 11, 11 and 10 bits; eight CTAs, which read each other's counts, have four of
// 8 (8 rows of 131072 tokens 15.6 us, 19.0 with three; 32 rows, of four CTAs each, 18.8 with three and 19.7 with four).
// The counts also say how many tokens the CTAs
// before this one keep.  Then a thread looks at some neighbouring tokens, and a prefix sum over the threads gives their places.
//
// What bounds it is the chain of rounds, not the bytes: a row of 1201 tokens 4.9 us, of which a launch is 2.2; 61 x 4 rows of up to
// 8192 tokens 8.9 us (floor 0.7); 4 x 8 rows of 131072 18.8 us (floor 2.6): 2 to load, then round
// after round 1.5 to 2.5 for the ranks and their shared atomics, 0.6 for the cluster's barrier, 0.6 for the counts over the cluster,
// 0.7 for the digit.  Equal weights are all counted in one bin, an atomic after the other: 32768 of 4 x 8 rows of 131072 tokens 43 us
// for 23 (rows of 8192 tokens 18 for 17).
constexpr int kChooseThreads = 1024;
constexpr int kWarps = kChooseThreads / 32;
constexpr int kBins = 2 * kChooseThreads;        // two bins a thread
constexpr int kBlock = 32 * kChooseThreads;      // tokens that the threads look at at once, at most
constexpr int kHeld = 49152;                     // tokens of a CTA that stay in shared memory; of longer runs, blocks are read again
constexpr int kEarly = 2;                        // tokens of a thread that are loaded before the length is there
constexpr size_t kChooseSmem = static_cast<size_t>(kHeld) * 4;
constexpr int kChooseTokens = 20480;             // of a row, beyond which more CTAs of a cluster (eight at most) bring more than they cost

__device__ __forceinline__ int upto_lane(int x) {  // over the lanes up to and with this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (static_cast<int>(threadIdx.x % 32) >= o) x += y;
  }
  return x;
}

// kCluster: the row has several CTAs.
template <bool kCluster>
__global__ void __launch_bounds__(kChooseThreads, 1) aatc_choose_tokens_kernel(const ChooseArgs a) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(16) uint32_t held[];             // ranks
  __shared__ int s_count[2][kBins], s_part[2][kWarps], s_before[2];
  __shared__ int2 s_found[2];                    // digit, places left in it
  const cg::cluster_group cluster = cg::this_cluster();
  const int n_ctas = kCluster ? cluster.num_blocks() : 1, me = kCluster ? cluster.block_rank() : 0;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, h = blockIdx.x / n_ctas, b = blockIdx.y;
  s_count[0][tid] = s_count[0][kChooseThreads + tid] = 0;
  if (tid < 2) s_before[tid] = 0;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int64_t row = static_cast<int64_t>(b) * a.n_heads + h;
  const float* w = a.weights + row * a.width;
  int32_t* kept = a.kept + row * a.keep;
  const int len = a.lens[b];
  float early[kEarly];                           // (of a row's only CTA, whose run begins at `first`)
#pragma unroll
  for (int i = 0; i < kEarly; ++i) {
    const int64_t t = static_cast<int64_t>(a.first) + i * kChooseThreads + tid;
    early[i] = !kCluster && t < a.width ? w[t] : 0.0f;
  }
  const int n = min(max(len, 0), a.width);
  const unsigned all_threads = n_ctas * kChooseThreads, thread = me * kChooseThreads + tid;    // (indexes may pass 2^31 by a step)
  if (n <= a.keep) {
    for (unsigned j = thread; j < static_cast<unsigned>(a.keep); j += all_threads) kept[j] = j < static_cast<unsigned>(n) ? j : -1;
    return;
  }
  for (unsigned j = thread; j < static_cast<unsigned>(a.first); j += all_threads) kept[j] = j;
  for (unsigned j = thread; j < static_cast<unsigned>(a.last); j += all_threads) kept[a.keep - a.last + j] = n - a.last + j;
  int left = a.keep - a.first - a.last;          // the places that tokens have to earn
  if (left == 0) return;
  const int some = n - a.first - a.last;         // the tokens that may
  const int from = a.first + static_cast<int>(static_cast<int64_t>(some) * me / n_ctas);
  const int mine = a.first + static_cast<int>(static_cast<int64_t>(some) * (me + 1) / n_ctas) - from;
  const bool stays = mine <= kHeld;
  auto hold = [&](int at, int i0, int count) {   // ranks of tokens from + at + i0 .. + count to the front (the caller synchronises)
#pragma unroll 8
    for (int i = i0 + tid; i < count; i += kChooseThreads) held[i] = rank_of(w[from + at + i]);
  };
  if (stays) {
    int i0 = 0;
    if (!kCluster) {
#pragma unroll
      for (int i = 0; i < kEarly; ++i)
        if (i * kChooseThreads + tid < mine) held[i * kChooseThreads + tid] = rank_of(early[i]);
      i0 = kEarly * kChooseThreads;
    }
    hold(0, i0, mine);
  }
  __syncthreads();
  // ---- the rank of the last one that is kept, how many of that rank are, and how many above it and of it the CTAs before have
  const bool fine = kCluster && n_ctas > 4 && some <= static_cast<int64_t>(n_ctas) * kHeld;    // four rounds of 8 bits (the same in all CTAs)
  const int rounds = fine ? 4 : 3, counters = fine ? 128 : kChooseThreads;
  uint32_t prefix = 0;
  int above_before = 0, equal_before = 0;
#pragma unroll 1
  for (int round = 0; round < rounds; ++round) {
    const int shift = fine ? 24 - 8 * round : round == 0 ? 21 : round == 1 ? 10 : 0, bits = fine ? 8 : round == 2 ? 10 : 11;
    const int turn = round & 1;
    int* count = s_count[turn];
    // the ranks whose upper digits are those found
    const uint32_t lowest = round == 0 ? 0u : prefix << (shift + bits), span = round == 0 ? 0xFFFFFFFFu : (1u << (shift + bits)) - 1u;
#pragma unroll 1
    for (int at = 0; at < mine; at += stays ? mine : kBlock) {
      const int here = stays ? mine : min(kBlock, mine - at);
      if (!stays) {
        __syncthreads();
        hold(at, 0, here);
        __syncthreads();
      }
      // (four ranks a load: 4.5 times the instructions were half of a long row's time)
      auto tell = [&](uint32_t u) {
        if (u - lowest <= span) atomicAdd(&count[(u - lowest) >> shift], 1);
      };
      const int whole = here > 2 * kChooseThreads ? here & ~3 : 0;
#pragma unroll 2
      for (int i = 4 * tid; i < whole; i += 4 * kChooseThreads) {
        const uint4 u = *reinterpret_cast<const uint4*>(held + i);
        tell(u.x);
        tell(u.y);
        tell(u.z);
        tell(u.w);
      }
#pragma unroll 1
      for (int i = whole + tid; i < here; i += kChooseThreads) tell(held[i]);
    }
    if (kCluster) cluster.sync();
    else __syncthreads();
    // thread t has bins 2 t', 2 t' + 1 from the top, t' = threads - 1 - t; the first one whose sum passes `left` finds the digit
    int2 two = make_int2(0, 0), lower = make_int2(0, 0);       // of all CTAs, of those before this one
    const int t2 = 2 * (counters - 1 - tid);
    if (!kCluster) {
      two = *reinterpret_cast<const int2*>(count + t2);
    } else if (tid < counters) {
#pragma unroll 8
      for (int c = 0; c < n_ctas; ++c) {
        const int2 y = *reinterpret_cast<const int2*>(cluster.map_shared_rank(count, c) + t2);
        two.x += y.x;
        two.y += y.y;
        lower.x += c < me ? y.x : 0;
        lower.y += c < me ? y.y : 0;
      }
    }
    // (the other counts have been read by all: they have passed this digit's barrier)
    s_count[turn ^ 1][tid] = s_count[turn ^ 1][kChooseThreads + tid] = 0;
    const int sum = two.x + two.y, of_warp = __reduce_add_sync(0xffffffffu, sum);
    if (lane == 0) s_part[turn][warp] = of_warp;
    __syncthreads();
    const int part = s_part[turn][lane], before_warp = __shfl_sync(0xffffffffu, upto_lane(part) - part, warp);
    if (before_warp < left && left <= before_warp + of_warp) {
      const int before = before_warp + upto_lane(sum) - sum;
      if (before < left && left <= before + sum) {
        const int rest = left - before;
        s_found[turn] = rest <= two.y ? make_int2(t2 + 1, rest) : make_int2(t2, rest - two.y);
      }
    }
    __syncthreads();
    const int2 found = s_found[turn];
    prefix = prefix << bits | static_cast<uint32_t>(found.x);
    left = found.y;
    if (kCluster) {
      const int above = (t2 > found.x ? lower.x : 0) + (t2 + 1 > found.x ? lower.y : 0);
      const int equal = round == rounds - 1 ? (t2 == found.x ? lower.x : 0) + (t2 + 1 == found.x ? lower.y : 0) : 0;
      const int above_warp = __reduce_add_sync(0xffffffffu, above), equal_warp = __reduce_add_sync(0xffffffffu, equal);
      if (lane == 0 && above_warp) atomicAdd(&s_before[0], above_warp);
      if (lane == 0 && equal_warp) atomicAdd(&s_before[1], equal_warp);
    }
  }
  if (kCluster) {
    cluster.sync();                              // (nobody leaves while its counts are still read)
    above_before = s_before[0];
    equal_before = s_before[1];
  }
  // ---- places: a thread looks at `each` neighbouring tokens, four at once, beginning at other ones than its neighbours (other banks)
#pragma unroll 1
  for (int at = 0; at < mine; at += kBlock) {
    const int here = min(kBlock, mine - at);
    int each = 4;
    while (each * kChooseThreads < here) each *= 2;
    __syncthreads();                             // (the last block's sums have been read)
    if (!stays) {
      hold(at, 0, here);
      __syncthreads();
    }
    const uint32_t* ranks = held + (stays ? at : 0);
    uint32_t above = 0, equal = 0;
    const int turned = tid * each / 32;          // in vectors
#pragma unroll 2
    for (int i = 0; i < each / 4; ++i) {
      const int j = 4 * ((i + turned) & (each / 4 - 1)), t = each * tid + j;
      if (t < here) {
        const uint4 u = *reinterpret_cast<const uint4*>(ranks + t);
        above |= (static_cast<uint32_t>(u.x > prefix) | static_cast<uint32_t>(u.y > prefix) << 1 | static_cast<uint32_t>(u.z > prefix) << 2 |
                  static_cast<uint32_t>(u.w > prefix) << 3) << j;
        equal |= (static_cast<uint32_t>(u.x == prefix) | static_cast<uint32_t>(u.y == prefix) << 1 |
                  static_cast<uint32_t>(u.z == prefix) << 2 | static_cast<uint32_t>(u.w == prefix) << 3) << j;
      }
    }
    if (here - each * tid < each) {              // (the last vector's end, which is nobody's)
      const uint32_t mine_only = (1u << max(here - each * tid, 0)) - 1u;
      above &= mine_only;
      equal &= mine_only;
    }
    // both counts in one number: at most 2^15 of each in a block
    const int counts = __popc(above) << 16 | __popc(equal), upto = upto_lane(counts);
    if (lane == 31) s_part[0][warp] = upto;
    __syncthreads();
    const int part = s_part[0][lane], sums = upto_lane(part);
    const uint32_t before = __shfl_sync(0xffffffffu, sums - part, warp) + upto - counts, all = __shfl_sync(0xffffffffu, sums, 31);
    // of those at the rank, the first `left` of the row
    int equals = equal_before + static_cast<int>(before & 0xFFFFu);
    int place = a.first + above_before + static_cast<int>(before >> 16) + min(equals, left);
    above_before += static_cast<int>(all >> 16);
    equal_before += static_cast<int>(all & 0xFFFFu);
    for (uint32_t both = above | equal; both; both &= both - 1) {
      const int j = __ffs(both) - 1;
      if (equal >> j & 1u && equals++ >= left) continue;
      kept[place++] = from + at + each * tid + j;
    }
  }
}

// The entry j of a sequence's list: the token that is moved to place j, or -1 for none.
struct List {
  const int32_t* kept;
  int n_kept, room;         // tokens from the first place on
  __device__ int2 entry(int j) const {           // and the one before
    return static_cast<unsigned>(j) < static_cast<unsigned>(n_kept) ? make_int2(kept[j], j > 0 ? kept[j - 1] : -1) : make_int2(-1, -1);
  }
  __device__ int of(int2 e, int j, int32_t* err) const {
    if (e.x < 0) return -1;
    if (e.x >= room || e.x <= e.y || (j > 0 && e.y < 0)) {
      raise(err, kBadRow);
      return -1;
    }
    return e.x;
  }
  __device__ int at(int j, int32_t* err) const { return of(entry(j), j, err); }
};

// One CTA per layer, sequence, head, kind (keys, values; one more: weights) and part of a token's 256 bytes.  A token never moves
// back, so what a chunk of places overwrites is needed by that chunk or earlier ones only: the CTA goes through the places in
// order, and stores a chunk when all threads have loaded it; the next chunk is on its way by then (its tokens lie behind the
// places that are written), the ids of the one after and the list's entries of the third.
// A quarter of 4 x 32768 tokens x 8 kv-heads to the front, other ones in every head: 51 us, 5.5 TB/s read and written (floor 41); its
// chunks wait for their loads, 32 KB a CTA at once.
constexpr int kKeepThreads = 256;
constexpr int kKeepCtas = 2 * 152;                 // CTAs that a call should have, if it takes parts of tokens for that (two fit an SM)
constexpr int kKeepLoads = 8;                      // 16-byte pieces of a thread in a chunk
__global__ void __launch_bounds__(kKeepThreads) aatc_paged_keep_kernel(const KeepArgs a, int parts) {
  constexpr int kMost = kKeepThreads * kKeepLoads / 4;       // places of a chunk: a quarter of a token (4 pieces) at least
  __shared__ int2 s_move[3][kMost];                // of a place: the blocks (page, kind, head) x page size + slot that it is moved from and to; -1: not
  const Pool& p = a.pool;
  const int tid = threadIdx.x, b = blockIdx.y, layer = blockIdx.z;
  const int part = blockIdx.x % parts, kind_head = blockIdx.x / parts;
  const bool moves_weights = blockIdx.x >= static_cast<unsigned>(2 * p.n_kv * parts);
  const int h = moves_weights ? blockIdx.x - 2 * p.n_kv * parts : kind_head % p.n_kv, kind = kind_head / p.n_kv;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int len = a.lens[b], first = a.first ? a.first[b] : 0, most = p.max_pages << p.page_shift;
  const int n = min(min(max(len, 0), most), a.weights ? a.width : most);
  if (len != n || first < 0 || first > n) {
    if (tid == 0) raise(p.err, kBadRow);
    return;
  }
  const List list = {a.kept + (a.per_head ? static_cast<int64_t>(b) * p.n_kv + h : b) * a.n_kept, a.n_kept, n - first};
  if (moves_weights) {
    constexpr int kEach = 8;
    float* w = a.weights + (static_cast<int64_t>(b) * p.n_kv + h) * a.width + first;
    const unsigned places = n - first, lists = min(a.n_kept, n - first);         // (indexes may pass 2^31 by a step)
    for (unsigned j0 = 0; j0 < lists; j0 += kKeepThreads * kEach) {
      float x[kEach];
      int from[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) from[i] = list.at(j0 + i * kKeepThreads + tid, p.err);
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = from[i] >= 0 ? w[from[i]] : 0.0f;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const unsigned j = j0 + i * kKeepThreads + tid;
        if (j < lists) w[j] = x[i];
      }
    }
    __syncthreads();
    for (unsigned j = lists + tid; j < places; j += kKeepThreads) w[j] = 0.0f;
    return;
  }
  const int32_t* ids = p.table + static_cast<int64_t>(b) * p.table_stride;
  char* base = static_cast<char*>(p.pages) + layer * a.layer_stride;
  const int pieces = 16 / parts, by = kKeepThreads / pieces, chunk = by * kKeepLoads;   // pieces of a token; places of a load and of a chunk
  const int c = tid & (pieces - 1), in = tid / pieces;
  const int places = min(a.n_kept, n - first), chunks = places / chunk + (places % chunk > 0);
  // The places of a chunk are looked up in two steps, by two threads' turns at most: the list's entries, then the pages' ids.
  constexpr int kLooks = kMost / kKeepThreads;
  int2 entry[kLooks], moved[kLooks], id[kLooks];
  auto entries = [&](int k) {
#pragma unroll
    for (int y = 0; y < kLooks; ++y) {
      const int i = y * kKeepThreads + tid, j = k * chunk + i;
      entry[y] = i < chunk && k < chunks && j < places ? list.entry(j) : make_int2(-1, -1);
    }
  };
  auto look = [&](int k) {
#pragma unroll
    for (int y = 0; y < kLooks; ++y) {
      const int j = k * chunk + y * kKeepThreads + tid, source = list.of(entry[y], j, p.err);
      moved[y] = source < 0 || source == j ? make_int2(-1, -1) : make_int2(first + source, first + j);
      id[y] = moved[y].x < 0 ? make_int2(0, 0) : make_int2(ids[moved[y].x >> p.page_shift], ids[moved[y].y >> p.page_shift]);
    }
  };
  // (page x page size + slot: below 2^32, as 2^24 pages have 2^8 tokens at most; -1 would be the last slot of a pool of 2^32 tokens, for
  // which there is no memory)
  auto tell = [&](int k) {
    const int slots = (1 << p.page_shift) - 1;
#pragma unroll
    for (int y = 0; y < kLooks; ++y) {
      const int i = y * kKeepThreads + tid;
      int2 m = make_int2(-1, -1);
      if (moved[y].x >= 0) {
        if (static_cast<uint32_t>(id[y].x) < static_cast<uint32_t>(p.n_pages) && static_cast<uint32_t>(id[y].y) < static_cast<uint32_t>(p.n_pages))
          m = make_int2(static_cast<int>(static_cast<uint32_t>(id[y].x) << p.page_shift | (moved[y].x & slots)),
                        static_cast<int>(static_cast<uint32_t>(id[y].y) << p.page_shift | (moved[y].y & slots)));
        else raise(p.err, kBadPage);
      }
      if (i < chunk) s_move[k % 3][i] = m;
    }
  };
  auto at = [&](int m) -> uint4* {
    const uint32_t token = static_cast<uint32_t>(m), mask = (1u << p.page_shift) - 1u;
    const int64_t block = (static_cast<int64_t>(token >> p.page_shift) * 2 + kind) * p.n_kv + h;
    return reinterpret_cast<uint4*>(base) + ((block << p.page_shift) + (token & mask)) * (D / 8) + part * pieces + c;
  };
  entries(0);
  look(0);
  tell(0);
  entries(1);
  look(1);
  tell(1);
  entries(2);
  __syncthreads();
  uint4 x[2][kKeepLoads];
  auto load = [&](int k, uint4 (&to)[kKeepLoads]) {
#pragma unroll
    for (int i = 0; i < kKeepLoads; ++i) {
      const int m = k < chunks ? s_move[k % 3][in + i * by].x : -1;
      if (m != -1) to[i] = *at(m);
    }
  };
  auto step = [&](int k, uint4 (&now)[kKeepLoads], uint4 (&next)[kKeepLoads]) {
    load(k + 1, next);
    look(k + 2);
    entries(k + 3);
    __syncthreads();                               // (what any thread loaded before it was there before what is stored after it)
#pragma unroll
    for (int i = 0; i < kKeepLoads; ++i) {
      const int m = s_move[k % 3][in + i * by].y;
      if (m != -1) *at(m) = now[i];
    }
    tell(k + 2);
    __syncthreads();
  };
#pragma unroll
  for (int i = 0; i < kKeepLoads; ++i) x[0][i] = x[1][i] = make_uint4(0, 0, 0, 0);
  load(0, x[0]);
  for (int k = 0; k < chunks; k += 2) {
    step(k, x[0], x[1]);
    if (k + 1 < chunks) step(k + 1, x[1], x[0]);
  }
  if (blockIdx.x < static_cast<unsigned>(p.n_kv * parts) && part == 0)        // entries for which there is no room
    for (unsigned j = places + tid; j < static_cast<unsigned>(a.n_kept); j += kKeepThreads) list.at(j, p.err);
}

// Few places without weights, as of a verified path: one chunk.  A CTA moves kFewHeads kv-heads' keys and values; a thread has a piece of a place
// in all of them, its loads before its stores.  16 paths of 6 tokens in 28 layers of 4 kv-heads: 4.3 us, a launch (2.2) and
// the chain of length, entry, ids and data (the general kernel, which looks up chunk by chunk, took 5.9).
constexpr int kFew = 16, kFewHeads = 2;
__global__ void __launch_bounds__(kFew * 16) aatc_paged_keep_few_kernel(const KeepArgs a) {
  const Pool& p = a.pool;
  const int c = threadIdx.x % 16, j = threadIdx.x / 16, h0 = blockIdx.x * kFewHeads, b = blockIdx.y, layer = blockIdx.z;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int len = a.lens[b], first = a.first ? a.first[b] : 0, n = min(max(len, 0), p.max_pages << p.page_shift);
  if (len != n || first < 0 || first > n) {
    if (threadIdx.x == 0) raise(p.err, kBadRow);
    return;
  }
  const int32_t* ids = p.table + static_cast<int64_t>(b) * p.table_stride;
  const int slots = (1 << p.page_shift) - 1;
  uint4* to[kFewHeads] = {};
  uint4 x[kFewHeads][2];
  const int64_t values = static_cast<int64_t>(p.n_kv) << p.page_shift << 4;    // from a key to its value, in 16-byte pieces
#pragma unroll
  for (int i = 0; i < kFewHeads; ++i) {
    const int h = h0 + i;
    if (h >= p.n_kv) break;
    const List list = {a.kept + (a.per_head ? static_cast<int64_t>(b) * p.n_kv + h : b) * a.n_kept, a.n_kept, n - first};
    const int from = list.at(j, p.err);
    if (from < 0 || from == j) continue;
    const int s = first + from, d = first + j;
    const int32_t si = ids[s >> p.page_shift], di = ids[d >> p.page_shift];
    if (static_cast<uint32_t>(si) >= static_cast<uint32_t>(p.n_pages) || static_cast<uint32_t>(di) >= static_cast<uint32_t>(p.n_pages)) {
      raise(p.err, kBadPage);
      continue;
    }
    uint4* base = reinterpret_cast<uint4*>(static_cast<char*>(p.pages) + layer * a.layer_stride) + c;
    const uint4* src = base + (((static_cast<int64_t>(si) * 2 * p.n_kv + h) << p.page_shift) + (s & slots)) * (D / 8);
    to[i] = base + (((static_cast<int64_t>(di) * 2 * p.n_kv + h) << p.page_shift) + (d & slots)) * (D / 8);
    x[i][0] = src[0];
    x[i][1] = src[values];
  }
  __syncthreads();                                 // (what any thread loaded before it was there before what is stored after it)
#pragma unroll
  for (int i = 0; i < kFewHeads; ++i)
    if (to[i]) {
      to[i][0] = x[i][0];
      to[i][values] = x[i][1];
    }
}

}  // namespace

cudaError_t launch_choose(const ChooseArgs& a, cudaStream_t st) {
  // CTAs of a row: twice as many while the rows' CTAs have an SM each, or while a run does not stay in shared memory but would in
  // one of eight.  (Rows x tokens, us with 1, 2, 4, 8 of them: 8 x 16384 9.6, 11.9, 11.3, 10.4; 8 x 32768 14.3, 14.3, 13.2,
  // 11.3; 32 x 131072 70, 51, 21, 25; 76 x 32768 14.5, 14.6, 29, 40; 60 x 131072 71, 51, 41, 46; 32 x 1000000 745, 469, 256, 284.)
  int n_ctas = 1;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.n_heads;
  while (n_ctas < 8 && a.width > kChooseTokens && (rows * n_ctas * 2 <= a.num_sms || (a.width / n_ctas > kHeld && a.width / 8 <= kHeld)))
    n_ctas *= 2;
  const int held = std::min(kHeld, (a.width / n_ctas + 4) & ~3);        // (a run of one more, to whole vectors)
  const size_t smem = static_cast<size_t>(std::max(held, 1024)) * 4;
  const auto kernel = n_ctas > 1 ? aatc_choose_tokens_kernel<true> : aatc_choose_tokens_kernel<false>;
  const cudaError_t e = ensure_smem_optin(reinterpret_cast<const void*>(kernel), kChooseSmem);
  if (e != cudaSuccess) return e;
  if (n_ctas == 1) return launch_pdl(kernel, dim3(a.n_heads, a.batch), dim3(kChooseThreads), smem, st, a);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.n_heads * n_ctas, a.batch);
  cfg.blockDim = dim3(kChooseThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

cudaError_t launch_keep(const KeepArgs& a, cudaStream_t st) {
  if (a.n_kept <= kFew && !a.weights)
    return launch_pdl(aatc_paged_keep_few_kernel, dim3((a.pool.n_kv + kFewHeads - 1) / kFewHeads, a.batch, a.n_layers), dim3(kFew * 16),
                      0, st, a);
  // parts of a token: as many as give every SM a few CTAs, down to 64 bytes
  const int64_t whole = static_cast<int64_t>(2) * a.pool.n_kv * a.batch * a.n_layers;
  const int parts = whole >= kKeepCtas ? 1 : whole * 2 >= kKeepCtas ? 2 : 4;
  return launch_pdl(aatc_paged_keep_kernel, dim3(a.pool.n_kv * (2 * parts + (a.weights ? 1 : 0)), a.batch, a.n_layers),
                    dim3(kKeepThreads), 0, st, a, parts);
}

}  // namespace paged
}  // namespace aatc
