// Paged cache of uncompressed keys and values: what its host entry points (paged_api.cpp) hand to its
// kernels (paged.cu).
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "aatc.h"

namespace aatc {
namespace paged {

// Device flags of the paged calls (include/aatc.h).
constexpr int kTimeout = 2;
constexpr int kBadPage = 4;
constexpr int kBadRow = 8;

// One layer's pages and the block table over them.
struct Pool {
  void* pages;              // [n_pages][2][n_kv][page_size][128]
  const int32_t* table;     // [rows][max_pages], rows table_stride apart
  int table_stride;
  int max_pages;
  int n_pages;
  int n_kv;
  int page_shift;           // page_size = 1 << page_shift
  int32_t* err;             // may be null
};

struct Heads {
  const void* x;            // [tokens][heads][128], strides in elements
  int64_t token_stride;
  int64_t head_stride;
};

struct Turn {
  const uint64_t* turns;    // null: nothing is rotated
  int rot_dim;
  int interleaved;
  float factor;
  float sign;               // -1: the other way
};

// Rotation of q (n_q heads) to q_out, and, where pool.pages is set, keys and values into their pages.
struct AppendArgs {
  Pool pool;
  Turn turn;
  const int32_t* rows;      // null: token t belongs to row t
  const int32_t* index;
  const int32_t* positions;
  int n_rows, n_tokens, n_q;
  Heads q, k, v;
  void* q_out;
  int64_t q_out_token_stride, q_out_head_stride;
};

struct DecodeArgs {
  Pool pool;
  const int32_t* lens;
  int batch, n_q, group;
  Heads q;
  float scale, cap;
  int window;
  const float* slopes;
  const float* prior_out;
  const float* prior_lse;
  float* out;
  float* lse;
  float* ws;
  int num_sms;
  bool whole;               // every segment to one CTA: nothing to join (set by the launcher)
};

struct GatherArgs {
  Pool pool;
  int n_rows, first, n_tokens;
  const int32_t* lens;
  void* k_out;
  void* v_out;
};

// Page pairs of one copy launch, in the kernel's parameters.
template <int N>
struct CopyPairs {
  int2 pair[N];             // (source, destination)
};

cudaError_t launch_append(int dtype, const AppendArgs& a, cudaStream_t st);
size_t decode_workspace(int num_sms);
cudaError_t launch_decode(int dtype, const DecodeArgs& a, cudaStream_t st);
// pairs: host (source, destination) ids, checked
cudaError_t launch_copy(void* pages, size_t page_bytes, int n_layers, size_t layer_stride, const int32_t* pairs,
                        int n_pairs, cudaStream_t st);
cudaError_t launch_gather(const GatherArgs& a, cudaStream_t st);

}  // namespace paged
}  // namespace aatc
