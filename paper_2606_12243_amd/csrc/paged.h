// The paged-cache operators (via_paged_*): arguments of their kernels, the
// geometry both sides agree on, and the launch wrappers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace via {

// Pages, sequences and rows of a call (via_paged), with the layer slot folded
// into the pool's address.
struct PagedRef {
  void* pool;  // pages of the call's layer slot: [kv_head][block][K|V][page]
  int n_blocks, KVH;
  const int32_t* table;  // [n_seqs][table_ld]
  int table_ld, n_seqs;
  const int32_t* row_start;  // [n_seqs + 1]
  const int32_t* kv_len;     // [n_seqs]
  int rows;                  // rows of the row arrays
  int cap;                   // cache positions a call looks at: min(max_kv, table_ld * kBlock, 2^30)
  int pages;                 // table entries that these are in
};

struct AppendArgs {
  PagedRef c;
  const void* qkv;
  int qkv_ld, H, hd;
  const int32_t* pos;  // nullable
  const void *q_gain, *k_gain;  // nullable
  float eps;
  void* q_out;
  int q_ld;
  double turn[64];  // rotations per position of pair i, in whole turns: theta^(-2i/hd) / (2 pi)
};

// Queries of one work-group of the streaming attention kernel: (row, head of
// the group) pairs, one column block of the matrix instruction.
constexpr int kPagedQueries = 32;
// ... and of the kernel for many rows.
constexpr int kPagedTileQueries = 128;
// Keys whose pages a work-group looks up at a time.
constexpr int kPagedChunk = 4096;

struct PagedAttnArgs {
  PagedRef c;
  const void* q;
  int q_ld, H, hd;
  float scale;
  int window;               // 0: none
  const uint64_t* row_mask;  // nullable
  // listed blocks (null: every key): sel[row][kv_head][n_sel], blocks of `block` keys
  const int32_t* sel;
  int n_sel, block;
  void* out;
  int out_ld;
  float* lse;  // nullable, [rows][H]
  // keys of a split (of the listed keys, or from the tile's first visible key on) and
  // the splits a launch has; one split writes the output itself
  int span, n_splits;
  int n_items;  // tiles a launch covers per K/V head
  int tile_q;   // queries of a tile: kPagedQueries or kPagedTileQueries
  int terms;    // bf16 values that a weight is held to in the latter
  float* part_o;   // [n_splits][rows][H][hd]
  float* part_ml;  // [n_splits][rows][H][2]: maximum (log2 units), sum
};

struct MeansArgs {
  PagedRef c;
  int hd, block;
  float* means;  // [n_seqs][KVH][max_blocks][hd]
  int max_blocks;
};

struct SelectArgs {
  PagedRef c;
  const void* q;
  int q_ld, H, hd;
  const float* means;
  int max_blocks, block, n_first, n_last, n_sel;
  int32_t* sel;      // [rows][KVH][n_sel]
  uint64_t* scores;  // workspace [rows][KVH][nb]: sortable scores
  int nb;            // blocks a row may see: ceil(cap / block), at most max_blocks
};

void launch_paged_append(bool bf16, const AppendArgs& a, hipStream_t s);
void launch_paged_attention(bool bf16, const PagedAttnArgs& a, hipStream_t s);
void launch_paged_means(bool bf16, const MeansArgs& a, hipStream_t s);
void launch_paged_select(bool bf16, const SelectArgs& a, hipStream_t s);

#ifdef __HIPCC__
// Rows [first, first + n) of sequence s.  Values that are not ascending row
// numbers give empty or overlapping ranges, never rows outside the arrays.
__device__ __forceinline__ void seq_rows(const PagedRef& c, int s, int& first, int& n) {
  first = min(max(c.row_start[s], 0), c.rows);
  n = min(max(c.row_start[s + 1], first), c.rows) - first;
}

__device__ __forceinline__ int seq_len(const PagedRef& c, int s) { return max(c.kv_len[s], 0); }

// The last sequence whose number base(s) is not above `item` (both uniform over the
// wave, base ascending), -1 if none: lanes look at 64 sequences over the whole range,
// then at those between two of them.  (Sequence after sequence, 64 at a time, took 0.8 us
// for every 64: with 1024 of them, 13 us at the start of every work-group.)
template <typename F>
__device__ __forceinline__ int last_seq(const PagedRef& c, int item, F base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, span = c.n_seqs;
  for (;;) {
    const int stride = (span + 63) >> 6;
    const uint64_t m = __ballot(lane * stride < span && base(lo + lane * stride) <= item);
    if (!m) return -1;
    const int at = (63 - __clzll((long long)m)) * stride;
    lo += at;
    if (stride <= 1) return lo;
    span = min(stride, span - at);
  }
}
__device__ __forceinline__ int first_row(const PagedRef& c, int s) { return min(max(c.row_start[s], 0), c.rows); }

// The sequence of row t (uniform over the wave).  -1: no sequence has it.
__device__ __forceinline__ int seq_of_row(const PagedRef& c, int t) {
  const int s = last_seq(c, t, [&](int i) { return first_row(c, i); });
  if (s < 0) return -1;
  int first, n;
  seq_rows(c, s, first, n);
  return t - first < n ? s : -1;
}

// Work items are numbered so that a sequence's first one is known from its first row
// alone: sequence s with rows [first, first + n) has items from first * units / per +
// extra * s on.  With `extra` 1 that is room for ceil(n * units / per) of them, or for the
// blocks of `per` rows that end among n (units 1); a launch covers rows * units / per +
// extra * n_seqs, and an item past what its sequence has does nothing.  rows * units is
// below 2^31.  Returns false where no sequence has the item.
__device__ __forceinline__ bool item_of(const PagedRef& c, int item, int units, int per, int extra, int& seq, int& no) {
  auto base = [&](int s) { return first_row(c, s) * units / per + extra * s; };
  seq = last_seq(c, item, base);
  if (seq < 0) return false;
  no = __builtin_amdgcn_readfirstlane(item - base(seq));
  return true;
}

// seq_rows and seq_len of a sequence that is the same in all lanes, as scalars.
__device__ __forceinline__ void seq_of_wave(const PagedRef& c, int s, int& first, int& n, int& len) {
  seq_rows(c, s, first, n);
  first = __builtin_amdgcn_readfirstlane(first);
  n = __builtin_amdgcn_readfirstlane(n);
  len = __builtin_amdgcn_readfirstlane(seq_len(c, s));
}

// Lets the matrix instructions before it finish (16 passes at most, 19 wait states).
// Their results may not be read earlier, and the compiler counts the wait states
// too low where the read is in another basic block that several paths lead to
// (fp32 scores after the branch around the masks: the last one was read 7
// states after the instruction and was wrong).
__device__ __forceinline__ void settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3");
  __builtin_amdgcn_sched_barrier(0);
}

// Page of a sequence's positions 16 i .. 16 i + 15; -1 where the table names
// none, which every kernel leaves alone.
__device__ __forceinline__ int page_of(const PagedRef& c, int seq, int i) {
  if (i < 0 || i >= c.pages) return -1;
  const int p = c.table[(size_t)seq * c.table_ld + i];
  return p >= 0 && p < c.n_blocks ? p : -1;
}
#endif

}  // namespace via
