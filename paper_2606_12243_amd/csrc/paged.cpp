// Entry points of the paged-cache operators (via_paged_*): argument checks,
// the split of the attention over work-groups, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/via.h"
#include "host_book.h"
#include "paged.h"

using namespace via;

namespace {

constexpr int kMaxPositions = 1 << 30;  // cache positions of a sequence
constexpr int kMaxSeqs = 65535;         // a grid's extent
constexpr int kMaxRows = 1 << 27;       // of a call
constexpr long long kMaxGroups = 1 << 24;  // work-groups of 256 threads in a launch (2^32 threads)
constexpr int kMaxSplits = 64;

int esize(const via_paged* c) { return c->dtype == VIA_DTYPE_BF16 ? 2 : 4; }
bool misaligned(const void* p) { return (uintptr_t)p % 16 != 0; }
bool block_ok(int block) { return block == 32 || block == 64 || block == 128; }

// Cache positions a call looks at.
int cap_of(const via_paged* c) {
  return (int)std::min<long long>({c->max_kv, (long long)c->table_ld * kBlock, kMaxPositions});
}

// Sizes of a via_paged alone (what the workspace functions need).
via_status check_sizes(const via_paged* c) {
  if (!c) return fail(VIA_EINVAL, "null via_paged");
  if (c->dtype != VIA_DTYPE_F32 && c->dtype != VIA_DTYPE_BF16) return fail(VIA_EINVAL, "dtype %d", c->dtype);
  if (c->n_slots < 1 || c->n_blocks < 1 || c->n_kv_heads < 1 || c->table_ld < 1)
    return fail(VIA_EINVAL, "n_slots, n_blocks, n_kv_heads and table_ld must be positive");
  if (c->n_seqs < 0 || c->rows < 0 || c->max_kv < 0) return fail(VIA_EINVAL, "n_seqs, rows and max_kv must not be negative");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(VIA_EUNSUPPORTED, "head_dim %d (64 and 128 run)", c->head_dim);
  if (c->rows > kMaxRows) return fail(VIA_EUNSUPPORTED, "more than %d rows", kMaxRows);
  if (c->n_seqs > kMaxSeqs || c->n_kv_heads > kMaxSeqs)
    return fail(VIA_EUNSUPPORTED, "more than %d sequences or K/V heads", kMaxSeqs);
  return VIA_OK;
}

// The whole of it, for a call that works on layer slot `slot`.
via_status check(const via_paged* c, int slot) {
  if (via_status st = check_sizes(c)) return st;
  if (slot < 0 || slot >= c->n_slots) return fail(VIA_EINVAL, "layer slot %d of %d", slot, c->n_slots);
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;  // nothing will be read
  if (!c->pool || !c->table || !c->row_start || !c->kv_len) return fail(VIA_EINVAL, "null pointer in via_paged");
  if (misaligned(c->pool)) return fail(VIA_EINVAL, "the pool must be 16-byte aligned");
  return VIA_OK;
}

// Row-major rows of n_heads heads.
via_status check_rows(const via_paged* c, const char* what, const void* p, int ld, long long heads) {
  if (!p) return fail(VIA_EINVAL, "%s is null", what);
  if (ld < heads * c->head_dim) return fail(VIA_EINVAL, "%s rows of %d elements hold no %lld heads", what, ld, heads);
  if (misaligned(p) || (long long)ld * esize(c) % 16)
    return fail(VIA_EINVAL, "%s and its rows must be 16-byte aligned", what);
  return VIA_OK;
}
via_status check_heads(const via_paged* c, int n_heads) {
  if (n_heads < 1 || n_heads % c->n_kv_heads)
    return fail(VIA_EINVAL, "n_heads %d must be a positive multiple of n_kv_heads %d", n_heads, c->n_kv_heads);
  return VIA_OK;
}

PagedRef ref_of(const via_paged* c, int slot) {
  PagedRef r{};
  const size_t layer = (size_t)c->n_kv_heads * c->n_blocks * 2 * kBlock * c->head_dim * esize(c);
  r.pool = (char*)c->pool + (size_t)slot * layer;
  r.n_blocks = c->n_blocks;
  r.KVH = c->n_kv_heads;
  r.table = c->table;
  r.table_ld = c->table_ld;
  r.n_seqs = c->n_seqs;
  r.row_start = c->row_start;
  r.kv_len = c->kv_len;
  r.rows = c->rows;
  r.cap = cap_of(c);
  r.pages = ceil_div(r.cap, kBlock);
  return r;
}

via_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? VIA_OK : fail(VIA_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

// How the attention's keys are split over work-groups.  Where the tiles of all
// K/V heads are fewer than kTargetGroups, each tile's keys are cut into spans of at
// least kMinSpan (of many-row tiles kMinTileSpan), up to kMaxSplits of them.
constexpr int kTargetGroups = 512;
constexpr int kMinSpan = 128;
constexpr int kMinTileSpan = 256;
// Several sequences are cut into spans of at most kMaxSpan keys besides (or kMaxSplits
// spans), however many tiles they have: they may differ, and a short batch's long one
// must not run on its own at the end.  The host knows only their bound, so this stops
// where its partial results would take more than kPartBytes (of n_splits times rows
// times heads; splits of the first kind take 34 MB at most) or its launch more
// work-groups than there can be.  With and without that limit (bf16, 32 heads of 128 on 8): 8 x 1000
// rows of 2000 keys, bound 131072, 442 and 828 us; 2 x 8192 of 16384, same bound, 3025 and 6791
// (0 and 4.1 GiB); 8 x 1000 of 32768 4389 and 4369; of 64 x 100 rows one of 60000 keys, the
// others of 500, 686 and 507.
constexpr int kMaxSpan = 8192;
constexpr long long kPartBytes = 256ll << 20;
struct Split {
  long long n_items;  // tiles a launch covers per K/V head
  int span, n_splits, tile_q, terms;
};
// Queries of a K/V head and sequence (rows times heads, on average over the sequences)
// from which a bf16 call takes the 128-query kernel: one more than the streaming
// kernel's 32 share of the keys (16 sequences of 8192 keys, 36 queries: 111 against 143 us;
// one of 4096: 18 both) ...
constexpr int kTileFrom = kPagedQueries + 1;
// ... and from which that holds its weights to one bf16 value.
constexpr int kOneTermFrom = 128;
Split split_of(const via_paged* c, int n_heads, int window, int n_sel, int block) {
  Split s{};
  const int G = n_heads / c->n_kv_heads;
  long long tiles, keys;  // tiles with work (about), keys of one
  if (n_sel > 0) {
    const int per_row = ceil_div(G, kPagedQueries);
    tiles = s.n_items = (long long)c->rows * per_row;
    keys = (long long)n_sel * block;
    s.tile_q = kPagedQueries;
  } else {
    const long long each = ((long long)c->rows + c->n_seqs - 1) / std::max(1, c->n_seqs);
    s.tile_q = c->dtype == VIA_DTYPE_BF16 && each * G >= kTileFrom ? kPagedTileQueries : kPagedQueries;
    s.terms = each * G >= kOneTermFrom ? 1 : 2;
    s.n_items = (long long)c->rows * G / s.tile_q + c->n_seqs;
    tiles = (each * G + s.tile_q - 1) / s.tile_q * c->n_seqs;
    keys = cap_of(c);
    // rows of a tile and the keys they look back on
    if (window > 0) keys = std::min<long long>(keys, (long long)window + s.tile_q / G + 32);
  }
  const long long groups = std::max<long long>(1, tiles * c->n_kv_heads);
  const long long want = std::min<long long>(std::max<long long>(1, kTargetGroups / groups), kMaxSplits);
  long long span = (keys + want - 1) / want;
  if (c->n_seqs > 1 && n_sel == 0) {
    // (of a split; as many rows times heads as are refused count as that)
    const long long part = std::clamp((long long)c->rows * n_heads, 1ll, kMaxGroups) * (c->head_dim + 2) * 4;
    const long long most = std::min({(long long)kMaxSplits, kPartBytes / part, (kMaxGroups - 1) / (s.n_items * c->n_kv_heads)});
    if (most > 1) span = std::min(span, std::max<long long>(kMaxSpan, (keys + most - 1) / most));
  }
  span = std::max<long long>(span, s.tile_q == kPagedQueries ? kMinSpan : kMinTileSpan);
  span = (span + 127) / 128 * 128;  // four waves' blocks
  s.span = (int)span;
  s.n_splits = (int)std::max<long long>(1, (keys + span - 1) / span);
  return s;
}
size_t split_bytes(const via_paged* c, int n_heads, const Split& s) {
  return s.n_splits > 1 ? (size_t)s.n_splits * c->rows * n_heads * (c->head_dim + 2) * 4 : 0;
}

via_status attention(const via_paged* c, int slot, PagedAttnArgs& a, void* workspace, size_t workspace_bytes,
                     void* stream, const char* what) {
  const Split s = split_of(c, a.H, a.window, a.sel ? a.n_sel : 0, a.block);
  if (s.n_items * c->n_kv_heads * s.n_splits >= kMaxGroups || (long long)c->rows * a.H >= kMaxGroups)
    return fail(VIA_EUNSUPPORTED, "%d rows of %d heads are more than one launch covers", c->rows, a.H);
  const size_t need = split_bytes(c, a.H, s);
  if (need && (!workspace || workspace_bytes < need))
    return fail(VIA_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (need && (uintptr_t)workspace % 256) return fail(VIA_EINVAL, "the workspace must be 256-byte aligned");
  a.c = ref_of(c, slot);
  a.hd = c->head_dim;
  a.span = s.span;
  a.n_splits = s.n_splits;
  a.n_items = (int)s.n_items;
  a.tile_q = s.tile_q;
  a.terms = s.terms;
  a.part_o = (float*)workspace;
  a.part_ml = (float*)workspace + (size_t)s.n_splits * c->rows * a.H * c->head_dim;
  launch_paged_attention(c->dtype == VIA_DTYPE_BF16, a, (hipStream_t)stream);
  return launched(what);
}

via_status check_attention(const via_paged* c, int slot, const void* q, int q_ld, int n_heads, float scale,
                           const void* out, int out_ld) {
  if (via_status st = check(c, slot)) return st;
  if (via_status st = check_heads(c, n_heads)) return st;
  if (!std::isnormal(scale) || !(scale > 0.f)) return fail(VIA_EINVAL, "scale must be positive and finite");
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  if (via_status st = check_rows(c, "q", q, q_ld, n_heads)) return st;
  if (via_status st = check_rows(c, "out", out, out_ld, n_heads)) return st;
  return out == q && out_ld != q_ld ? fail(VIA_EINVAL, "out over q must have its row length") : VIA_OK;
}

}  // namespace

extern "C" {

via_status via_paged_append(const via_paged* c, int32_t slot, const void* qkv, int32_t qkv_ld, int32_t n_heads,
                            const int32_t* pos, const void* q_gain, const void* k_gain, float eps, float theta,
                            void* q_out, int32_t q_ld, void* stream) {
  if (via_status st = check(c, slot)) return st;
  if (via_status st = check_heads(c, n_heads)) return st;
  if (!(theta > 0.f) || !std::isfinite(theta)) return fail(VIA_EINVAL, "theta must be positive and finite");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(VIA_EINVAL, "eps must not be negative");
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  if (via_status st = check_rows(c, "qkv", qkv, qkv_ld, (long long)n_heads + 2 * c->n_kv_heads)) return st;
  if (via_status st = check_rows(c, "q_out", q_out, q_ld, n_heads)) return st;
  if (q_out == qkv && q_ld != qkv_ld) return fail(VIA_EINVAL, "q_out over qkv must have its row length");
  AppendArgs a{};
  a.c = ref_of(c, slot);
  a.qkv = qkv;
  a.qkv_ld = qkv_ld;
  a.H = n_heads;
  a.hd = c->head_dim;
  a.pos = pos;
  a.q_gain = q_gain;
  a.k_gain = k_gain;
  a.eps = eps;
  a.q_out = q_out;
  a.q_ld = q_ld;
  // (products of long doubles: 64 calls of pow are 2 us of every call)
  const long double ratio = std::pow((long double)theta, -2.0L / c->head_dim);
  long double turn = 1.0L / 6.283185307179586476925286766559L;
  for (int i = 0; i < c->head_dim / 2; ++i, turn *= ratio) a.turn[i] = (double)turn;
  launch_paged_append(c->dtype == VIA_DTYPE_BF16, a, (hipStream_t)stream);
  return launched("append");
}

size_t via_paged_attend_bytes(const via_paged* c, int32_t n_heads, int32_t window) {
  if (check_sizes(c) || check_heads(c, n_heads) || window < 0) return 0;
  return split_bytes(c, n_heads, split_of(c, n_heads, window, 0, 0));
}

via_status via_paged_attend(const via_paged* c, int32_t slot, const void* q, int32_t q_ld, int32_t n_heads, float scale,
                            int32_t window, const uint64_t* row_mask, void* out, int32_t out_ld, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream) {
  if (via_status st = check_attention(c, slot, q, q_ld, n_heads, scale, out, out_ld)) return st;
  if (window < 0) return fail(VIA_EINVAL, "window must not be negative");
  if (window > 0 && row_mask) return fail(VIA_EINVAL, "a window and row masks exclude each other");
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  PagedAttnArgs a{};
  a.q = q;
  a.q_ld = q_ld;
  a.H = n_heads;
  a.scale = scale;
  a.window = window;
  a.row_mask = row_mask;
  a.out = out;
  a.out_ld = out_ld;
  a.lse = lse;
  return attention(c, slot, a, workspace, workspace_bytes, stream, "attend");
}

via_status via_paged_block_means(const via_paged* c, int32_t slot, int32_t block, float* means, int32_t max_blocks,
                                 void* stream) {
  if (via_status st = check(c, slot)) return st;
  if (!block_ok(block)) return fail(VIA_EUNSUPPORTED, "blocks of %d tokens (32, 64 and 128 run)", block);
  if (max_blocks < 1) return fail(VIA_EINVAL, "max_blocks must be positive");
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  if (!means || misaligned(means)) return fail(VIA_EINVAL, "means must be given and 16-byte aligned");
  MeansArgs a{};
  a.c = ref_of(c, slot);
  a.hd = c->head_dim;
  a.block = block;
  a.means = means;
  a.max_blocks = max_blocks;
  if (a.c.cap < block) return VIA_OK;  // no sequence is long enough to complete a block
  launch_paged_means(c->dtype == VIA_DTYPE_BF16, a, (hipStream_t)stream);
  return launched("block means");
}

size_t via_paged_select_bytes(const via_paged* c, int32_t block) {
  if (check_sizes(c) || !block_ok(block)) return 0;
  return (size_t)c->rows * c->n_kv_heads * ceil_div(cap_of(c), block) * sizeof(uint64_t);
}

via_status via_paged_select(const via_paged* c, const void* q, int32_t q_ld, int32_t n_heads, const float* means,
                            int32_t max_blocks, int32_t block, int32_t n_first, int32_t n_last, int32_t n_sel,
                            int32_t* sel, void* workspace, size_t workspace_bytes, void* stream) {
  if (via_status st = check(c, 0)) return st;
  if (via_status st = check_heads(c, n_heads)) return st;
  if (!block_ok(block)) return fail(VIA_EUNSUPPORTED, "blocks of %d tokens (32, 64 and 128 run)", block);
  if (n_first < 0 || n_last < 1 || n_sel < 1 || (long long)n_first + n_last > n_sel)
    return fail(VIA_EINVAL, "need n_first >= 0, n_last >= 1 and n_first + n_last <= n_sel");
  if ((long long)c->rows * c->n_kv_heads >= kMaxGroups)
    return fail(VIA_EUNSUPPORTED, "%d rows of %d K/V heads are more than one launch covers", c->rows, c->n_kv_heads);
  const int nb = ceil_div(cap_of(c), block);
  if (max_blocks < 1 || max_blocks < nb) return fail(VIA_EINVAL, "means of %d blocks, sequences of %d", max_blocks, nb);
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  if (via_status st = check_rows(c, "q", q, q_ld, n_heads)) return st;
  if (!means || misaligned(means)) return fail(VIA_EINVAL, "means must be given and 16-byte aligned");
  if (!sel) return fail(VIA_EINVAL, "sel is null");
  const size_t need = via_paged_select_bytes(c, block);
  if (need && (!workspace || workspace_bytes < need))
    return fail(VIA_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (need && (uintptr_t)workspace % 256) return fail(VIA_EINVAL, "the workspace must be 256-byte aligned");
  SelectArgs a{};
  a.c = ref_of(c, 0);
  a.q = q;
  a.q_ld = q_ld;
  a.H = n_heads;
  a.hd = c->head_dim;
  a.means = means;
  a.max_blocks = max_blocks;
  a.block = block;
  a.n_first = n_first;
  a.n_last = n_last;
  a.n_sel = n_sel;
  a.sel = sel;
  a.scores = (uint64_t*)workspace;
  a.nb = nb;
  launch_paged_select(c->dtype == VIA_DTYPE_BF16, a, (hipStream_t)stream);
  return launched("select");
}

size_t via_paged_attend_blocks_bytes(const via_paged* c, int32_t n_heads, int32_t block, int32_t n_sel) {
  if (check_sizes(c) || check_heads(c, n_heads) || !block_ok(block) || n_sel < 1) return 0;
  return split_bytes(c, n_heads, split_of(c, n_heads, 0, n_sel, block));
}

via_status via_paged_attend_blocks(const via_paged* c, int32_t slot, const void* q, int32_t q_ld, int32_t n_heads,
                                   float scale, int32_t block, const int32_t* sel, int32_t n_sel, void* out,
                                   int32_t out_ld, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (via_status st = check_attention(c, slot, q, q_ld, n_heads, scale, out, out_ld)) return st;
  if (!block_ok(block)) return fail(VIA_EUNSUPPORTED, "blocks of %d tokens (32, 64 and 128 run)", block);
  if (n_sel < 1 || n_sel > kMaxPositions / block) return fail(VIA_EINVAL, "n_sel %d", n_sel);
  if (c->rows == 0 || c->n_seqs == 0) return VIA_OK;
  if (!sel) return fail(VIA_EINVAL, "sel is null");
  PagedAttnArgs a{};
  a.q = q;
  a.q_ld = q_ld;
  a.H = n_heads;
  a.scale = scale;
  a.sel = sel;
  a.n_sel = n_sel;
  a.block = block;
  a.out = out;
  a.out_ld = out_ld;
  a.lse = lse;
  return attention(c, slot, a, workspace, workspace_bytes, stream, "attend blocks");
}

}  // extern "C"
