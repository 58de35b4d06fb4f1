// Operators around the attention over a paged cache: rows entering it
// (via_paged_append), mean keys of its blocks (via_paged_block_means) and the
// choice of blocks for each row (via_paged_select).
#include <algorithm>

#include "paged.h"

namespace via {

namespace {

// ---------------------------------------------------------------------------
// Rows entering the cache.  Each head of q and k: y = x g / sqrt(mean x^2 + eps)
// where gains are given, then the pairs (i, i + hd/2) turned by pos theta^(-2i/hd);
// v as it is.  Bound by memory: a value is read and written once.
//
// A work-group takes the rows that enter one page of a sequence (at most 16) and
// some of their heads, q, k and v in one list.  A team of 16 lanes holds a token's
// head of 128 (or two of 64), 8 dims a lane, so a head's sum of
// squares and a dim's partner are lane exchanges, and q and k go out 16 bytes a
// thread or more.  More than 8 rows have a team for each of the page's tokens, and V,
// transposed in its page, goes through LDS and out as 8 tokens of a dim a thread, a
// whole page's in one piece.  Where fewer rows enter, as in single-token steps, the
// teams share out the heads instead.
//
// Angles are whole turns in fp64, pos * (theta^(-2i/hd) / 2 pi), of which only the
// fraction is kept: fp32 would lose it at far positions (2^-24 of 10^5 turns).
// Norms and rotations are fp32, rounded once where they are stored.
__device__ __forceinline__ float ror8(float x) {  // from lane ^ 8 (of 16)
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xF, 0xF, true));
}
// x of the lane's partner, half a head (TPH / 2 lanes) away
template <int TPH>
__device__ __forceinline__ float partner(float x) {
  return TPH == 16 ? ror8(x) : __shfl_xor(x, TPH / 2, 64);
}
// sum over the TPH (8 or 16) lanes of a head: quad_perm exchanges 1 and 2 lanes
// away, then the other quad (half mirror) and the other half (rotate by 8)
template <int TPH>
__device__ __forceinline__ float head_sum(float x) {
  x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true));
  x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, true));
  x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, true));
  return TPH == 16 ? x + ror8(x) : x;
}

// Page `item` (uniform over the wave) of those that the sequences' rows enter, at most n / 16
// + 2 of n rows: its sequence and position / 16 (pages of positions below 0 included: their
// rows only have queries).  Up to 64 sequences' pages are counted one after another,
// which leaves no items without work in between: with them some compute units get more
// work-groups than others (16 prompts of 500 rows 55 against 47 us).  More are
// searched (1024 single tokens 19 against 51 us with counting); a page behind the last one has no
// work.
__device__ __forceinline__ bool page_of_item(const PagedRef& c, int item, int& seq, int& page) {
  if (c.n_seqs > 64) {
    if (!item_of(c, item, 1, 16, 2, seq, page)) return false;
    int first, n, len;
    seq_of_wave(c, seq, first, n, len);
    page += (len - n) >> 4;
    return true;
  }
  const int lane = threadIdx.x & 63;
  int first = 0, n = 0, len = 0;
  if (lane < c.n_seqs) {
    seq_rows(c, lane, first, n);
    len = seq_len(c, lane);
  }
  const int p0 = (len - n) >> 4, pages = n > 0 ? ((len - 1) >> 4) - p0 + 1 : 0;
  int end = pages;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(end, o, 64);
    if (lane >= o) end += v;
  }
  const uint64_t m = __ballot(item < end);
  if (!m) return false;
  seq = __ffsll((unsigned long long)m) - 1;
  page = __builtin_amdgcn_readlane(p0, seq) + item - (__builtin_amdgcn_readlane(end, seq) - __builtin_amdgcn_readlane(pages, seq));
  return true;
}

// 8 values as floats, and back
template <typename T>
struct Eight {
  uint4 v[sizeof(T) == 2 ? 1 : 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) v[i] = ((const uint4*)p)[i];
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    } else {
      const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
    }
  }
};
__device__ __forceinline__ void store8(uint16_t* p, const float (&y)[8]) {
  *(uint4*)p = make_uint4(pack_bf16x2(f2bf(y[0]), f2bf(y[1])), pack_bf16x2(f2bf(y[2]), f2bf(y[3])),
                          pack_bf16x2(f2bf(y[4]), f2bf(y[5])), pack_bf16x2(f2bf(y[6]), f2bf(y[7])));
}
__device__ __forceinline__ void store8(float* p, const float (&y)[8]) {
  *(float4*)p = make_float4(y[0], y[1], y[2], y[3]);
  *(float4*)(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
}

template <typename T, int HD, bool NORM>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int TPH = HD / 8, HPP = 16 / TPH, HALF = HD / 2;  // threads of a row per head; heads per pass
  constexpr int kVec = 16 / sizeof(T);                        // tokens of a dim a thread stores
  constexpr int kStride = 16 + kVec;                          // of a dim in LDS (no bank conflicts on reading)
  __shared__ __align__(16) T vt[HPP * HD * kStride];
  const int l = threadIdx.x & 15, d0 = (l % TPH) * 8, team = threadIdx.x >> 4;
  int seq, page_no, first, n, len;
  if (!page_of_item(a.c, blockIdx.x, seq, page_no)) return;
  seq_of_wave(a.c, seq, first, n, len);
  if (n == 0 || page_no > (len - 1) >> 4) return;
  const int slot0 = page_no * 16;
  // the page's tokens t0 .. t1 - 1 are rows of the call: `rows` teams take them (or the whole page), the others
  // further heads
  const int t0 = max(len - n - slot0, 0), t1 = min(len - slot0, 16);
  const int bits = t1 - t0 > 8 ? 4 : t1 - t0 > 4 ? 3 : t1 - t0 > 2 ? 2 : t1 - t0 - 1, rows = 1 << bits;
  const int t = (rows == 16 ? 0 : t0) + (team & (rows - 1)), sub = (team >> bits) * HPP + l / TPH;
  const bool live = t >= t0 && t < t1;
  const int pos0 = slot0 + min(max(t, t0), t1 - 1), row = first + pos0 - (len - n);  // the thread's position and row
  const bool cached = slot0 >= 0 && pos0 < a.c.cap;
  const int page = slot0 >= 0 ? __builtin_amdgcn_readfirstlane(page_of(a.c, seq, page_no)) : -1;
  const int heads = a.H + 2 * a.c.KVH, width = HPP * 16 >> bits;  // heads a pass takes
  // the work-group's passes y, y + gridDim.y, ..., from another one in every work-group: rows whose length is a
  // multiple of 4 KiB would have all of them read the same memory channels
  const int passes = ((heads + width - 1) / HPP >> (4 - bits)) - (int)blockIdx.y;
  const int count = passes > 0 ? (passes + gridDim.y - 1) / gridDim.y : 0;
  if (count == 0) return;
  int at = blockIdx.x % count;
  const T* src = (const T*)a.qkv + (size_t)row * a.qkv_ld + d0;
  Eight<T> next;
  auto head_of = [&](int i) { return ((int)blockIdx.y + i * (int)gridDim.y) * width; };
  next.load(src + (size_t)min(head_of(at) + sub, heads - 1) * HD);
  const bool low = d0 < HALF;
  float cs[8], sn[8], qg[8], kg[8];
  {
    const double pos = (double)(a.pos ? a.pos[row] : pos0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = pos * a.turn[d0 % HALF + e];
      const float f = (float)(turns - rint(turns));
      if constexpr (sizeof(T) == 2) {
        // the hardware's, 2^-22.9 off at most over a turn (measured): far below a bf16 step
        sn[e] = __builtin_amdgcn_sinf(f);
        cs[e] = __builtin_amdgcn_cosf(f);
      } else {
        sincospif(2.f * f, &sn[e], &cs[e]);
      }
      if (low) sn[e] = -sn[e];
    }
  }
  if (NORM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      qg[e] = a.q_gain ? to_f<T>(((const T*)a.q_gain)[d0 + e]) : 0.f;
      kg[e] = a.k_gain ? to_f<T>(((const T*)a.k_gain)[d0 + e]) : 0.f;
    }
  }
  for (int i = 0; i < count; ++i) {
    const int h0 = head_of(at), h = h0 + sub;
    at = at + 1 == count ? 0 : at + 1;
    float x[8];
    next.floats(x);
    if (i + 1 < count) next.load(src + (size_t)min(head_of(at) + sub, heads - 1) * HD);
    if (h0 < a.H + a.c.KVH) {  // uniform: q or k heads
      if (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        ss = head_sum<TPH>(ss);
        const float sc = 1.0f / sqrtf(ss / (float)HD + a.eps);
        const bool norm = h < a.H ? a.q_gain != nullptr : a.k_gain != nullptr && h < a.H + a.c.KVH;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float gq = qg[e], gk = kg[e];
          x[e] = norm ? x[e] * sc * (h < a.H ? gq : gk) : x[e];
        }
      }
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e] * cs[e] + partner<TPH>(x[e]) * sn[e];
      if (live && h < a.H)
        store8((T*)a.q_out + (size_t)row * a.q_ld + (size_t)h * HD + d0, y);
      else if (live && cached && page >= 0 && h < a.H + a.c.KVH)
        store8((T*)a.c.pool + k_off(0, page, a.c.n_blocks, a.c.KVH, HD, h - a.H, t, d0), y);
    }
    if (rows < 16) {
      const int g = h - a.H - a.c.KVH;
      if (g >= 0 && g < a.c.KVH && live && cached && page >= 0) {
        T* to = (T*)a.c.pool + v_off(0, page, a.c.n_blocks, a.c.KVH, HD, g, t, d0);
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e * kBlock] = from_f<T>(x[e]);
      }
    } else if (h0 + HPP > a.H + a.c.KVH) {  // uniform: v heads of a whole page
      const int g0 = h0 - a.H - a.c.KVH, end = min(t1, a.c.cap - slot0);
#pragma unroll
      for (int e = 0; e < 8; ++e) vt[(l / TPH * HD + d0 + e) * kStride + t] = from_f<T>(x[e]);
      __syncthreads();
      if (page >= 0) {
        for (int i = threadIdx.x; i < HPP * HD * 16 / kVec; i += 256) {
          const int d = i * kVec / 16, from = i * kVec % 16, g = g0 + d / HD;
          if (g < 0 || g >= a.c.KVH) continue;
          const T* v = &vt[d * kStride + from];
          T* to = (T*)a.c.pool + v_off(0, page, a.c.n_blocks, a.c.KVH, HD, g, from, d % HD);
          if (t0 <= from && from + kVec <= end) {
            *(uint4*)to = *(const uint4*)v;
          } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (from + e >= t0 && from + e < end) to[e] = v[e];
          }
        }
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Mean keys of the blocks a batch's rows complete: block b of a sequence where
// (kv_len - n) / block <= b < kv_len / block.  Bound by reading the K pages.  A wave a
// (block, K/V head): lane t reads dim group t / 16 of token t % 16, pages one
// after another, and the 16 tokens' sums meet by lane exchanges.  Sums are fp32
// (at most 128 terms).
template <typename T, int HD>
__global__ __launch_bounds__(64) void paged_means_kernel(MeansArgs a) {
  const int g = blockIdx.y, lane = threadIdx.x;
  int seq, no, first, n, all;
  if (!item_of(a.c, blockIdx.x, 1, a.block, 1, seq, no)) return;
  seq_of_wave(a.c, seq, first, n, all);
  const int len = min(all, a.c.cap), old = max(all - n, 0);
  const int b = old / a.block + no;
  if (b >= len / a.block || b >= a.max_blocks) return;
  float acc[HD / 32][8];
#pragma unroll
  for (int j = 0; j < HD / 32; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[j][e] = 0.f;
  const int pages = a.block / kBlock;
  bool whole = true;
  for (int i = 0; i < pages; ++i) {
    const int page = page_of(a.c, seq, b * pages + i);
    whole &= page >= 0;
    if (page < 0) continue;
    const T* kp = (const T*)a.c.pool + k_off(0, page, a.c.n_blocks, a.c.KVH, HD, g, 0, 0);
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      const T* p = kp + (size_t)(j * 64 + lane) * 8;  // dim group 4 j + lane / 16, token lane % 16
      if constexpr (sizeof(T) == 2) {
        const uint4 v = *(const uint4*)p;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[j][2 * e] += __uint_as_float(w[e] << 16);
          acc[j][2 * e + 1] += __uint_as_float(w[e] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[j][e] += p[e];
      }
    }
  }
  if (!whole) return;  // a block with an absent page keeps its mean as it was
  float* dst = a.means + (((size_t)seq * a.c.KVH + g) * a.max_blocks + b) * HD;
  const float inv = 1.0f / (float)a.block;
#pragma unroll
  for (int j = 0; j < HD / 32; ++j) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) acc[j][e] += __shfl_xor(acc[j][e], o, 64);
    if ((lane & 15) < 2) {
      const int e = (lane & 1) * 4, d = (j * 4 + (lane >> 4)) * 8 + e;
      const float* x = acc[j];
      *(float4*)(dst + d) = e ? make_float4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)
                              : make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    }
  }
}

// ---------------------------------------------------------------------------
// The choice of blocks.  Score of block b for a row and K/V head: the dot product
// of the group's summed queries with the block's mean key, in fp64: a chosen
// block is a whole number, and fp32 sums would choose another where two scores
// nearly tie.  A row at position p sees blocks 0 .. p / block; the first n_first and
// the last n_last of them are kept, and of the others the highest scores, ties
// to the lower block, until n_sel are chosen.
//
// Two kernels.  The first scores: a work-group takes 16 rows of a sequence, one
// K/V head and some of the blocks, sums the queries into LDS and lets each wave take
// 16 blocks at a time with v_mfma_f64_16x16x4_f64.  A score is kept as 64 bits that order
// like it.  The second chooses, a wave a (row, K/V head): it holds the upper halves of
// the row's scores in registers and finds the n_sel-th largest bit by bit, which
// ends as soon as n_sel of them are as large; lower halves are read only where upper
// ones tie.  (One kernel for both left half the card idle on few rows, and the
// scores' registers kept the choice from running beside them on many.)
// Work-groups a launch aims for: fewer, with more blocks each, share the queries'
// sums and the wait for them among more products.
constexpr int kScoreGroups = 1024;
constexpr int kSelectHeld = 32;  // scores a lane holds: rows of up to 64 * kSelectHeld blocks
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef double f64x2 __attribute__((ext_vector_type(2)));

// order of the doubles as unsigned numbers; NaN lowest, its upper half above 0
__device__ __forceinline__ uint64_t sortable(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  if (x != x) return 1ull << 32;
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// x[i] += the N values at p (16-byte aligned)
template <typename T, int N>
__device__ __forceinline__ void add_to(double (&x)[N], const T* p) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const uint4 v = *(const uint4*)(p + i);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[i + 2 * e] += (double)__uint_as_float(w[e] << 16);
        x[i + 2 * e + 1] += (double)__uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *(const float4*)(p + i);
      x[i] += (double)v.x;
      x[i + 1] += (double)v.y;
      x[i + 2] += (double)v.z;
      x[i + 3] += (double)v.w;
    }
  }
}

template <typename T, int HD>
__global__ __launch_bounds__(256, 4) void paged_score_kernel(SelectArgs a, int per) {
  constexpr int KS = HD / 4;  // k steps; lane l holds dims 16 i + 4 (l/16) .. + 3 of row or block l % 16
  constexpr int kRow = HD + 2;  // doubles of a row in LDS (rows 4 banks apart)
  __shared__ __align__(16) double sq[16 * kRow];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = blockIdx.y, m = lane & 15, kq = lane >> 4, G = a.H / a.c.KVH;
  int seq, tile, first, n, len;
  if (!item_of(a.c, blockIdx.x, 1, 16, 1, seq, tile)) return;
  seq_of_wave(a.c, seq, first, n, len);
  const int r0 = tile * 16;
  if (r0 >= n) return;
  const int rows = min(16, n - r0);
  // blocks the tile's last row sees (positions past the cap see what the last one does)
  const int last = min(max(len - n + r0 + rows - 1, -1), a.c.cap - 1);
  const int seen = last < 0 ? 0 : min(last / a.block + 1, a.nb);
  const int from = blockIdx.z * per, to = min(seen, from + per);
  if (from >= to) return;
  const float* means = a.means + ((size_t)seq * a.c.KVH + g) * (size_t)a.max_blocks * HD + kq * 4;
  float4 v[KS / 4];
  auto load = [&](int b0) {
    const float* p = means + (size_t)min(b0 + m, to - 1) * HD;
#pragma unroll
    for (int i = 0; i < KS / 4; ++i) v[i] = *(const float4*)(p + i * 16);
  };
  load(min(from + wave * 16, to - 1));
  {  // the group's summed queries: thread t has dims 8 (t % (HD / 8)) .. + 7 of rows t / (HD / 8), ...
    constexpr int TPR = HD / 8;
    for (int r = threadIdx.x / TPR; r < 16; r += 256 / TPR) {
      const int d = threadIdx.x % TPR * 8;
      double q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = 0.0;
      if (r < rows) {
        const T* p = (const T*)a.q + (size_t)(first + r0 + r) * a.q_ld + (size_t)g * G * HD + d;
        int h = 0;
        for (; h + 4 <= G; h += 4) {  // (four heads' loads together)
#pragma unroll
          for (int i = 0; i < 4; ++i) add_to<T, 8>(q, p + (size_t)(h + i) * HD);
        }
        for (; h < G; ++h) add_to<T, 8>(q, p + (size_t)h * HD);
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) *(f64x2*)&sq[r * kRow + d + i] = f64x2{q[i], q[i + 1]};
    }
  }
  __syncthreads();
  double q[KS];
#pragma unroll
  for (int i = 0; i < KS; i += 2) {
    const f64x2 x = *(const f64x2*)&sq[m * kRow + (i >> 2) * 16 + kq * 4 + (i & 3)];
    q[i] = x[0];
    q[i + 1] = x[1];
  }
  for (int b0 = from + wave * 16; b0 < to; b0 += 64) {
    f64x4 s = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int i = 0; i < KS / 4; ++i) {
      s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i], (double)v[i].x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 1], (double)v[i].y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 2], (double)v[i].z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 3], (double)v[i].w, s, 0, 0, 0);
    }
    settle();
    if (b0 + 64 < to) load(b0 + 64);
    // register i of lane l: row 4 i + l / 16, block l % 16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * i + kq;
      if (row < rows && b0 + m < to)
        a.scores[((size_t)(first + r0 + row) * a.c.KVH + g) * a.nb + b0 + m] = sortable(s[i]);
    }
  }
}

__global__ __launch_bounds__(256, 8) void paged_choose_kernel(SelectArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int item = blockIdx.x * 4 + wave, row = item / a.c.KVH, g = item % a.c.KVH;
  if (row >= a.c.rows) return;
  const int seq = seq_of_row(a.c, row);
  if (seq < 0) return;
  int first, n, len;
  seq_of_wave(a.c, seq, first, n, len);
  const int pos = min(len - n + row - first, a.c.cap - 1);
  const int vis = pos < 0 ? 0 : min(pos / a.block + 1, a.nb);
  const uint64_t* sc = a.scores + ((size_t)row * a.c.KVH + g) * a.nb;
  int32_t* out = a.sel + ((size_t)row * a.c.KVH + g) * a.n_sel;
  const int rounds = (vis + 63) >> 6;  // block of round j: 64 j + lane
  auto kept = [&](int b) { return b < a.n_first || b >= vis - a.n_last; };
  auto read = [&](int b) { return sc[min(b, vis - 1)]; };
  auto upper = [&](int b, uint64_t k) { return b >= vis ? 0u : kept(b) ? ~0u : (uint32_t)(k >> 32); };
  auto lower = [&](int b) { return kept(b) ? ~0u : (uint32_t)read(b); };
  uint32_t held[kSelectHeld];
#pragma unroll
  for (int j0 = 0; j0 < kSelectHeld; j0 += 8) {
    uint64_t k[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      held[j0 + j] = 0;
      if (j0 < rounds) k[j] = read((j0 + j) * 64 + lane);  // (eight reads in flight)
    }
    if (j0 < rounds) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        held[j0 + j] = upper((j0 + j) * 64 + lane, k[j]);
        __builtin_amdgcn_sched_barrier(0);  // (keeps the comparisons' masks few)
      }
    }
  }
  // f(round, upper half) for every round
  auto each = [&](auto f) {
#pragma unroll
    for (int j0 = 0; j0 < kSelectHeld; j0 += 4) {  // (past the last round they are 0)
      if (j0 >= rounds) break;
#pragma unroll
      for (int j = j0; j < j0 + 4; ++j) f(j, held[j]);
    }
    for (int j = kSelectHeld; j < rounds; ++j) f(j, upper(j * 64 + lane, read(j * 64 + lane)));
  };
  // chosen: upper halves above hi; of those equal to it, lower halves above lo, and the first `ties` equal to that
  uint32_t hi = 0, lo = ~0u;
  int ties = 0;
  if (vis > a.n_sel) {
    bool exact = false;
    for (int bit = 31; bit >= 0 && !exact; --bit) {
      const uint32_t t = hi | (1u << bit);
      int c = 0;
      each([&](int, uint32_t k) { c += __popcll(__ballot(k >= t)); });
      if (c >= a.n_sel) hi = t;
      exact = c == a.n_sel;
    }
    if (exact) {
      hi -= 1;
    } else {
      int above = 0;
      each([&](int, uint32_t k) { above += __popcll(__ballot(k > hi)); });
      const int want = a.n_sel - above;
      auto tied = [&](uint32_t t) {  // equal upper halves with lower ones >= t
        int l = lane, c = 0;
        asm volatile("" : "+v"(l));  // (recomputes the blocks: their masks would not fit the scalar registers)
        each([&](int j, uint32_t k) { c += __popcll(__ballot(k == hi && lower(j * 64 + l) >= t)); });
        return c;
      };
      lo = 0;
      for (int bit = 31; bit >= 0; --bit)
        if (tied(lo | (1u << bit)) >= want) lo |= 1u << bit;
      ties = want - (lo == ~0u ? 0 : tied(lo + 1));
    }
  }
  int done = 0;
  const uint64_t before = (1ull << lane) - 1;
  each([&](int j, uint32_t k) {
    const int b = j * 64 + lane;
    bool take = k > hi;  // (0 where the row sees no block)
    if (ties > 0 || lo != ~0u) {  // (uniform)
      const bool eq = k == hi;
      const uint32_t l = eq ? lower(b) : 0u;
      const uint64_t tied = __ballot(eq && l == lo);
      take |= eq && (l > lo || (l == lo && __popcll(tied & before) < ties));
      ties -= min(ties, __popcll(tied));
    }
    const uint64_t taken = __ballot(take);
    if (take) out[done + __popcll(taken & before)] = b;
    done += __popcll(taken);
  });
  for (int i = done + lane; i < a.n_sel; i += 64) out[i] = -1;
}

// Work-groups an append aims for, to the nearest count (4 x 2047 rows of 48 heads: 512 62 us,
// 1024 53, 2048 60; 4 x 1900: 47, 47, 58; 1 x 1000: 14, 15, 20: more work out the rotations again, fewer
// leave loads too few).
constexpr int kAppendGroups = 1024;

}  // namespace

void launch_paged_append(bool bf16, const AppendArgs& a, hipStream_t s) {
  // passes over heads go to further work-groups where the pages leave compute units idle
  const int pages = a.c.rows / 16 + 2 * a.c.n_seqs, per_pass = 128 / a.hd, heads = a.H + 2 * a.c.KVH;
  const dim3 grid(pages, std::min((heads + per_pass - 1) / per_pass, std::max(1, (kAppendGroups + pages / 2) / pages)));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
  const bool norm = a.q_gain || a.k_gain;
  auto by = [&](auto k128, auto n128, auto k64, auto n64) {
    a.hd == 128 ? (norm ? go(n128) : go(k128)) : (norm ? go(n64) : go(k64));
  };
  if (bf16)
    by(paged_append_kernel<uint16_t, 128, false>, paged_append_kernel<uint16_t, 128, true>,
       paged_append_kernel<uint16_t, 64, false>, paged_append_kernel<uint16_t, 64, true>);
  else
    by(paged_append_kernel<float, 128, false>, paged_append_kernel<float, 128, true>,
       paged_append_kernel<float, 64, false>, paged_append_kernel<float, 64, true>);
}

void launch_paged_means(bool bf16, const MeansArgs& a, hipStream_t s) {
  const dim3 grid(a.c.rows / a.block + a.c.n_seqs, a.c.KVH);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, a); };
  if (bf16)
    a.hd == 128 ? go(paged_means_kernel<uint16_t, 128>) : go(paged_means_kernel<uint16_t, 64>);
  else
    a.hd == 128 ? go(paged_means_kernel<float, 128>) : go(paged_means_kernel<float, 64>);
}

void launch_paged_select(bool bf16, const SelectArgs& a, hipStream_t s) {
  // blocks of a work-group: a multiple of the 64 that its waves score at a time
  const int tiles = (a.c.rows + 15) / 16 + a.c.n_seqs;
  const int parts = std::max(1, kScoreGroups / std::max(1, (int)std::min<long long>((long long)tiles * a.c.KVH, kScoreGroups)));
  const int per = ((a.nb + parts - 1) / parts + 63) / 64 * 64;
  const dim3 grid(tiles, a.c.KVH, per ? (a.nb + per - 1) / per : 1);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, per); };
  if (a.nb > 0) {
    if (bf16)
      a.hd == 128 ? go(paged_score_kernel<uint16_t, 128>) : go(paged_score_kernel<uint16_t, 64>);
    else
      a.hd == 128 ? go(paged_score_kernel<float, 128>) : go(paged_score_kernel<float, 64>);
  }
  const int items = a.c.rows * a.c.KVH;
  hipLaunchKernelGGL(paged_choose_kernel, dim3((items + 3) / 4), dim3(256), 0, s, a);
}

}  // namespace via
