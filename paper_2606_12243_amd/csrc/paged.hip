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
// A work-group takes 16 consecutive rows and some of one K/V head's share of
// them, its G query heads, its K and its V head.  Thread t holds 8 dims of row
// t / 16 (16 lanes a row: a head of 128, or two of 64), so a head's sum of
// squares and a dim's partner are lane exchanges, and q and k go out 16 bytes a
// thread or more.  V, transposed in its pages, goes through LDS: 16 lanes write
// 16 tokens of a dim next to each other.
//
// Angles are whole turns in fp64, pos * (theta^(-2i/hd) / 2 pi), of which only the
// fraction is kept: fp32 would lose it at far positions (2^-24 of 10^5 turns).
// Norms and rotations are fp32, rounded once where they are stored.
template <typename T, int HD, bool NORM>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int TPH = HD / 8, HPP = 16 / TPH, HALF = HD / 2;  // threads of a row per head; heads per pass
  const int lane = threadIdx.x & 63, r = threadIdx.x >> 4, l = threadIdx.x & 15, sub = l / TPH, d0 = (l % TPH) * 8;
  const int g = blockIdx.y, G = a.H / a.c.KVH;
  const int row0 = blockIdx.x * 16, row = row0 + r;
  __shared__ int s_seq[16], s_slot[16];
  // sequences of the 16 rows: wave w finds rows 4 w .. 4 w + 3
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int m = (threadIdx.x >> 6) * 4 + i, t = row0 + m;
    int seq = t < a.c.rows ? seq_of_row(a.c, t) : -1, slot = -1;
    if (seq >= 0) {
      int first, n;
      seq_rows(a.c, seq, first, n);
      slot = seq_len(a.c, seq) - n + (t - first);
    }
    if (lane == 0) {
      s_seq[m] = seq;
      s_slot[m] = slot;
    }
  }
  __syncthreads();
  const int seq = s_seq[r], slot = s_slot[r];
  const bool live = seq >= 0;
  const bool first = d0 < HALF;
  float cs[8], sn[8];
  {
    const double pos = live ? (double)(a.pos ? a.pos[row] : slot) : 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = pos * a.turn[d0 % HALF + e];
      const float f = (float)(turns - rint(turns));
      sincospif(2.f * f, &sn[e], &cs[e]);
    }
  }
  auto page_at = [&](int s, int p) { return s >= 0 && p >= 0 && p < a.c.cap ? page_of(a.c, s, p >> 4) : -1; };
  const int page = page_at(seq, slot);
  __shared__ float vt[HD][17];
  // heads of this work-group: 0 .. G - 1 its queries, G the K head, G + 1 the V head
  auto head = [&](int h) { return h < G ? g * G + h : h == G ? a.H + g : a.H + a.c.KVH + g; };
  for (int h0 = blockIdx.z * HPP; h0 < G + 2; h0 += gridDim.z * HPP) {
    const int h = h0 + sub;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live && h < G + 2) {
      const T* p = (const T*)a.qkv + (size_t)row * a.qkv_ld + (size_t)head(h) * HD + d0;
      if constexpr (sizeof(T) == 2) {
        const uint4 v = *(const uint4*)p;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = __uint_as_float(w[e] << 16);
          x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[e];
      }
    }
    float y[8];
    if (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int o = 1; o < TPH; o <<= 1) ss += __shfl_xor(ss, o, 64);
      const T* gain = (const T*)(h < G ? a.q_gain : h == G ? a.k_gain : nullptr);
      const float sc = 1.0f / sqrtf(ss / (float)HD + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = gain ? x[e] * sc * to_f<T>(gain[d0 + e]) : x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float o = __shfl_xor(y[e], TPH / 2, 64);  // the pair's other half
      const float t = first ? y[e] * cs[e] - o * sn[e] : y[e] * cs[e] + o * sn[e];
      y[e] = h <= G ? t : y[e];
    }
    T* dst = nullptr;
    if (live && h < G)
      dst = (T*)a.q_out + (size_t)row * a.q_ld + (size_t)head(h) * HD + d0;
    else if (h == G && page >= 0)
      dst = (T*)a.c.pool + k_off(0, page, a.c.n_blocks, a.c.KVH, HD, g, slot & 15, d0);
    if (dst) {
      if constexpr (sizeof(T) == 2) {
        *(uint4*)dst = make_uint4(pack_bf16x2(f2bf(y[0]), f2bf(y[1])), pack_bf16x2(f2bf(y[2]), f2bf(y[3])),
                                  pack_bf16x2(f2bf(y[4]), f2bf(y[5])), pack_bf16x2(f2bf(y[6]), f2bf(y[7])));
      } else {
        *(float4*)dst = make_float4(y[0], y[1], y[2], y[3]);
        *(float4*)(dst + 4) = make_float4(y[4], y[5], y[6], y[7]);
      }
    }
    if (h0 <= G + 1 && G + 1 < h0 + HPP) {  // uniform: this pass holds the V head
      if (h == G + 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) vt[d0 + e][r] = x[e];
      }
      __syncthreads();
      // lane -> token threadIdx.x % 16, dims threadIdx.x / 16, + 16, ...
      const int vr = threadIdx.x & 15, vslot = s_slot[vr], vpage = page_at(s_seq[vr], vslot);
      if (vpage >= 0) {
        T* vp = (T*)a.c.pool + v_off(0, vpage, a.c.n_blocks, a.c.KVH, HD, g, vslot & 15, 0);
        for (int d = threadIdx.x >> 4; d < HD; d += 16) vp[(size_t)d * kBlock] = from_f<T>(vt[d][vr]);
      }
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
  const int g = blockIdx.y, seq = blockIdx.z, lane = threadIdx.x;
  int first, n, all;
  seq_of_wave(a.c, seq, first, n, all);
  const int len = min(all, a.c.cap), old = max(all - n, 0);
  const int b = old / a.block + blockIdx.x;
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
// A work-group takes 16 rows of a sequence and one K/V head: its eight waves score
// 16 blocks at a time with v_mfma_f64_16x16x4_f64, the next 16 blocks' means in
// flight, and then choose for one row after another.  A score is kept as 64 bits
// that order like it; a wave holds the upper halves of a row's scores in
// registers and finds the n_sel-th largest bit by bit, which ends as soon as
// n_sel of them are as large; lower halves are read only where upper ones tie.
constexpr int kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;
constexpr int kSelectHeld = 32;  // scores a lane holds: rows of up to 64 * kSelectHeld blocks
typedef double f64x4 __attribute__((ext_vector_type(4)));

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
__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(SelectArgs a) {
  constexpr int KS = HD / 4;  // k steps; lane l holds dims (l/16) * KS .. + KS - 1 of row or block l % 16
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = blockIdx.y, m = lane & 15, kq = lane >> 4;
  const int G = a.H / a.c.KVH;
  int seq, tile, first, n, len;
  if (!tile_of_item(a.c, blockIdx.x, 1, 16, seq, tile)) return;
  seq_of_wave(a.c, seq, first, n, len);
  const int r0 = tile * 16;
  if (tile < 0 || r0 >= n) return;
  const int pos0 = len - n + r0;  // position of the tile's first row
  const int rows = min(16, n - r0);
  // blocks the tile's last row sees (positions past the cap see what the last one does)
  const int seen = min(min(max(pos0 + rows - 1, -1), a.c.cap - 1) / a.block + 1, a.nb);
  if (wave * 16 < seen) {
    const float* means = a.means + ((size_t)seq * a.c.KVH + g) * (size_t)a.max_blocks * HD + kq * KS;
    float4 v[KS / 4], u[KS / 4];
    auto load = [&](float4 (&d)[KS / 4], int b0) {
      const float* p = means + (size_t)min(b0 + m, seen - 1) * HD;
#pragma unroll
      for (int i = 0; i < KS / 4; ++i) d[i] = *(const float4*)(p + i * 4);
    };
    load(v, wave * 16);
    double q[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) q[i] = 0.0;
    if (m < rows) {
      const T* p = (const T*)a.q + (size_t)(first + r0 + m) * a.q_ld + (size_t)g * G * HD + kq * KS;
      int h = 0;
      for (; h + 4 <= G; h += 4) {  // (four heads' loads together)
#pragma unroll
        for (int i = 0; i < 4; ++i) add_to<T, KS>(q, p + (size_t)(h + i) * HD);
      }
      for (; h < G; ++h) add_to<T, KS>(q, p + (size_t)h * HD);
    }
    auto score = [&](const float4 (&d)[KS / 4], int b0) {
      f64x4 s = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int i = 0; i < KS / 4; ++i) {
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i], (double)d[i].x, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 1], (double)d[i].y, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 2], (double)d[i].z, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * i + 3], (double)d[i].w, s, 0, 0, 0);
      }
      // register i of lane l: row 4 i + l / 16, block l % 16
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 4 * i + kq;
        if (row < rows && b0 + m < seen)
          a.scores[((size_t)(first + r0 + row) * a.c.KVH + g) * a.nb + b0 + m] = sortable(s[i]);
      }
    };
    constexpr int kStep = kSelectWaves * 16;
    for (int b0 = wave * 16; b0 < seen; b0 += 2 * kStep) {
      load(u, b0 + kStep);
      score(v, b0);
      if (b0 + kStep >= seen) break;
      load(v, b0 + 2 * kStep);
      score(u, b0 + kStep);
    }
  }
  __syncthreads();
  for (int r = wave; r < rows; r += kSelectWaves) {
    const int row = first + r0 + r, pos = min(pos0 + r, a.c.cap - 1);
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
}

}  // namespace

void launch_paged_append(bool bf16, const AppendArgs& a, hipStream_t s) {
  // passes over heads go to further work-groups where the rows leave compute units idle
  const int tiles = (a.c.rows + 15) / 16, heads = a.H / a.c.KVH + 2, passes = a.hd == 128 ? heads : (heads + 1) / 2;
  const dim3 grid(tiles, a.c.KVH, std::min(passes, (512 + tiles * a.c.KVH - 1) / (tiles * a.c.KVH)));
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
  const dim3 grid(a.per_seq, a.c.KVH, a.c.n_seqs);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, a); };
  if (bf16)
    a.hd == 128 ? go(paged_means_kernel<uint16_t, 128>) : go(paged_means_kernel<uint16_t, 64>);
  else
    a.hd == 128 ? go(paged_means_kernel<float, 128>) : go(paged_means_kernel<float, 64>);
}

void launch_paged_select(bool bf16, const SelectArgs& a, hipStream_t s) {
  const dim3 grid((a.c.rows + 15) / 16 + a.c.n_seqs, a.c.KVH);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelectThreads), 0, s, a); };
  if (bf16)
    a.hd == 128 ? go(paged_select_kernel<uint16_t, 128>) : go(paged_select_kernel<uint16_t, 64>);
  else
    a.hd == 128 ? go(paged_select_kernel<float, 128>) : go(paged_select_kernel<float, 64>);
}

}  // namespace via
