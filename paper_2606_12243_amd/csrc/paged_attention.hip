// Attention of a batch's rows over the paged cache (via_paged_attend,
// via_paged_attend_blocks): out = softmax(scale q K^T) V over the keys a row
// sees, every key of its sequence up to its own (causal, optionally the last
// `window` of them, or a tree mask over the batch's own keys) or those of the
// blocks listed for it.
//
// Few rows: the cached keys and values are read once at the rate of a large
// copy (that bounds it), so a work-group streams a span of keys straight into
// matrix-instruction operands.  Its 32 queries are (row, head) pairs of one K/V
// head, which share every byte read.  The keys of a tile are cut into n_splits
// spans where there are too few tiles to fill the card, and a second kernel
// joins the partial results in span order.
//
// Four waves a work-group; wave w takes the 32-key blocks w, w + 4, ... (bf16:
// with the next block's loads in flight).  S^T = K Q^T keeps one query a lane (two
// lanes a query, 16 keys each), so a running maximum and sum needs one lane
// exchange, and its registers are the P^T operand of O^T += V^T P^T as they are:
//   bf16, v_mfma_f32_32x32x16_bf16: A-row m of the K tile holds key
//     (m/16)*16 + ((m/4)%2)*8 + ((m/8)%2)*4 + m%4, so register i of lane l holds
//     key (i/8)*16 + (l/32)*8 + i%8: eight consecutive keys, a V page's 16 bytes.
//     P is split in two bf16 terms (16 bits): the loop waits for memory, and one
//     term would add about as much error again as the output's rounding has.
//   fp32, v_mfma_f32_32x32x2_f32: register i holds key (i/4)*8 + (l/32)*4 + i%4,
//     four consecutive tokens of a V page a lane.  The contraction over the head
//     dimension takes dims j and j + 4 of a group of eight in one instruction.
// Scores, maxima (log2 units), sums and outputs are fp32.
//
// A key that some of the queries do not see must not reach them even as 0 times
// an infinity or NaN.  In blocks that not all queries see whole, such values are
// taken out of V and added, to the queries that see them, by counting them.
#include <algorithm>

#include "paged.h"

namespace via {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mma_bf16(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma_f32(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint4 load_stream(const void* p) {  // read once: past the caches
  const u32x4 v = __builtin_nontemporal_load((const u32x4*)p);
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ float lane_f(const uint4& v, int e) {
  return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
}

// Operand pieces of a 32-key block, 16 bytes a lane each.
template <typename T, int HD>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int NQ = kBf16 ? HD / 16 : HD / 8;  // K (and Q) pieces: the lane's share of a key's dims
  static constexpr int NV = kBf16 ? 2 : 4;             // V pieces per 32 dims: the lane's share of the keys
  static constexpr int DT = HD / 32;
};
// dims a lane holds of piece j: the first one
template <typename T>
__device__ __forceinline__ int piece_dim(int j, int half) {
  return sizeof(T) == 2 ? j * 16 + half * 8 : j * 8 + half * 4;
}
// key (within the 32) of score register i
template <typename T>
__device__ __forceinline__ int reg_key(int i, int half) {
  return sizeof(T) == 2 ? (i >> 3) * 16 + half * 8 + (i & 7) : (i >> 2) * 8 + half * 4 + (i & 3);
}

template <typename T, int HD>
struct Block {
  uint4 k[Shape<T, HD>::NQ];
  uint4 v[Shape<T, HD>::DT][Shape<T, HD>::NV];
};

// V piece n of the lane for the first 32 dims
template <typename T, int HD>
__device__ __forceinline__ const T* v_piece(const PagedRef& c, int g, int page0, int page1, int n, int ql, int half) {
  using S = Shape<T, HD>;
  const int tok = S::kBf16 ? half * 8 : (n & 1) * 8 + half * 4;
  return (const T*)c.pool + v_off(0, max(n >= S::NV / 2 ? page1 : page0, 0), c.n_blocks, c.KVH, HD, g, tok, ql);
}

// pages: the two pages of the block, -1 (absent) read as page 0 and masked by the caller
template <typename T, int HD>
__device__ __forceinline__ void load_block(Block<T, HD>& b, const PagedRef& c, int g, int page0, int page1, int ql,
                                           int half) {
  using S = Shape<T, HD>;
  const T* pool = (const T*)c.pool;
  const int key = S::kBf16 ? ((ql >> 4) << 4) + (((ql >> 2) & 1) << 3) + (((ql >> 3) & 1) << 2) + (ql & 3) : ql;
  const T* kp = pool + k_off(0, max(key >= 16 ? page1 : page0, 0), c.n_blocks, c.KVH, HD, g, key & 15, 0);
#pragma unroll
  for (int j = 0; j < S::NQ; ++j) {
    const int d = piece_dim<T>(j, half);
    b.k[j] = load_stream(kp + (d >> 3) * kBlock * 8 + (d & 7));
  }
#pragma unroll
  for (int n = 0; n < S::NV; ++n) {
    const T* vp = v_piece<T, HD>(c, g, page0, page1, n, ql, half);
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) b.v[dt][n] = load_stream(vp + dt * 32 * kBlock);
  }
}

// Two register sets for a wave's blocks, or one and other waves to run meanwhile: an
// fp32 block is twice as large, and two of them are spilled at a head of 128 (16 x
// 4096 keys of 8 heads: 291 us against 122) and leave one work-group a compute unit at 64
// (64 us against 59).
template <typename T>
constexpr bool kTwoSets = sizeof(T) == 2;

// What the lane's query sees: keys [lo, vis), and key base + o where bit o of mask is set.
struct Query {
  bool valid;
  int row, head;  // row of the batch, query head
  int lo, vis, base;
  uint64_t mask;
};
__device__ __forceinline__ bool sees(const Query& q, int key) {
  const int o = key - q.base;
  return (key >= q.lo && key < q.vis) || (o >= 0 && o < 64 && ((q.mask >> o) & 1));
}

template <typename T, int HD>
struct Acc {
  f32x16 o[HD / 32];
  float m, l;  // running maximum (log2 units) and sum
};

// Two weights as bf16: rounded to nearest, or (hi, lo) truncated and the rest rounded.
__device__ __forceinline__ uint32_t round_pair(float p0, float p1) {
  const bf16x2 r = {(__bf16)p0, (__bf16)p1};
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t split_pair(float p0, float p1, uint32_t& lo) {
  lo = round_pair(p0 - __uint_as_float(__float_as_uint(p0) & 0xFFFF0000u), p1 - __uint_as_float(__float_as_uint(p1) & 0xFFFF0000u));
  return __builtin_amdgcn_perm(__float_as_uint(p1), __float_as_uint(p0), 0x07060302u);
}

// O^T += V^T P^T for weights given as a function of the score register
template <typename T, int HD, typename P>
__device__ __forceinline__ f32x16 add_pv(const uint4 (&v)[Shape<T, HD>::NV], P p, f32x16 o) {
  using S = Shape<T, HD>;
#pragma unroll
  for (int n = 0; n < S::NV; ++n) {
    if constexpr (S::kBf16) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(p(n * 8 + 2 * e), p(n * 8 + 2 * e + 1));
      o = mma_bf16(v[n], make_uint4(w[0], w[1], w[2], w[3]), o);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o = mma_f32(lane_f(v[n], e), __uint_as_float(p(n * 4 + e)), o);
    }
  }
  return o;
}

// One bit per value of a 32-bit word (two bf16, or one float): infinite or NaN.
// All ones in the exponent carry into the sign's place.
template <typename T>
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
  return sizeof(T) == 2 ? ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u : ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u;
}
template <typename T, int HD>
__device__ __forceinline__ bool has_odd_values(const Block<T, HD>& b) {
  using S = Shape<T, HD>;
  uint32_t m = 0;
#pragma unroll
  for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
    for (int n = 0; n < S::NV; ++n)
      m |= odd_bits<T>(b.v[dt][n].x) | odd_bits<T>(b.v[dt][n].y) | odd_bits<T>(b.v[dt][n].z) | odd_bits<T>(b.v[dt][n].w);
  return m != 0;
}
// Takes them out of V.
template <typename T>
__device__ __forceinline__ uint32_t drop_odd(uint32_t w) {
  const uint32_t m = odd_bits<T>(w);
  return w & ~(sizeof(T) == 2 ? (m >> 15) * 0xFFFFu : (uint32_t)((int32_t)m >> 31));
}
template <typename T, int HD>
__device__ __forceinline__ void drop_odd_values(Block<T, HD>& b) {
  using S = Shape<T, HD>;
#pragma unroll
  for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
    for (int n = 0; n < S::NV; ++n) {
      uint4& v = b.v[dt][n];
      v = make_uint4(drop_odd<T>(v.x), drop_odd<T>(v.y), drop_odd<T>(v.z), drop_odd<T>(v.w));
    }
}
// Bit i: the lane's query sees the key of score register i.
template <typename T>
__device__ __forceinline__ uint32_t seen_keys(const Query& q, int kb, bool page0, bool page1, int half) {
  uint32_t seen = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int o = reg_key<T>(i, half);
    seen |= q.valid && (o < 16 ? page0 : page1) && sees(q, kb + o) ? 1u << i : 0u;
  }
  return seen;
}
__device__ __forceinline__ bool sees_whole(const Query& q, int kb, bool page0, bool page1) {
  return page0 && page1 && __all(!q.valid || (kb >= q.lo && kb + 32 <= q.vis));
}

// Infinities and NaN of V in a block that not every query sees whole: counted
// for every query that sees them, and added to its outputs.
template <typename T, int HD>
__device__ __forceinline__ void add_odd_values(const PagedRef& c, int g, int page0, int page1, int ql, int half,
                                               uint32_t seen, Acc<T, HD>& a) {
  using S = Shape<T, HD>;
  constexpr uint32_t kOne = S::kBf16 ? 0x3F80u : 0x3F800000u;
  // one of them a time, as ones: kind 0 NaN, 1 +infinity, 2 -infinity
  auto pick = [](uint32_t bits, int kind) -> uint32_t {  // bits of a float
    const bool nan = (bits & 0x7FFFFFFFu) > 0x7F800000u;
    return (kind == 0 ? nan : bits == (kind == 1 ? 0x7F800000u : 0xFF800000u)) ? kOne : 0u;
  };
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {
    const float add = __uint_as_float(kind == 0 ? 0x7FC00000u : kind == 1 ? 0x7F800000u : 0xFF800000u);
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) {
      uint4 f[S::NV];
#pragma unroll
      for (int n = 0; n < S::NV; ++n) {
        auto word = [&](uint32_t w) {
          return S::kBf16 ? pick(w << 16, kind) | (pick(w & 0xFFFF0000u, kind) << 16) : pick(w, kind);
        };
        const uint4 v = *(const uint4*)(v_piece<T, HD>(c, g, page0, page1, n, ql, half) + dt * 32 * kBlock);
        f[n] = make_uint4(word(v.x), word(v.y), word(v.z), word(v.w));
        __builtin_amdgcn_sched_barrier(0);  // (keeps the comparisons' masks few)
      }
      f32x16 count;
#pragma unroll
      for (int i = 0; i < 16; ++i) count[i] = 0.f;
      count = add_pv<T, HD>(f, [&](int i) { return (0u - ((seen >> i) & 1)) & kOne; }, count);
      settle();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        a.o[dt][i] += count[i] > 0.f ? add : 0.f;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}

// One 32-key block (keys kb .. kb + 31, its pages present or not) for the wave's 32 queries.
template <typename T, int HD>
__device__ __forceinline__ void compute_block(Block<T, HD>& b, int kb, bool page0, bool page1, const Query& q,
                                              const uint4 (*sq)[64], int lane, float sl2, Acc<T, HD>& a, bool& odd) {
  using S = Shape<T, HD>;
  const int half = lane >> 5;
  // Q is read from LDS for every block (the registers of two work-groups per
  // compute unit do not hold it): an opaque zero keeps the reads in the loop
  int zero;
  asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int j = 0; j < S::NQ; ++j) {
    const uint4 qj = sq[j][lane + zero];
    if constexpr (S::kBf16) {
      s = mma_bf16(b.k[j], qj, s);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) s = mma_f32(lane_f(b.k[j], e), lane_f(qj, e), s);
    }
  }
  settle();
  if (!sees_whole(q, kb, page0, page1)) {
    const uint32_t seen = seen_keys<T>(q, kb, page0, page1, half);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = (seen >> i) & 1 ? s[i] : -INFINITY;
    if (__any(has_odd_values<T, HD>(b))) {
      drop_odd_values<T, HD>(b);
      odd = true;
    }
  }
  // the maximum is taken on unscaled scores (scale > 0)
  float bm = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) bm = fmaxf(bm, s[i]);
  bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
  const float mn = fmaxf(a.m, bm * sl2);
  if (__any(mn > a.m)) {
    const float alpha = mn == a.m ? 1.f : __builtin_amdgcn_exp2f(a.m - mn);
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) a.o[dt] *= alpha;
    a.l *= alpha;
    a.m = mn;
  }
  const float neg_m = a.m == -INFINITY ? 0.f : -a.m;  // nothing seen yet: every weight is 0
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, neg_m));
    a.l += p[i];
  }
  if constexpr (S::kBf16) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      uint32_t hw[4], lw[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) hw[e] = split_pair(p[n * 8 + 2 * e], p[n * 8 + 2 * e + 1], lw[e]);
      const uint4 hi = make_uint4(hw[0], hw[1], hw[2], hw[3]), lo = make_uint4(lw[0], lw[1], lw[2], lw[3]);
#pragma unroll
      for (int dt = 0; dt < S::DT; ++dt) {
        a.o[dt] = mma_bf16(b.v[dt][n], hi, a.o[dt]);
        a.o[dt] = mma_bf16(b.v[dt][n], lo, a.o[dt]);
      }
    }
  } else {
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt)
      a.o[dt] = add_pv<T, HD>(b.v[dt], [&](int i) { return __float_as_uint(p[i]); }, a.o[dt]);
  }
}

// First position of the window at `pos` (no difference that a window of all positions overflows).
__device__ __forceinline__ int window_from(const PagedAttnArgs& a, int pos) {
  return a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
}

// Queries q0 .. q0 + tile_q - 1 of a sequence: the keys [lo, end) that their rows
// see, lo on a page-pair border.
__device__ __forceinline__ void tile_keys(const PagedAttnArgs& a, int len, int n, int q0, int& lo, int& end) {
  const int G = a.H / a.c.KVH, pos0 = len - n;
  const int r0 = q0 / G, r1 = min(n - 1, (q0 + a.tile_q - 1) / G);
  end = min(a.row_mask ? len : pos0 + r1 + 1, a.c.cap);
  lo = min(window_from(a, pos0 + r0), max(end, 0)) & ~31;
}

// Query qi = row * G + head of a sequence's queries under K/V head g.
__device__ __forceinline__ Query query_of(const PagedAttnArgs& a, int g, int qi, int first, int n, int len) {
  const int G = a.H / a.c.KVH, r = qi / G, pos = len - n + r;
  Query q;
  q.valid = r < n;
  q.row = first + min(r, n - 1);
  q.head = g * G + qi % G;
  q.lo = window_from(a, pos);
  q.vis = a.row_mask ? min(len - n, a.c.cap) : min(pos, a.c.cap - 1) + 1;
  q.base = len - n;
  q.mask = 0;
  if (a.row_mask) {
    // bits past the batch's own rows, or past the last key that a call looks at, are no keys
    const int own = min(min(n, 64), max(a.c.cap - q.base, 0));
    q.mask = (q.valid ? a.row_mask[q.row] : 0) & (own >= 64 ? ~0ull : (1ull << own) - 1);
  }
  return q;
}

template <typename T, int HD, bool LISTED>
__global__ __launch_bounds__(256, (sizeof(T) * HD <= 256 ? 2 : 1)) void paged_stream_kernel(PagedAttnArgs a) {
  using S = Shape<T, HD>;
  constexpr int DT = S::DT;
  const int G = a.H / a.c.KVH;
  // blocks of a launch: split fastest, K/V head, tile slowest
  const int split = blockIdx.x % a.n_splits, gi = blockIdx.x / a.n_splits, g = gi % a.c.KVH, item = gi / a.c.KVH;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, ql = lane & 31,
            half = lane >> 5;
  int seq, tile = 0, first, n, len;
  if constexpr (LISTED) {
    const int tiles = (G + kPagedQueries - 1) / kPagedQueries;  // tiles of a row's group
    seq = seq_of_row(a.c, item / tiles);
    if (seq < 0) return;
  } else {
    if (!item_of(a.c, item, G, kPagedQueries, 1, seq, tile)) return;
  }
  seq_of_wave(a.c, seq, first, n, len);
  if ((long long)tile * kPagedQueries >= (long long)n * G) return;
  Query q;
  int k0, k1;  // the work-group's keys: positions, or places in the row's list
  const int32_t* list = nullptr;
  if constexpr (LISTED) {
    const int tiles = (G + kPagedQueries - 1) / kPagedQueries;
    const int row = item / tiles, hg = (item % tiles) * kPagedQueries + ql;
    const int pos = len - n + (row - first);
    q.valid = hg < G;
    q.row = row;
    q.head = g * G + min(hg, G - 1);
    q.lo = 0;
    q.vis = min(pos, a.c.cap - 1) + 1;
    q.base = 0;
    q.mask = 0;
    list = a.sel + ((size_t)row * a.c.KVH + g) * a.n_sel;
    k0 = split * a.span;
    k1 = min(a.n_sel * a.block, k0 + a.span);
  } else {
    int lo, end;
    tile_keys(a, len, n, tile * kPagedQueries, lo, end);
    q = query_of(a, g, tile * kPagedQueries + ql, first, n, len);
    k0 = lo + split * a.span;
    k1 = min(end, k0 + a.span);
    if (a.n_splits > 1 && k0 >= end) return;  // the joining kernel does not read it
  }

  __shared__ int spage[kPagedChunk / kBlock];
  __shared__ int sbase[LISTED ? kPagedChunk / 32 : 1];
  __shared__ float mo[2][DT * 16][64];  // wave merge: unscaled outputs, maxima, sums
  __shared__ float mm[2][64], ml[2][64];
  __shared__ uint4 sq[S::NQ][64];  // Q as the matrix instructions take it

  {
    const T* src = (const T*)a.q + (size_t)q.row * a.q_ld + (size_t)q.head * HD;
#pragma unroll
    for (int i = 0; i < S::NQ / 4; ++i) {
      const int j = i * 4 + wave;
      const uint4 v = *(const uint4*)(src + piece_dim<T>(j, half));
      sq[j][lane] = q.valid ? v : make_uint4(0, 0, 0, 0);
    }
  }
  const float sl2 = a.scale * 1.4426950408889634f;
  Acc<T, HD> acc;
  acc.m = -INFINITY;
  acc.l = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc.o[dt][i] = 0.f;

  for (int c0 = k0; c0 < k1; c0 += kPagedChunk) {
    const int nblk = (min(k1 - c0, kPagedChunk) + 31) >> 5;
    if (c0 > k0) __syncthreads();  // the last chunk's pages are no longer read
    for (int t = threadIdx.x; t < 2 * nblk; t += 256) {
      if constexpr (LISTED) {
        const int at = c0 + t * kBlock, b = list[at / a.block];
        // block b is real where its first key is one the row can see
        const bool ok = b >= 0 && b <= (q.vis - 1) / a.block && q.vis > 0;
        const int key = ok ? b * a.block + at % a.block : 0x40000000;
        spage[t] = ok ? page_of(a.c, seq, key >> 4) : -1;
        if (!(t & 1)) sbase[t >> 1] = key;
      } else {
        spage[t] = page_of(a.c, seq, (c0 >> 4) + t);
      }
    }
    __syncthreads();
    const int cnt = nblk > wave ? (nblk - wave + 3) >> 2 : 0;
    if (cnt > 0) {
      auto blk = [&](int i) { return wave + 4 * min(i, cnt - 1); };
      auto load = [&](Block<T, HD>& b, int i) {
        load_block<T, HD>(b, a.c, g, spage[2 * blk(i)], spage[2 * blk(i) + 1], ql, half);
      };
      bool odd = false;
      auto compute = [&](Block<T, HD>& b, int i) {
        const int kb = LISTED ? sbase[blk(i)] : c0 + blk(i) * 32;
        compute_block<T, HD>(b, kb, spage[2 * blk(i)] >= 0, spage[2 * blk(i) + 1] >= 0, q, sq, lane, sl2, acc, odd);
      };
      if constexpr (kTwoSets<T>) {
        // the next block's loads are in flight while one is multiplied; past the
        // wave's last block it reads that one again, so that every load is unconditional
        Block<T, HD> b0, b1;
        load(b0, 0);
        for (int i = 0; i < cnt; i += 2) {
          load(b1, i + 1);
          compute(b0, i);
          if (i + 1 >= cnt) break;
          load(b0, i + 2);
          compute(b1, i + 1);
        }
      } else {
        Block<T, HD> b;
        for (int i = 0; i < cnt; ++i) {
          load(b, i);
          compute(b, i);
        }
      }
      if (odd) {  // (the same in all lanes)
#pragma unroll 1
        for (int i = 0; i < cnt; ++i) {
          const int kb = LISTED ? sbase[blk(i)] : c0 + blk(i) * 32;
          const int page0 = spage[2 * blk(i)], page1 = spage[2 * blk(i) + 1];
          if (sees_whole(q, kb, page0 >= 0, page1 >= 0)) continue;
          add_odd_values<T, HD>(a.c, g, page0, page1, ql, half, seen_keys<T>(q, kb, page0 >= 0, page1 >= 0, half), acc);
        }
      }
    }
  }

  settle();
  // merge the four waves in a fixed order: (w0 + w2) + (w1 + w3)
  float lt = acc.l + __shfl_xor(acc.l, 32, 64);
  float mx = acc.m;
  auto store_to = [&](int buf) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mo[buf][dt * 16 + i][lane] = acc.o[dt][i];
    mm[buf][lane] = mx;
    ml[buf][lane] = lt;
  };
  auto weight = [](float m, float M) { return M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M); };
  if (wave >= 2) store_to(wave - 2);
  __syncthreads();
  if (wave < 2) {
    const float mb = mm[wave][lane], M = fmaxf(mx, mb);
    const float ca = weight(mx, M), cb = weight(mb, M);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc.o[dt][i] = acc.o[dt][i] * ca + mo[wave][dt * 16 + i][lane] * cb;
    lt = lt * ca + ml[wave][lane] * cb;
    mx = M;
  }
  __syncthreads();
  if (wave < 2) store_to(wave);
  __syncthreads();
  // the last merge and the output: a quarter of the dims a wave
  const float m0 = mm[0][lane], m1 = mm[1][lane], M = fmaxf(m0, m1);
  const float ca = weight(m0, M), cb = weight(m1, M);
  const float l = ml[0][lane] * ca + ml[1][lane] * cb;
  if (!q.valid) return;
  const bool direct = a.n_splits == 1;
  const float inv = direct ? (l == 0.f ? 0.f : 1.f / l) : 1.f;  // a row that sees nothing: zeros
  const size_t at = ((size_t)split * a.c.rows + q.row) * a.H + q.head;
  // O^T lane l, register i of d tile dt -> dim dt*32 + (i/4)*8 + (l/32)*4 + i%4
#pragma unroll
  for (int j = 0; j < DT; ++j) {
    const int u = wave * DT + j, dt = u >> 2, i4 = u & 3;  // registers 4 i4 .. 4 i4 + 3 of d tile dt
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (mo[0][u * 4 + i][lane] * ca + mo[1][u * 4 + i][lane] * cb) * inv;
    const int d = dt * 32 + i4 * 8 + half * 4;
    if (!direct) {
      *(float4*)(a.part_o + at * HD + d) = make_float4(x[0], x[1], x[2], x[3]);
    } else if constexpr (S::kBf16) {
      *(uint2*)((T*)a.out + (size_t)q.row * a.out_ld + (size_t)q.head * HD + d) =
          make_uint2(pack_bf16x2(f2bf(x[0]), f2bf(x[1])), pack_bf16x2(f2bf(x[2]), f2bf(x[3])));
    } else {
      *(float4*)((T*)a.out + (size_t)q.row * a.out_ld + (size_t)q.head * HD + d) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
  if (wave == 0 && half == 0) {
    if (!direct) {
      a.part_ml[at * 2] = M;
      a.part_ml[at * 2 + 1] = l;
    } else if (a.lse) {
      a.lse[(size_t)q.row * a.H + q.head] = (M + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
  }
}

// ---------------------------------------------------------------------------
// More than 32 queries, bf16: with many rows the matrix instructions bound it.  A work-group takes 128
// queries of one K/V head, a wave 32 of them; 64 keys at a time are copied into LDS
// (asynchronously, the next 64 in flight) and read by all four waves as matrix
// operands.  Pages are copied as they are, but that the two 16-byte halves of a V
// row go apart, so that every operand read is 256 consecutive bytes per 16 lanes.
// Two work-groups share a compute unit: one's softmax runs beside the other's
// products.  The weights are one bf16 value each (TERMS = 1, to nearest: 2^-8 of
// a weight at most, about what the output's own rounding costs, where two would be
// half again the products), or two where few rows leave the loop waiting for
// memory.  The running maximum is raised only when it grows by more than 2^8,
// which spares most rescalings of O; weights up to 2^8 lose nothing.
constexpr int kTileQueries = kPagedTileQueries, kTileKeys = 64;

// 16 bytes a lane from base + voff to LDS at lds + 16 * lane (base, lds wave-uniform).  A copy into
// LDS needs a wait state after the write of its m0, which the compiler does not put into inline assembly.
__device__ __forceinline__ void lds_copy16(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds) : "memory", "m0");
}

// maximum over the lane and its partner, lane ^ 32
__device__ __forceinline__ float other_half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int HD, int TERMS>
__global__ __launch_bounds__(256, 2) void paged_tile_kernel(PagedAttnArgs a) {
  using S = Shape<uint16_t, HD>;
  constexpr int DT = S::DT, NQ = S::NQ, kPage = kBlock * HD * 2;  // bytes of a K or V page
  constexpr int kPieces = kPage / 1024;
  __shared__ __align__(1024) unsigned char smem[2][2][4][kPage];  // [buffer][K, V][page]
  const int G = a.H / a.c.KVH;
  // blocks of a launch: K/V head fastest (with 8 of them an XCD keeps one head's pages in its L2), split, tile slowest
  const int g = blockIdx.x % a.c.KVH, rest = blockIdx.x / a.c.KVH, split = rest % a.n_splits, item = rest / a.n_splits;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, ql = lane & 31, half = lane >> 5;
  int seq, tile, first, n, len;
  if (!item_of(a.c, item, G, kTileQueries, 1, seq, tile)) return;
  seq_of_wave(a.c, seq, first, n, len);
  if ((long long)tile * kTileQueries >= (long long)n * G) return;
  // the last rows, which see most keys, go first
  tile = (int)(((long long)n * G + kTileQueries - 1) / kTileQueries) - 1 - tile;
  int lo, end;
  tile_keys(a, len, n, tile * kTileQueries, lo, end);
  const Query q = query_of(a, g, tile * kTileQueries + wave * 32 + ql, first, n, len);
  const int k0 = lo + split * a.span, k1 = min(end, k0 + a.span);
  if (a.n_splits > 1 && k0 >= end) return;  // the joining kernel does not read it
  // no query of the wave sees a key before `from` or from `top` on
  int from = q.valid ? q.lo : 0x7FFFFFFF, top = !q.valid ? 0 : a.row_mask ? min(len, a.c.cap) : q.vis;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    from = min(from, __shfl_xor(from, o, 64));
    top = max(top, __shfl_xor(top, o, 64));
  }
  from = __builtin_amdgcn_readfirstlane(from);
  top = __builtin_amdgcn_readfirstlane(top);
  auto whole = [&](int kb) { return __all(!q.valid || (kb >= q.lo && kb + kTileKeys <= q.vis)); };

  uint4 qf[NQ];
  {
    const uint16_t* src = (const uint16_t*)a.q + (size_t)q.row * a.q_ld + (size_t)q.head * HD + half * 8;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const uint4 v = *(const uint4*)(src + j * 16);
      qf[j] = q.valid ? v : make_uint4(0, 0, 0, 0);
    }
  }
  const float sl2 = a.scale * 1.4426950408889634f;
  Acc<uint16_t, HD> acc;
  acc.m = -INFINITY;
  acc.l = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc.o[dt][i] = 0.f;

  const int tiles = k1 > k0 ? (k1 - k0 + kTileKeys - 1) / kTileKeys : 0;
  const uint32_t lds = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)&smem[0][0][0][0];
  const uint32_t lds_w = __builtin_amdgcn_readfirstlane(lds + wave * kPage);
  const uint32_t voff_k = lane * 16, voff_v = ((lane & 31) * 2 + half) * 16;
  // lane i % 4 holds the page of tile t's keys 16 i .. 16 i + 15; wave w copies page w
  auto pages_of = [&](int t) { return page_of(a.c, seq, (k0 >> 4) + t * 4 + (lane & 3)); };
  auto copy = [&](int t, int pages) {
    const int page = max(__builtin_amdgcn_readlane(pages, wave), 0);
    const char* src = (const char*)a.c.pool + ((size_t)g * a.c.n_blocks + page) * 2 * kPage;
    const uint32_t dst = lds_w + (t & 1) * 8 * kPage;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      lds_copy16(src + i * 1024, voff_k, dst + i * 1024);
      lds_copy16(src + kPage + i * 1024, voff_v, dst + 4 * kPage + i * 1024);
    }
  };
  const int key = ((ql >> 4) << 4) + (((ql >> 2) & 1) << 3) + (((ql >> 3) & 1) << 2) + (ql & 3);
  const int k_at = (key >> 4) * kPage + half * 256 + (key & 15) * 16;

  bool any_odd = false;
  int pages = pages_of(0), pages1 = pages_of(1);
  if (tiles > 0) copy(0, pages);
  for (int t = 0; t < tiles; ++t) {
    __builtin_amdgcn_s_waitcnt(0);  // the wave's copies have landed ...
    __builtin_amdgcn_s_barrier();   // ... and all waves', and nobody reads the other buffer any more
    const int pages2 = pages_of(t + 2);
    if (t + 1 < tiles) copy(t + 1, pages1);
    const int kb = k0 + t * kTileKeys;
    const unsigned char* sk = &smem[t & 1][0][0][0] + k_at;
    const unsigned char* sv = &smem[t & 1][1][0][0] + lane * 16;
    if (kb < top && kb + kTileKeys > from) {
      const uint32_t absent = (uint32_t)__ballot(pages < 0) & 15;
      const bool all = !absent && whole(kb);
      f32x16 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
        for (int j = 0; j < NQ; ++j) s[b] = mma_bf16(*(const uint4*)(sk + b * 2 * kPage + j * 512), qf[j], s[b]);
      }
      // four operand reads ahead of the products
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < 2 * NQ - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
      settle();
      if (!all) {
        if (absent || a.row_mask) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint32_t seen =
                seen_keys<uint16_t>(q, kb + b * 32, !((absent >> (2 * b)) & 1), !((absent >> (2 * b + 1)) & 1), half);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = (seen >> i) & 1 ? s[b][i] : -INFINITY;
          }
        } else {  // keys lo .. vis - 1: a comparison a score
          const int lo = q.lo - kb - half * 8;
          const uint32_t n_seen = q.valid ? max(q.vis - q.lo, 0) : 0;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              s[b][i] = (uint32_t)(b * 32 + (i >> 3) * 16 + (i & 7) - lo) < n_seen ? s[b][i] : -INFINITY;
        }
      }
      // (maximum, not fmaxf: one instruction for two values, NaN kept)
      float bm = s[0][0], bm1 = s[1][0];
#pragma unroll
      for (int i = 1; i < 15; i += 2) {
        bm = __builtin_elementwise_maximum(__builtin_elementwise_maximum(bm, s[0][i]), s[0][i + 1]);
        bm1 = __builtin_elementwise_maximum(__builtin_elementwise_maximum(bm1, s[1][i]), s[1][i + 1]);
      }
      bm = __builtin_elementwise_maximum(__builtin_elementwise_maximum(bm, s[0][15]), bm1);
      bm = other_half_max(__builtin_elementwise_maximum(bm, s[1][15]));
      const float mn = __builtin_elementwise_maximum(acc.m, bm * sl2);
      if (__any(mn > acc.m + 8.f)) {  // (from -infinity: at the first key seen)
        const float alpha = mn == acc.m ? 1.f : __builtin_amdgcn_exp2f(acc.m - mn);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc.o[dt] *= alpha;
        acc.l *= alpha;
        acc.m = mn;
      }
      const float neg_m = acc.m == -INFINITY ? 0.f : -acc.m;
      // half a tile's weights and values at a time: the second half's weights run beside the first half's products
      uint4 v[2][2 * DT], p[2][2], p2[2][2];
      auto values = [&](int b) {
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) v[b][i] = *(const uint4*)(sv + (b * 2 + i / DT) * kPage + i % DT * 1024);
      };
      auto weights = [&](int b) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t w[4], w2[4];
          float sum[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = c * 8 + 2 * e;
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], sl2, neg_m));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], sl2, neg_m));
            sum[e] = p0 + p1;
            w[e] = TERMS == 2 ? split_pair(p0, p1, w2[e]) : round_pair(p0, p1);
          }
          if constexpr (TERMS == 2) p2[b][c] = make_uint4(w2[0], w2[1], w2[2], w2[3]);
          acc.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          p[b][c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      };
      auto products = [&](int b) {
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
          acc.o[i % DT] = mma_bf16(v[b][i], p[b][i / DT], acc.o[i % DT]);
          if constexpr (TERMS == 2) acc.o[i % DT] = mma_bf16(v[b][i], p2[b][i / DT], acc.o[i % DT]);
        }
      };
      auto clean = [&](int b) {
        if (!all) {
          uint32_t bits = 0;
#pragma unroll
          for (int i = 0; i < 2 * DT; ++i) {
            const uint4& x = v[b][i];
            bits |= odd_bits<uint16_t>(x.x) | odd_bits<uint16_t>(x.y) | odd_bits<uint16_t>(x.z) | odd_bits<uint16_t>(x.w);
          }
          if (__any(bits != 0)) {
            any_odd = true;
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i) {
              uint4& x = v[b][i];
              x = make_uint4(drop_odd<uint16_t>(x.x), drop_odd<uint16_t>(x.y), drop_odd<uint16_t>(x.z), drop_odd<uint16_t>(x.w));
            }
          }
        }
      };
      values(0);
      weights(0);
      clean(0);
      values(1);
      products(0);
      weights(1);
      clean(1);
      products(1);
    }
    pages = pages1;
    pages1 = pages2;
  }
  settle();
  if (any_odd) {  // (the same in all lanes)
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
      const int at = pages_of(t);
      // every half of a tile that was not whole
      const int kb = k0 + t * kTileKeys;
      if (!(__ballot(at < 0) & 15) && whole(kb)) continue;
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        const int page0 = __builtin_amdgcn_readlane(at, 2 * b), page1 = __builtin_amdgcn_readlane(at, 2 * b + 1);
        add_odd_values<uint16_t, HD>(a.c, g, page0, page1, ql, half,
                                     seen_keys<uint16_t>(q, kb + b * 32, page0 >= 0, page1 >= 0, half), acc);
      }
    }
  }
  if (!q.valid) return;
  const float l = acc.l + __shfl_xor(acc.l, 32, 64);  // (a query's two lanes are both valid)
  const bool direct = a.n_splits == 1;
  const float inv = direct ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
  const size_t at = ((size_t)split * a.c.rows + q.row) * a.H + q.head;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int d = dt * 32 + i4 * 8 + half * 4;
      const f32x16& o = acc.o[dt];
      const float x[4] = {o[i4 * 4] * inv, o[i4 * 4 + 1] * inv, o[i4 * 4 + 2] * inv, o[i4 * 4 + 3] * inv};
      if (direct)
        *(uint2*)((uint16_t*)a.out + (size_t)q.row * a.out_ld + (size_t)q.head * HD + d) =
            make_uint2(pack_bf16x2(f2bf(x[0]), f2bf(x[1])), pack_bf16x2(f2bf(x[2]), f2bf(x[3])));
      else
        *(float4*)(a.part_o + at * HD + d) = make_float4(x[0], x[1], x[2], x[3]);
    }
  if (half == 0) {
    if (!direct) {
      a.part_ml[at * 2] = acc.m;
      a.part_ml[at * 2 + 1] = l;
    } else if (a.lse) {
      a.lse[(size_t)q.row * a.H + q.head] = (acc.m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
  }
}

// Join the splits of each query in split order.  A work-group: one row, 1024 / HD
// heads, HD / 8 threads each (8 dims a thread).
template <typename T, int HD, bool LISTED>
__global__ __launch_bounds__(128) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int TPH = HD / 8, HPW = 128 / TPH;
  const int groups = (a.H + HPW - 1) / HPW;
  const int row = blockIdx.x / groups, head = (blockIdx.x % groups) * HPW + threadIdx.x / TPH, d = threadIdx.x % TPH * 8;
  const int seq = seq_of_row(a.c, row);
  if (seq < 0 || head >= a.H) return;
  int splits = a.n_splits;
  if constexpr (!LISTED) {
    int first, n, len, lo, end;
    seq_of_wave(a.c, seq, first, n, len);
    const int G = a.H / a.c.KVH;
    tile_keys(a, len, n, ((row - first) * G + head % G) / a.tile_q * a.tile_q, lo, end);
    splits = end > lo ? (int)min((long long)a.n_splits, ((long long)end - lo + a.span - 1) / a.span) : 0;
  }
  const size_t at = (size_t)row * a.H + head, step = (size_t)a.c.rows * a.H;
  float M = -INFINITY, L = 0.f, O[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += 8) {
    // eight splits' loads together (past the last: it again, with no weight)
    float4 v[8][2];
    float2 ml[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const size_t o = (size_t)min(s0 + i, splits - 1) * step + at;
      ml[i] = *(const float2*)(a.part_ml + o * 2);
      v[i][0] = *(const float4*)(a.part_o + o * HD + d);
      v[i][1] = *(const float4*)(a.part_o + o * HD + d + 4);
    }
    float mn = M;
#pragma unroll
    for (int i = 0; i < 8; ++i) mn = fmaxf(mn, s0 + i < splits ? ml[i].x : -INFINITY);
    const float c = mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    L *= c;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] *= c;
    M = mn;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s0 + i < splits) {
        const float w = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - M);
        L += ml[i].y * w;
        const float x[8] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w, v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) O[e] += x[e] * w;
      }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < 8; ++e) O[e] *= inv;
  T* out = (T*)a.out + (size_t)row * a.out_ld + (size_t)head * HD + d;
  if constexpr (sizeof(T) == 2) {
    *(uint4*)out = make_uint4(pack_bf16x2(f2bf(O[0]), f2bf(O[1])), pack_bf16x2(f2bf(O[2]), f2bf(O[3])),
                              pack_bf16x2(f2bf(O[4]), f2bf(O[5])), pack_bf16x2(f2bf(O[6]), f2bf(O[7])));
  } else {
    *(float4*)out = make_float4(O[0], O[1], O[2], O[3]);
    *(float4*)(out + 4) = make_float4(O[4], O[5], O[6], O[7]);
  }
  if (a.lse && d == 0) a.lse[at] = (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

template <typename T, int HD, bool LISTED>
void launch(const PagedAttnArgs& a, hipStream_t s) {
  const int blocks = a.n_items * a.c.KVH * a.n_splits;
  if constexpr (sizeof(T) == 2 && !LISTED) {
    if (a.tile_q == kTileQueries && a.terms == 2)
      hipLaunchKernelGGL((paged_tile_kernel<HD, 2>), dim3(blocks), dim3(256), 0, s, a);
    else if (a.tile_q == kTileQueries)
      hipLaunchKernelGGL((paged_tile_kernel<HD, 1>), dim3(blocks), dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((paged_stream_kernel<T, HD, LISTED>), dim3(blocks), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((paged_stream_kernel<T, HD, LISTED>), dim3(blocks), dim3(256), 0, s, a);
  }
  if (a.n_splits > 1) {
    const int hpw = 128 / (HD / 8);
    hipLaunchKernelGGL((paged_join_kernel<T, HD, LISTED>), dim3(a.c.rows * ((a.H + hpw - 1) / hpw)), dim3(128), 0, s, a);
  }
}
template <typename T, int HD>
void launch(const PagedAttnArgs& a, hipStream_t s) {
  a.sel ? launch<T, HD, true>(a, s) : launch<T, HD, false>(a, s);
}

}  // namespace

void launch_paged_attention(bool bf16, const PagedAttnArgs& a, hipStream_t s) {
  if (a.hd == 128)
    bf16 ? launch<uint16_t, 128>(a, s) : launch<float, 128>(a, s);
  else
    bf16 ? launch<uint16_t, 64>(a, s) : launch<float, 64>(a, s);
}

}  // namespace via
