// What the kernels that read the paged key-value cache share (attn_decode.cu, attn_weights.cu): which keys a warp's thread
// holds, how they travel from the pages into registers, the heads that read a KV position, their queries, and the scores.
// The reasons for the layout stand in attn_decode.cu.  D: elements of a head; B: bytes of a cached element, 2 (bf16) or 1 (e4m3
// beside a scale for each 16 keys of a KV position).
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kCols = 8;                   // heads per pass over the keys (columns of the MMA tile)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

struct DecParams {
  const __nv_bfloat16* q;
  const void* k;              // elements of B bytes
  const void* v;
  const float2* scales;       // 8 bits: (K, V) of every 16 tokens [n_pages][kv_max][page_size / 16]
  const int32_t* table;
  const int32_t* len;
  const int32_t* head_idx;
  const int32_t* kv_pos;
  __nv_bfloat16* out;
  float* lse;
  float* part;                // [2 G][kCols][D + 4]: see kPartRow
  int4* desc;                 // [items or warps] a cut item: (sequence, heads, further parts, warp that has its beginning)
  long long page_stride, q_stride;
  int S, n_seqs, heads, kv_max, per_group, n_kv_heads, row_tiles;
  int by_item;                // desc has an entry for every item (few items), else one for every warp
  int page_shift, n_pages, max_pages;
  float scale_log2;
  int quit_every, quit_tile;  // self-test: the warps that give up, and before which tile of an item
  int* status;
};

__device__ inline void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 matrix of 16-bit elements held as one row-pair per thread, transposed across the warp.
__device__ inline uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ inline float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&t);
}
__device__ inline void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ inline uint32_t pack_f16(float lo, float hi) {
  __half2 t = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&t);
}
// Four e4m3 numbers as two pairs of fp16 (exact).
__device__ inline void widen(uint32_t v, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(v));
}
__device__ inline float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ inline float hi_f(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// `W` 32-bit words (W = 4, 2, 1) of a row that is read once.  Coherent loads: the launch before may still be writing the cache
// when this one is placed (see launch_overlapped).
template <int W>
__device__ inline void load_words(uint32_t (&r)[W], const void* p) {
  if constexpr (W == 4)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
  else if constexpr (W == 2)
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
  else
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(r[0]) : "l"(p));
}

// An element of the cache: B bytes, bf16 or e4m3.
template <int B>
using Elem = std::conditional_t<B == 2, __nv_bfloat16, uint8_t>;

// How a thread (g = lane / 4, t = lane % 4) holds a tile.  K: rows g and g + 8 of each 16 keys, KCH chunks of KW words at
// word c * 4 KW + t * KW.  V: rows 2t, 2t+1, 2t+8, 2t+9, VCH chunks of VW words at word (c * 8 + g) * VW.  (d = 8 in 16 bits and
// d = 16 in 8: V has half a word per thread; d = 8: the upper half of the MMA tile is zero.)
template <int D, int B>
struct Shape {
  static constexpr int ROW = D * B / 4;                     // words of a row
  static constexpr int KW = ROW >= 16 ? 4 : ROW / 4;
  static constexpr int KCH = ROW / (4 * KW);
  static constexpr bool HALF_V = ROW == 4;
  static constexpr int VW = ROW >= 32 ? 4 : (HALF_V ? 1 : ROW / 8);
  static constexpr int VCH = HALF_V ? 1 : ROW / (8 * VW);
  static constexpr int MT = D >= 16 ? D / 16 : 1;           // MMA tiles over d
  static constexpr int SUB = D >= 64 ? (D == 64 && B == 1 ? 2 : 1) : 4;      // steps of 16 keys
  static constexpr int TILE = 16 * SUB;
  static constexpr int QW = KW * 2 / B;                     // words of a query beside KW words of a key
  static constexpr int PER = 4 / B;                         // elements of a word
};

template <int D, int B>
struct Tile {
  using Sh = Shape<D, B>;
  uint32_t k[Sh::SUB][2][Sh::KCH][Sh::KW];
  uint32_t v[Sh::SUB][4][Sh::VCH][Sh::VW];
  float2 scale;                                             // 8 bits: of step lane % SUB
};

// Page ids of coming tiles, fetched ahead, one 16-key step per lane, so that no key waits for its page entry: lane l gets
// the entry of step l % SUB of the tile `tile0 + (l / SUB) * stride`.  The read stays inside the sequence's row of the
// table whatever its length is, so it need not wait for that.
template <int SUB>
__device__ inline uint32_t step_key(int tile0, int stride, int lane) {
  return ((uint32_t)tile0 + (uint32_t)(lane / SUB) * stride) * (16 * SUB) + 16 * (lane % SUB);
}
template <int SUB>
__device__ inline int fetch_pages(const DecParams& p, long long seq, int tile0, int stride, int lane) {
  return p.table[seq * p.max_pages + min(step_key<SUB>(tile0, stride, lane) >> p.page_shift, (uint32_t)p.max_pages - 1)];
}
// Before use: an entry outside the pool is replaced by page 0, and reported if a key of the sequence needs it.
template <int SUB>
__device__ inline int check_pages(const DecParams& p, int id, int last_key, int tile0, int stride, int lane) {
  if ((unsigned)id >= (unsigned)p.n_pages) {
    if (last_key >= 0 && step_key<SUB>(tile0, stride, lane) <= (uint32_t)last_key) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
    id = 0;
  }
  return id;
}

// Rows behind a sequence's end must not reach the products, whatever they hold.  Two ways.  CLAMP: they are replaced by rows
// before it, whose scores are masked.  Otherwise they are read as they are (a page has all its rows) and the values
// cleared right before their product: fewer instructions in every tile, but up to 15 rows more are read per item.
// Measured, cleared against clamped, 64 sequences of up to 16000 keys, 32 heads on 4: d = 8 51.9 us against 60.5, d = 16 33.9
// against 35.1, d = 32 54.2 against 54.6, d = 64 91.8 against 92.5 (short items are the other way round there: 15232 of 274
// keys, 181 against 177); d = 128, where a tile has half the rows a thread, 952 ragged sequences of up to 274 keys on 4
// positions: 54.2 against 52.1, eight subnets of long sequences 351.8 against 350.9.  Neither a predicate on the loads nor
// clearing the values before the softmax is an alternative: the compiler then waits for them long before their use (a fifth
// more time with tiles of 32 keys).
template <int D, int B>
constexpr bool kClamp = D == 128 && B == 2;

// The tile that begins at key0 <= last_key, number n of its window of page ids: `put(step, row, chunk, address)` is called
// for every piece that this thread (g, t) holds.  Steps that lie wholly behind the end are replaced by the tile's first.
template <int D, int B, typename Put>
__device__ inline void tile_k(const DecParams& p, int ids, int n, int key0, int last_key, long long at, int g, Put put) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int step = key0 + 16 * s <= last_key ? s : 0, key = key0 + 16 * step;
    const int id = __shfl_sync(0xffffffffu, ids, n * Sh::SUB + step);
    const Elem<B>* row = static_cast<const Elem<B>*>(p.k) + (id * p.page_stride + (key & ((1 << p.page_shift) - 1)) * D + at);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int down = kClamp<D, B> ? min(g + 8 * r, last_key - key) - g : 8 * r;
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c) put(s, r, c, row + down * D + c * 4 * Sh::KW * Sh::PER);
    }
  }
}
template <int D, int B, typename Put>
__device__ inline void tile_v(const DecParams& p, int ids, int n, int key0, int last_key, long long at, int t, Put put) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int step = key0 + 16 * s <= last_key ? s : 0, key = key0 + 16 * step;
    const int id = __shfl_sync(0xffffffffu, ids, n * Sh::SUB + step);
    const Elem<B>* row = static_cast<const Elem<B>*>(p.v) + (id * p.page_stride + (key & ((1 << p.page_shift) - 1)) * D + at);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int to = (r & 1) + 8 * (r >> 1), down = kClamp<D, B> ? min(2 * t + to, last_key - key) - 2 * t : to;
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c) put(s, r, c, row + down * D + c * 8 * Sh::VW * Sh::PER);
    }
  }
}
// Offsets inside a page of the pieces of thread (g, t) for KV position `pos`: its first row and element.
template <int D, int B>
__device__ inline long long at_k(const DecParams& p, int pos, int g, int t) {
  return (((long long)pos << p.page_shift) + g) * D + t * Shape<D, B>::KW * Shape<D, B>::PER;
}
template <int D, int B>
__device__ inline long long at_v(const DecParams& p, int pos, int g, int t) {
  return (((long long)pos << p.page_shift) + 2 * t) * D + (Shape<D, B>::HALF_V ? g * 2 / B : g * Shape<D, B>::VW * Shape<D, B>::PER);
}

// The scales of the tile's steps (8 bits), the lane's own the one of step lane % SUB.
template <int D, int B>
__device__ inline const float2* scale_at(const DecParams& p, int ids, int n, int key0, int last_key, int pos, int lane) {
  constexpr int SUB = Shape<D, B>::SUB;
  const int mine = lane % SUB, step = key0 + 16 * mine <= last_key ? mine : 0, key = key0 + 16 * step;
  const int id = __shfl_sync(0xffffffffu, ids, n * SUB + step);
  return p.scales + ((((long long)id * p.kv_max + pos) << (p.page_shift - 4)) + ((key & ((1 << p.page_shift) - 1)) >> 4));
}
__device__ inline float2 load_scale(const float2* a) {
  float2 v;
  asm volatile("ld.global.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(a));
  return v;
}

template <int D, int B>
__device__ inline void load_k(Tile<D, B>& x, const DecParams& p, int ids, int n, int key0, int last_key, int pos, long long at, int lane) {
  if constexpr (B == 1) x.scale = load_scale(scale_at<D, B>(p, ids, n, key0, last_key, pos, lane));
  auto put = [&](int s, int r, int c, const Elem<B>* a) { load_words<Shape<D, B>::KW>(x.k[s][r][c], a); };
  tile_k<D, B>(p, ids, n, key0, last_key, at, lane >> 2, put);
}
template <int D, int B>
__device__ inline void load_v(Tile<D, B>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int lane) {
  auto put = [&](int s, int r, int c, const Elem<B>* a) {
    if constexpr (Shape<D, B>::HALF_V) x.v[s][r][c][0] = *reinterpret_cast<const unsigned short*>(a);
    else load_words<Shape<D, B>::VW>(x.v[s][r][c], a);
  };
  tile_v<D, B>(p, ids, n, key0, last_key, at, lane & 3, put);
}

// The same pieces through shared memory, two tiles deep, where registers do not suffice: every thread copies its own
// pieces asynchronously to places of its own and reads them back itself, so nothing is waited for but the copies.
template <int D, int B>
struct Stage {
  using Sh = Shape<D, B>;
  uint32_t k[Sh::SUB][2][Sh::KCH][32][Sh::KW];
  uint32_t v[Sh::SUB][4][Sh::VCH][32][Sh::VW];
};
template <int BYTES>
__device__ inline void copy_async(const void* smem, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem)), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(smem)), "l"(src), "n"(BYTES) : "memory");
}
__device__ inline void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ inline void wait_copies_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int D, int B>
__device__ inline void stage_k(Stage<D, B>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int lane) {
  auto put = [&](int s, int r, int c, const Elem<B>* a) { copy_async<4 * Shape<D, B>::KW>(x.k[s][r][c][lane], a); };
  tile_k<D, B>(p, ids, n, key0, last_key, at, lane >> 2, put);
}
template <int D, int B>
__device__ inline void stage_v(Stage<D, B>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int lane) {
  auto put = [&](int s, int r, int c, const Elem<B>* a) { copy_async<4 * Shape<D, B>::VW>(x.v[s][r][c][lane], a); };
  tile_v<D, B>(p, ids, n, key0, last_key, at, lane & 3, put);
}
template <int D, int B>
__device__ inline void take_k(Tile<D, B>& x, const Stage<D, B>& y, int lane) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
        for (int w = 0; w < Sh::KW; ++w) x.k[s][r][c][w] = y.k[s][r][c][lane][w];
}
template <int D, int B>
__device__ inline void take_v(Tile<D, B>& x, const Stage<D, B>& y, int lane) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c)
#pragma unroll
        for (int w = 0; w < Sh::VW; ++w) x.v[s][r][c][w] = y.v[s][r][c][lane][w];
}

template <int W>
__device__ inline void take_words(uint32_t (&r)[W], const uint8_t* a) {
  if constexpr (W == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(a);
    r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
  } else if constexpr (W == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(a);
    r[0] = v.x; r[1] = v.y;
  } else {
    r[0] = *reinterpret_cast<const uint32_t*>(a);
  }
}
// 16 keys whose rows lie one behind another in shared memory.
template <int D, int B>
__device__ inline void take_keys(uint32_t (&x)[2][Shape<D, B>::KCH][Shape<D, B>::KW], const uint8_t* k, int g, int t) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < Sh::KCH; ++c) take_words<Sh::KW>(x[r][c], k + (8 * r + g) * D * B + 4 * Sh::KW * (4 * c + t));
}

// Where a CTA finds the index data of the heads: in shared memory where it fits, copied with the first loads of the kernel.
struct Heads {
  const int32_t* idx;         // [S][heads] or null
  const int32_t* pos;         // [S][n_kv_heads]
};
constexpr int kHeadCache = 512, kPosCache = 256;

__device__ inline void copy_words(int32_t* dst, const int32_t* src, int n) {
  for (int i = threadIdx.x; i < n; i += kDecThreads)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst + i)), "l"(src + i) : "memory");
}
// Begins the copy of the rows of `subnets` subnets from subnet s0 on (complete after wait_copies and a barrier).
__device__ inline Heads cache_heads(const DecParams& p, int32_t* idx, int32_t* pos, int s0, int subnets) {
  Heads h{p.head_idx, p.kv_pos};
  if (p.head_idx && subnets * p.heads <= kHeadCache && subnets * p.n_kv_heads <= kPosCache) {
    copy_words(idx, p.head_idx + (long long)s0 * p.heads, subnets * p.heads);
    copy_words(pos, p.kv_pos + (long long)s0 * p.n_kv_heads, subnets * p.n_kv_heads);
    h.idx = idx - (long long)s0 * p.heads;                      // indexed by the subnet's own number
    h.pos = pos - (long long)s0 * p.n_kv_heads;
  }
  return h;
}
__device__ inline void wait_copies() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// KV position among the subnet's kept groups that kept head hq reads, checked.
__device__ inline int position_of(const DecParams& p, const Heads& hd, int s, int hq) {
  const int h = hd.idx[(long long)s * p.heads + hq];
  int g = h < 0 ? -1 : h / p.per_group;
  if ((unsigned)g >= (unsigned)p.n_kv_heads) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); g = 0; }
  int pos = hd.pos[(long long)s * p.n_kv_heads + g];
  if ((unsigned)pos >= (unsigned)p.kv_max) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); pos = 0; }
  return pos;
}

// The kept heads number 8 rt .. 8 rt + 7 among those that read KV position `pos`, into cols[0..7] (-1: none).  One warp.
// A position takes as many heads as a group has (what the join is launched for): more, by a list that repeats heads or
// sends two groups to one position, are reported and left out.
__device__ inline void find_heads(const DecParams& p, const Heads& hd, int s, int pos, int rt, int lane, int* cols) {
  if (!p.head_idx) {
    if (lane < kCols) cols[lane] = lane == 0 ? pos : -1;
    __syncwarp();
    return;
  }
  if (lane < kCols) cols[lane] = -1;
  __syncwarp();
  int seen = 0;
  for (int h0 = 0; h0 < p.heads; h0 += 32) {
    const int hq = h0 + lane;
    const bool mine = hq < p.heads && position_of(p, hd, s, hq) == pos;
    const unsigned vote = __ballot_sync(0xffffffffu, mine);
    const int number = seen + __popc(vote & ((1u << lane) - 1)), rank = number - kCols * rt;
    if (mine && number < p.per_group && rank >= 0 && rank < kCols) cols[rank] = hq;
    seen += __popc(vote);
  }
  if (lane == 0 && rt == 0 && seen > p.per_group) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
  __syncwarp();
}

// Queries of the warp's columns in the order the K loads have (column g of this thread: head hq, -1: none), copied to
// shared memory ahead of their use: every thread copies and later reads its own words.
template <int D, int B>
struct QueryBuf {
  uint32_t w[Shape<D, B>::KCH][32][Shape<D, B>::QW];
};

template <int D, int B>
__device__ inline void prefetch_q(QueryBuf<D, B>& buf, const DecParams& p, long long seq, int hq, int lane) {
  using Sh = Shape<D, B>;
  constexpr int STEP = Sh::QW < 4 ? Sh::QW : 4;             // words of a copy
  const __nv_bfloat16* row = p.q + seq * p.q_stride + (long long)(hq < 0 ? 0 : hq) * D + (lane & 3) * 2 * Sh::QW;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
    for (int w = 0; w < Sh::QW; w += STEP)
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(smem_u32(buf.w[c][lane] + w)), "l"(row + c * 8 * Sh::QW + 2 * w),
                   "n"(4 * STEP), "r"(hq < 0 ? 0 : 4 * STEP) : "memory");
}

// The queries as an operand.  Beside e4m3 keys they are fp16, every head's brought near 2^15 by a power of two (f0, f1 undo it
// for the thread's heads 2t and 2t + 1): what is more than 2^29 below the head's largest element loses bits, which is less than
// an fp32 sum keeps of it.  Elements that are not finite stay what they are.
template <int D, int B>
struct Query {
  uint32_t w[Shape<D, B>::KCH][Shape<D, B>::QW];
  float f0, f1;
};
template <int D, int B>
__device__ inline void take_q(Query<D, B>& q, const QueryBuf<D, B>& buf, int lane) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
    for (int w = 0; w < Sh::QW; ++w) q.w[c][w] = buf.w[c][lane][w];
  if constexpr (B == 1) {
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
      for (int w = 0; w < Sh::QW; ++w) {
        const float x = fabsf(lo_f(q.w[c][w])), y = fabsf(hi_f(q.w[c][w]));
        top = fmaxf(top, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 127);      // top < 2^(e + 1)
    const float up = __uint_as_float((uint32_t)(min(14 - e, 127) + 127) << 23), down = __uint_as_float((uint32_t)(max(e - 14, -126) + 127) << 23);
#pragma unroll
    for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
      for (int w = 0; w < Sh::QW; ++w) q.w[c][w] = pack_f16(lo_f(q.w[c][w]) * up, hi_f(q.w[c][w]) * up);
    q.f0 = __shfl_sync(0xffffffffu, down, 8 * (lane & 3));
    q.f1 = __shfl_sync(0xffffffffu, down, 8 * (lane & 3) + 4);
  }
}

// The scales (K in x, V in y) of a tile's steps (8 bits).
template <int D, int B>
struct Scales {
  float2 of[B == 1 ? Shape<D, B>::SUB : 1];
};
// From the lanes that loaded them.
template <int D, int B>
__device__ inline Scales<D, B> gather_scales(const Tile<D, B>& x) {
  Scales<D, B> r{};
  if constexpr (B == 1) {
#pragma unroll
    for (int s = 0; s < Shape<D, B>::SUB; ++s)
      r.of[s] = Shape<D, B>::SUB == 1 ? x.scale : make_float2(__shfl_sync(0xffffffffu, x.scale.x, s), __shfl_sync(0xffffffffu, x.scale.y, s));
  }
  return r;
}

// Scores q . k of 16 keys: thread (g, t) has keys g, g + 8 and heads 2t, 2t + 1.
template <int D, int B>
__device__ inline void step_scores(float (&sc)[4], const uint32_t (&k)[2][Shape<D, B>::KCH][Shape<D, B>::KW], const Query<D, B>& q, float scale) {
  using Sh = Shape<D, B>;
#pragma unroll
  for (int e = 0; e < 4; ++e) sc[e] = 0.f;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c) {
    if constexpr (B == 1) {
#pragma unroll
      for (int w = 0; w < Sh::KW; ++w) {
        uint32_t a0, a1, a2, a3;
        widen(k[0][c][w], a0, a2);
        widen(k[1][c][w], a1, a3);
        mma16816_f16(sc, a0, a1, a2, a3, q.w[c][2 * w], q.w[c][2 * w + 1]);
      }
    } else if constexpr (Sh::KW == 4) {
#pragma unroll
      for (int h = 0; h < 4; h += 2) mma16816(sc, k[0][c][h], k[1][c][h], k[0][c][h + 1], k[1][c][h + 1], q.w[c][h], q.w[c][h + 1]);
    } else if constexpr (Sh::KW == 2) {
      mma16816(sc, k[0][c][0], k[1][c][0], k[0][c][1], k[1][c][1], q.w[c][0], q.w[c][1]);
    } else {
      mma16816(sc, k[0][c][0], k[1][c][0], 0u, 0u, q.w[c][0], 0u);
    }
  }
  if constexpr (B == 1) {
    // (finite: a product that is zero stays zero beside a scale and a query whose sizes are beyond fp32 together)
    const float f0 = fminf(scale * q.f0, 0x1p127f), f1 = fminf(scale * q.f1, 0x1p127f);
    sc[0] *= f0; sc[1] *= f1; sc[2] *= f0; sc[3] *= f1;
  }
}
template <int D, int B>
__device__ inline void tile_scores(float (&sc)[Shape<D, B>::SUB][4], const Tile<D, B>& x, const Query<D, B>& q, const Scales<D, B>& scale) {
#pragma unroll
  for (int s = 0; s < Shape<D, B>::SUB; ++s) step_scores<D, B>(sc[s], x.k[s], q, B == 1 ? scale.of[B == 1 ? s : 0].x : 1.f);
}

__device__ inline int clamped_len(const DecParams& p, int n) {
  const int most = p.max_pages << p.page_shift;
  if (n < 0 || n > most) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); n = n < 0 ? 0 : most; }
  return n;
}

}  // namespace
}  // namespace twist
