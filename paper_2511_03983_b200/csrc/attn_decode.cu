// twist_attn_decode: attention of one new token per sequence over a paged key-value cache,
//     out_h = sum_j softmax_j(q_h . k_j / sqrt(d)) v_j,
// split over the cache's length and joined.  Every cached K and V element is read once from memory and used by the few
// heads that share it, so the kernel is bound by HBM: the design keeps as many bytes as possible in flight and spends as
// few instructions per byte as possible.
//
// One pass, from registers.  A warp takes tiles of 16 * SUB keys of one KV position.  Both products run on the warp-level
// tensor instruction (mma m16n8k16) in the transposed form: S^T = K Q^T (16 keys x 8 heads) and O^T += V^T P^T
// (d x 8 heads), so up to eight heads that share a KV position ride on one pass over its keys, and a lone head costs
// no more than eight.  The operands come straight from global memory into registers with 16-byte loads: the order of
// the contraction index is free, so the thread that owns four consecutive k-indices of two MMA steps simply loads
// eight consecutive elements (the query is loaded in the same order), and the rows of V^T a thread owns are chosen as
// eight consecutive elements of a cached row, paired over keys by a byte permute.  No shared memory, no barrier in the
// loop; the next tile's loads are issued as soon as the registers of this one have been consumed, so a warp keeps about
// a tile in flight all the time (4 KB and 16 warps an SM at d = 64, 8 KB and 12 warps at d = 128; at d = 64 two steps a
// tile and 12 warps were 3 to 6 % slower, at d = 128 two steps and 8 warps 8 %).  Smaller heads spend more instructions
// on a byte, and the registers of one tile do not cover the latency: there the tiles pass through shared memory, two
// deep (d = 32: 113 -> 83 us for 463 MB; the same at d = 64 and 128 is 15 to 50 % slower, its copies of half and whole
// rows being issued piece by piece through the same queue; bulk copies of whole rows have not been tried).  (tcgen05 takes
// its operands from shared and tensor memory, where the keys and the probabilities would have to be laid out for it first;
// with 1 to 12 operations a byte the products are far from bounding this kernel.)
//
// Softmax in fp32 with a running reference maximum per head that moves only when a score exceeds it by more than 2^8 (one
// vote per tile instead of a reduction).  The probabilities enter the second product as the sum of two bf16 numbers
// (value and remainder: 16 bits), so that rounding them costs nothing against the one rounding of the result.
//
// Splitting.  The work of a call is a line of tiles: sequence after sequence, KV position after KV position.  Warp w of G
// takes the w-th G-th of the line, whatever the lengths are: a ragged batch is balanced on the device, and a warp's loads
// run on across the borders of items (an item: the tiles of one KV position of one sequence).  A warp writes the items it
// has whole; of an item that a border between warps cuts, every warp writes its unnormalised part (fp32 sums, maximum,
// sum) to the workspace, and a second small launch joins the parts in the order of the warps.
//
// Calls whose length and number of items leave little to balance take a shorter way instead: one cluster of 1 to 8 CTAs
// per item, whose warps take the item's tiles in turn and join through (distributed) shared memory: one launch, no
// workspace.
#include <cooperative_groups.h>

#include "common.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kCols = 8;                   // heads per pass over the keys (columns of the MMA tile)
constexpr int kMaxCtasPerSm = 4;
constexpr int kItemCost = 1;               // what changing to the next item costs a warp, in tiles
constexpr int kMinCost = 2;                // least work of a warp, in tiles
constexpr int kJoinThreads = 512;
// The short way, one cluster per item (see run).
constexpr int kMaxCluster = 8, kShortTiles = 8, kShortWork = 8, kShortWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kSlack = 8.0f;             // log2 headroom of the lazily moved reference maximum

struct DecParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
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
  int* status;
};

// Row of a part: d sums, then maximum (log2), sum of probabilities, head, padding.
__host__ __device__ constexpr int kPartRow(int d) { return d + 4; }

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
// Weight of a part with maximum x (log2) and sum l against the maximum m of all parts.  A part without a reference maximum
// has no finite score: it counts for nothing, unless its sum is NaN.
__device__ inline float part_weight(float x, float l, float m) { return x == -INFINITY ? (l == 0.f ? 0.f : 1.f) : ex2(x - m); }
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&t);
}
__device__ inline float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ inline float hi_f(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// `W` 32-bit words (W = 4, 2, 1) of a row that is read once.  Coherent loads: the launch before may still be writing the cache
// when this one is placed (see launch_overlapped).
template <int W>
__device__ inline void load_words(uint32_t (&r)[W], const __nv_bfloat16* p) {
  if constexpr (W == 4)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
  else if constexpr (W == 2)
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
  else
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(r[0]) : "l"(p));
}

// How a thread (g = lane / 4, t = lane % 4) holds a tile.  K: rows g and g + 8 of each 16 keys, KCH chunks of KW words
// (2 KW elements) at element c * 8 KW + t * 2 KW.  V: rows 2t, 2t+1, 2t+8, 2t+9, VCH chunks of VW words at element
// c * 64 + g * 2 VW.  (d = 8: V has half a word per thread, and the upper half of the MMA tile is zero.)
template <int D>
struct Shape {
  static constexpr int KCH = D >= 64 ? D / 32 : 1;
  static constexpr int KW = D >= 32 ? 4 : D / 8;
  static constexpr int VCH = D == 128 ? 2 : 1;
  static constexpr int VW = D >= 64 ? 4 : (D >= 16 ? D / 16 : 1);
  static constexpr int MT = D >= 16 ? D / 16 : 1;           // MMA tiles over d
  static constexpr int SUB = D >= 64 ? 1 : 4;
  static constexpr int TILE = 16 * SUB;
};

template <int D>
struct Tile {
  using Sh = Shape<D>;
  uint32_t k[Sh::SUB][2][Sh::KCH][Sh::KW];
  uint32_t v[Sh::SUB][4][Sh::VCH][Sh::VW];
};

// Page ids of coming tiles, fetched ahead, one 16-key step per lane, so that no key waits for its page entry: lane l gets
// the entry of step l % SUB of the tile `tile0 + (l / SUB) * stride`.  The read stays inside the sequence's row of the
// table whatever its length is, so it need not wait for that.
template <int D>
__device__ inline uint32_t step_key(int tile0, int stride, int lane) {
  constexpr int SUB = Shape<D>::SUB;
  return ((uint32_t)tile0 + (uint32_t)(lane / SUB) * stride) * Shape<D>::TILE + 16 * (lane % SUB);
}
template <int D>
__device__ inline int fetch_pages(const DecParams& p, long long seq, int tile0, int stride, int lane) {
  return p.table[seq * p.max_pages + min(step_key<D>(tile0, stride, lane) >> p.page_shift, (uint32_t)p.max_pages - 1)];
}
// Before use: an entry outside the pool is replaced by page 0, and reported if a key of the sequence needs it.
template <int D>
__device__ inline int check_pages(const DecParams& p, int id, int last_key, int tile0, int stride, int lane) {
  if ((unsigned)id >= (unsigned)p.n_pages) {
    if (last_key >= 0 && step_key<D>(tile0, stride, lane) <= (uint32_t)last_key) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
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
template <int D>
constexpr bool kClamp = D == 128;

// The tile that begins at key0 <= last_key, number n of its window of page ids: `put(step, row, chunk, address)` is called
// for every piece that this thread (g, t) holds.  Steps that lie wholly behind the end are replaced by the tile's first.
template <int D, typename Put>
__device__ inline void tile_k(const DecParams& p, int ids, int n, int key0, int last_key, long long at, int g, Put put) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int step = key0 + 16 * s <= last_key ? s : 0, key = key0 + 16 * step;
    const int id = __shfl_sync(0xffffffffu, ids, n * Sh::SUB + step);
    const __nv_bfloat16* row = p.k + (id * p.page_stride + (key & ((1 << p.page_shift) - 1)) * D + at);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int down = kClamp<D> ? min(g + 8 * r, last_key - key) - g : 8 * r;
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c) put(s, r, c, row + down * D + c * 8 * Sh::KW);
    }
  }
}
template <int D, typename Put>
__device__ inline void tile_v(const DecParams& p, int ids, int n, int key0, int last_key, long long at, int t, Put put) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int step = key0 + 16 * s <= last_key ? s : 0, key = key0 + 16 * step;
    const int id = __shfl_sync(0xffffffffu, ids, n * Sh::SUB + step);
    const __nv_bfloat16* row = p.v + (id * p.page_stride + (key & ((1 << p.page_shift) - 1)) * D + at);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int to = (r & 1) + 8 * (r >> 1), down = kClamp<D> ? min(2 * t + to, last_key - key) - 2 * t : to;
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c) put(s, r, c, row + down * D + c * 64);
    }
  }
}
// Offsets inside a page of the pieces of thread (g, t) for KV position `pos`: its first row and element.
template <int D>
__device__ inline long long at_k(const DecParams& p, int pos, int g, int t) {
  return (((long long)pos << p.page_shift) + g) * D + t * 2 * Shape<D>::KW;
}
template <int D>
__device__ inline long long at_v(const DecParams& p, int pos, int g, int t) {
  return (((long long)pos << p.page_shift) + 2 * t) * D + (D == 8 ? g : g * 2 * Shape<D>::VW);
}

template <int D>
__device__ inline void load_k(Tile<D>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int g) {
  auto put = [&](int s, int r, int c, const __nv_bfloat16* a) { load_words<Shape<D>::KW>(x.k[s][r][c], a); };
  tile_k<D>(p, ids, n, key0, last_key, at, g, put);
}
template <int D>
__device__ inline void load_v(Tile<D>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int t) {
  auto put = [&](int s, int r, int c, const __nv_bfloat16* a) {
    if constexpr (D == 8) x.v[s][r][c][0] = *reinterpret_cast<const unsigned short*>(a);
    else load_words<Shape<D>::VW>(x.v[s][r][c], a);
  };
  tile_v<D>(p, ids, n, key0, last_key, at, t, put);
}

// The same pieces through shared memory, two tiles deep, where registers do not suffice: every thread copies its own
// pieces asynchronously to places of its own and reads them back itself, so nothing is waited for but the copies.
template <int D>
struct Stage {
  using Sh = Shape<D>;
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
template <int D>
__device__ inline void stage_k(Stage<D>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int lane) {
  auto put = [&](int s, int r, int c, const __nv_bfloat16* a) { copy_async<4 * Shape<D>::KW>(x.k[s][r][c][lane], a); };
  tile_k<D>(p, ids, n, key0, last_key, at, lane >> 2, put);
}
template <int D>
__device__ inline void stage_v(Stage<D>& x, const DecParams& p, int ids, int n, int key0, int last_key, long long at, int lane) {
  auto put = [&](int s, int r, int c, const __nv_bfloat16* a) { copy_async<4 * Shape<D>::VW>(x.v[s][r][c][lane], a); };
  tile_v<D>(p, ids, n, key0, last_key, at, lane & 3, put);
}
template <int D>
__device__ inline void take_k(Tile<D>& x, const Stage<D>& y, int lane) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
        for (int w = 0; w < Sh::KW; ++w) x.k[s][r][c][w] = y.k[s][r][c][lane][w];
}
template <int D>
__device__ inline void take_v(Tile<D>& x, const Stage<D>& y, int lane) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c)
#pragma unroll
        for (int w = 0; w < Sh::VW; ++w) x.v[s][r][c][w] = y.v[s][r][c][lane][w];
}

// Running state of a warp: up to eight heads (columns); the thread's columns are 2t and 2t + 1.
template <int D>
struct State {
  float o[Shape<D>::MT][4];
  float m0, m1, l0, l1;
};

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

template <int D>
__device__ inline void reset(State<D>& st) {
#pragma unroll
  for (int i = 0; i < Shape<D>::MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[i][e] = 0.f;
  st.m0 = st.m1 = -INFINITY;
  st.l0 = st.l1 = 0.f;
}

// Queries of the warp's columns in the order the K loads have (column g of this thread: head hq, -1: none), copied to
// shared memory ahead of their use: every thread copies and later reads its own words.
template <int D>
struct QueryBuf {
  uint32_t w[Shape<D>::KCH][32][Shape<D>::KW];
};

template <int D>
__device__ inline void prefetch_q(QueryBuf<D>& buf, const DecParams& p, long long seq, int hq, int lane) {
  using Sh = Shape<D>;
  const __nv_bfloat16* row = p.q + seq * p.q_stride + (long long)(hq < 0 ? 0 : hq) * D + (lane & 3) * 2 * Sh::KW;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c)
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(smem_u32(buf.w[c][lane])), "l"(row + c * 8 * Sh::KW),
                 "n"(4 * Sh::KW), "r"(hq < 0 ? 0 : 4 * Sh::KW) : "memory");
}

template <int D>
__device__ inline void take_q(uint32_t (&q)[Shape<D>::KCH][Shape<D>::KW], const QueryBuf<D>& buf, int lane) {
  using Sh = Shape<D>;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c)
#pragma unroll
    for (int w = 0; w < Sh::KW; ++w) q[c][w] = buf.w[c][lane][w];
}

// Raw scores q . k of a tile: thread (g, t) has keys g, g + 8 of each 16 and heads 2t, 2t + 1.
template <int D>
__device__ inline void tile_scores(float (&sc)[Shape<D>::SUB][4], const Tile<D>& x, const uint32_t (&q)[Shape<D>::KCH][Shape<D>::KW]) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[s][e] = 0.f;
#pragma unroll
    for (int c = 0; c < Sh::KCH; ++c) {
      if constexpr (Sh::KW == 4) {
#pragma unroll
        for (int h = 0; h < 4; h += 2)
          mma16816(sc[s], x.k[s][0][c][h], x.k[s][1][c][h], x.k[s][0][c][h + 1], x.k[s][1][c][h + 1], q[c][h], q[c][h + 1]);
      } else if constexpr (Sh::KW == 2) {
        mma16816(sc[s], x.k[s][0][c][0], x.k[s][1][c][0], x.k[s][0][c][1], x.k[s][1][c][1], q[c][0], q[c][1]);
      } else {
        mma16816(sc[s], x.k[s][0][c][0], x.k[s][1][c][0], 0u, 0u, q[c][0], 0u);
      }
    }
  }
}

// Softmax step and O^T += V^T P^T of the tile that begins at key0 of `len` keys.
template <int D>
__device__ inline void tile_values(State<D>& st, float (&sc)[Shape<D>::SUB][4], Tile<D>& x, float scale_log2, int key0, int len, int g, int t) {
  using Sh = Shape<D>;
  if (key0 + Sh::TILE > len) {                     // keys behind the end count for nothing
#pragma unroll
    for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key0 + 16 * s + g + 8 * (e >> 1) >= len) sc[s][e] = -INFINITY;
  }
  float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    mx0 = fmaxf(mx0, fmaxf(sc[s][0], sc[s][2]));
    mx1 = fmaxf(mx1, fmaxf(sc[s][1], sc[s][3]));
  }
  if (__any_sync(0xffffffffu, (mx0 - st.m0) * scale_log2 > kSlack || (mx1 - st.m1) * scale_log2 > kSlack)) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
      mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
    }
    const float n0 = fmaxf(st.m0, mx0), n1 = fmaxf(st.m1, mx1);
    const float f0 = st.m0 == -INFINITY ? 0.f : ex2((st.m0 - n0) * scale_log2);
    const float f1 = st.m1 == -INFINITY ? 0.f : ex2((st.m1 - n1) * scale_log2);
    st.m0 = n0; st.m1 = n1;
    st.l0 *= f0; st.l1 *= f1;
#pragma unroll
    for (int i = 0; i < Sh::MT; ++i) { st.o[i][0] *= f0; st.o[i][1] *= f1; st.o[i][2] *= f0; st.o[i][3] *= f1; }
  }
  const float r0 = st.m0 == -INFINITY ? 0.f : st.m0 * scale_log2, r1 = st.m1 == -INFINITY ? 0.f : st.m1 * scale_log2;
  uint32_t b0[Sh::SUB], b1[Sh::SUB], c0[Sh::SUB], c1[Sh::SUB];
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    float pr[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) pr[e] = ex2(fmaf(sc[s][e], scale_log2, (e & 1) ? -r1 : -r0));
    st.l0 += pr[0] + pr[2];
    st.l1 += pr[1] + pr[3];
    const uint32_t h0 = pack_bf16(pr[0], pr[1]), h1 = pack_bf16(pr[2], pr[3]);
    const uint32_t e0 = pack_bf16(pr[0] - lo_f(h0), pr[1] - hi_f(h0)), e1 = pack_bf16(pr[2] - lo_f(h1), pr[3] - hi_f(h1));
    b0[s] = transpose8x8(h0); b1[s] = transpose8x8(h1); c0[s] = transpose8x8(e0); c1[s] = transpose8x8(e1);
  }
  if (!kClamp<D> && key0 + Sh::TILE > len) {
#pragma unroll
    for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (key0 + 16 * s + 2 * t + (r & 1) + 8 * (r >> 1) >= len) {
#pragma unroll
          for (int c = 0; c < Sh::VCH; ++c)
#pragma unroll
            for (int w = 0; w < Sh::VW; ++w) x.v[s][r][c][w] = 0;
        }
  }
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
#pragma unroll
    for (int i = 0; i < Sh::MT; ++i) {
      uint32_t a[4];                               // (rows g, g + 8) x (keys 2t, 2t+1 | 2t+8, 2t+9): element 2i and 2i + 1
      if constexpr (D == 8) {
        a[0] = x.v[s][0][0][0] | (x.v[s][1][0][0] << 16);
        a[2] = x.v[s][2][0][0] | (x.v[s][3][0][0] << 16);
        a[1] = a[3] = 0;
      } else {
        const int c = i / Sh::VW, w = i % Sh::VW;
        a[0] = __byte_perm(x.v[s][0][c][w], x.v[s][1][c][w], 0x5410);
        a[1] = __byte_perm(x.v[s][0][c][w], x.v[s][1][c][w], 0x7632);
        a[2] = __byte_perm(x.v[s][2][c][w], x.v[s][3][c][w], 0x5410);
        a[3] = __byte_perm(x.v[s][2][c][w], x.v[s][3][c][w], 0x7632);
      }
      mma16816(st.o[i], a[0], a[1], a[2], a[3], b0[s], b1[s]);
      mma16816(st.o[i], a[0], a[1], a[2], a[3], c0[s], c1[s]);
    }
  }
}

// The sums of the eight thread rows; maxima in log2 units from here on.
template <int D>
__device__ inline void finish(State<D>& st, float scale_log2) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    st.l0 += __shfl_xor_sync(0xffffffffu, st.l0, o);
    st.l1 += __shfl_xor_sync(0xffffffffu, st.l1, o);
  }
  st.m0 *= scale_log2;
  st.m1 *= scale_log2;
}

// Element of the head that accumulator row (i, half) of thread g holds (half: rows g / g + 8 of the MMA tile).
template <int D>
__device__ inline int elem_of(int i, int half, int g) {
  if constexpr (D == 8) return half ? -1 : g;
  const int e = 2 * i + half;
  if constexpr (D == 128) return (e / 8) * 64 + g * 8 + e % 8;
  return g * (D / 8) + e;
}

__device__ inline int clamped_len(const DecParams& p, int n) {
  const int most = p.max_pages << p.page_shift;
  if (n < 0 || n > most) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); n = n < 0 ? 0 : most; }
  return n;
}

__device__ inline long long lse_at(const DecParams& p, long long seq, int head) {
  const long long s = seq / p.n_seqs;
  return (s * p.heads + head) * p.n_seqs + (seq - s * p.n_seqs);
}

// A warp's result for one of the thread's two heads (col 0, 1): the finished row, or a part.
template <int D>
__device__ inline void store_head(const DecParams& p, const State<D>& st, int col, long long seq, int head, int g, int len) {
  using Sh = Shape<D>;
  const float l = col ? st.l1 : st.l0, m = col ? st.m1 : st.m0, inv = len == 0 ? 0.f : 1.f / l;
  __nv_bfloat16* out = p.out + (seq * p.heads + head) * D;
  if constexpr (D == 8) {
    out[g] = __float2bfloat16(st.o[0][col] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < Sh::VCH; ++c) {
      uint32_t w[Sh::VW];
#pragma unroll
      for (int j = 0; j < Sh::VW; ++j) w[j] = pack_bf16(st.o[c * Sh::VW + j][col] * inv, st.o[c * Sh::VW + j][2 + col] * inv);
      __nv_bfloat16* dst = out + c * 64 + g * 2 * Sh::VW;
      if constexpr (Sh::VW == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      else if constexpr (Sh::VW == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
  }
  if (g == 0 && p.lse) p.lse[lse_at(p, seq, head)] = len == 0 ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int D>
__device__ inline void store_part(float* row, const State<D>& st, int col, int head, int g) {
  using Sh = Shape<D>;
  if constexpr (D == 8) {
    row[g] = st.o[0][col];
  } else {
#pragma unroll
    for (int c = 0; c < Sh::VCH; ++c)
#pragma unroll
      for (int j = 0; j < Sh::VW; ++j)
        *reinterpret_cast<float2*>(row + c * 64 + g * 2 * Sh::VW + 2 * j) =
            make_float2(st.o[c * Sh::VW + j][col], st.o[c * Sh::VW + j][2 + col]);
  }
  if (g == 0)
    *reinterpret_cast<float4*>(row + D) = make_float4(col ? st.m1 : st.m0, col ? st.l1 : st.l0, __int_as_float(head), 0.f);
}

// Whole items, one cluster of CTAs per (sequence, KV position, row tile): its warps take the item's tiles in turn; the warps
// of a CTA join in shared memory, the CTAs in the others' shared memory, every one for its share of the result.
template <int D>
__global__ void __launch_bounds__(kDecThreads, D == 128 ? 3 : (D >= 32 ? 4 : 5)) decode_whole_kernel(const DecParams p) {
  using Sh = Shape<D>;
  __shared__ float sm[kDecWarps * kCols * (D + 2)];
  __shared__ float joined[kCols * (D + 2)];
  __shared__ int cols[kDecWarps][kCols];
  __shared__ __align__(16) QueryBuf<D> qbuf[kDecWarps];
  __shared__ int32_t head_cache[kHeadCache], pos_cache[kPosCache];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), stride = ctas * kDecWarps;
  const int first = rank * kDecWarps + warp;       // the warp's first tile
  const int items = p.kv_max * p.row_tiles, number = blockIdx.x / ctas;
  const long long seq = number / items;
  const int rest = number - (int)seq * items, pos = rest / p.row_tiles, rt = rest % p.row_tiles;
  const int s = (int)(seq / p.n_seqs);
  griddep_launch_dependents();
  griddep_wait();
  // one round trip: the length, the first pages, the heads
  const Heads hd = cache_heads(p, head_cache, pos_cache, s, 1);
  int ids = fetch_pages<D>(p, seq, first, stride, lane);
  const int len = clamped_len(p, p.len[seq]), tiles = (len + Sh::TILE - 1) / Sh::TILE;
  ids = check_pages<D>(p, ids, len - 1, first, stride, lane);
  wait_copies();
  const long long k_at = at_k<D>(p, pos, g, t), v_at = at_v<D>(p, pos, g, t);
  constexpr int AHEAD = 32 / Sh::SUB;
  State<D> st;
  reset<D>(st);
  Tile<D> x;
  int key0 = first * Sh::TILE;
  if (first < tiles) {
    load_k<D>(x, p, ids, 0, key0, len - 1, k_at, g);
    load_v<D>(x, p, ids, 0, key0, len - 1, v_at, t);
  }
  __syncthreads();
  find_heads(p, hd, s, pos, rt, lane, cols[warp]);
  if (cols[warp][0] < 0) return;                   // no head reads this position (the same in the whole cluster)
  uint32_t q[Sh::KCH][Sh::KW];
  prefetch_q<D>(qbuf[warp], p, seq, cols[warp][g], lane);
  wait_copies();
  take_q<D>(q, qbuf[warp], lane);
  for (int tile = first, n = 0; tile < tiles; tile += stride, key0 += stride * Sh::TILE) {
    const bool more = tile + stride < tiles;
    const int next0 = key0 + stride * Sh::TILE;
    float sc[Sh::SUB][4];
    tile_scores<D>(sc, x, q);
    if (more) {
      if (++n == AHEAD) {
        ids = check_pages<D>(p, fetch_pages<D>(p, seq, tile + stride, stride, lane), len - 1, tile + stride, stride, lane);
        n = 0;
      }
      load_k<D>(x, p, ids, n, next0, len - 1, k_at, g);
    }
    tile_values<D>(st, sc, x, p.scale_log2, key0, len, g, t);
    if (more) load_v<D>(x, p, ids, n, next0, len - 1, v_at, t);
  }
  finish<D>(st, p.scale_log2);
  float* mine = sm + warp * kCols * (D + 2);       // [head][D + 2]
#pragma unroll
  for (int i = 0; i < Sh::MT; ++i)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = elem_of<D>(i, half, g);
      if (d >= 0) {
        mine[(2 * t) * (D + 2) + d] = st.o[i][2 * half];
        mine[(2 * t + 1) * (D + 2) + d] = st.o[i][2 * half + 1];
      }
    }
  if (g == 0) {
    mine[(2 * t) * (D + 2) + D] = st.m0; mine[(2 * t) * (D + 2) + D + 1] = st.l0;
    mine[(2 * t + 1) * (D + 2) + D] = st.m1; mine[(2 * t + 1) * (D + 2) + D + 1] = st.l1;
  }
  __syncthreads();
  // element (h, d) of the sum of `n` states, state i at at(i)
  auto merge = [&](int n, auto at, int h, int d, float& m, float& l) {
    m = -INFINITY;
    for (int i = 0; i < n; ++i) m = fmaxf(m, at(i)[h * (D + 2) + D]);
    float acc = 0.f;
    l = 0.f;
    for (int i = 0; i < n; ++i) {
      const float* y = at(i) + h * (D + 2);
      const float f = part_weight(y[D], y[D + 1], m);
      acc += f * y[d];
      l += f * y[D + 1];
    }
    return acc;
  };
  auto store = [&](int h, int d, float acc, float m, float l) {
    const int head = cols[warp][h];
    p.out[(seq * p.heads + head) * D + d] = __float2bfloat16(len == 0 ? 0.f : acc / l);
    if (d == 0 && p.lse) p.lse[lse_at(p, seq, head)] = len == 0 ? -INFINITY : (m + log2f(l)) * kLn2;
  };
  auto warps = [&](int i) { return sm + i * kCols * (D + 2); };
  for (int k = threadIdx.x; k < kCols * D; k += kDecThreads) {
    const int h = k / D, d = k % D;
    if (cols[warp][h] < 0) continue;
    float m, l;
    const float acc = merge(kDecWarps, warps, h, d, m, l);
    if (ctas == 1) {
      store(h, d, acc, m, l);
    } else {
      joined[h * (D + 2) + d] = acc;
      if (d == 0) { joined[h * (D + 2) + D] = m; joined[h * (D + 2) + D + 1] = l; }
    }
  }
  if (ctas == 1) return;
  cluster.sync();
  auto others = [&](int i) { return (const float*)cluster.map_shared_rank(joined, i); };
  for (int k = rank * kDecThreads + threadIdx.x; k < kCols * D; k += ctas * kDecThreads) {
    const int h = k / D, d = k % D;
    if (cols[warp][h] < 0) continue;
    float m, l;
    const float acc = merge(ctas, others, h, d, m, l);
    store(h, d, acc, m, l);
  }
  cluster.sync();                                  // the others may still be reading this CTA's sums
}

// The line of work.  A sequence has an item for every KV position that heads read and eight of them (a row tile); an item
// counts kItemCost units for itself (the warp that has its first tile pays them) and one for each of its max(1, tiles of
// its keys) tiles.
template <int D>
__device__ inline int tiles_of(int len) { return max(1, (len + Shape<D>::TILE - 1) / Shape<D>::TILE); }

// The line cut into G pieces whose sizes differ by at most one: piece w begins at w * small + min(w, extra).
struct Cut {
  uint32_t small, extra;
  __device__ uint32_t begin(uint32_t w) const { return w * small + min(w, extra); }
  __device__ uint32_t piece_of(uint32_t u) const {
    const uint32_t big = extra * (small + 1);
    return u < big ? u / (small + 1) : extra + (u - big) / small;
  }
};

// Where a warp stands in the line: an item and the range of its tiles that is the warp's.
struct Segment {
  int seq, s, len, nt;                // sequence, its subnet, its keys, tiles of an item
  int pos, rt;                        // KV position and row tile of the item
  int t0, t1;
};

constexpr int kLenCache = 512;        // sequences whose lengths a CTA keeps in shared memory

// Tiles that go through shared memory in the split kernel.
template <int D>
constexpr bool kStaged = D == 16 || D == 32;
template <int D>
constexpr int kRingBytes = kStaged<D> ? 2 * kDecWarps * (int)sizeof(Stage<D>) : 0;

constexpr int kCountCache = 256;      // KV positions of all subnets whose heads a CTA counts

template <int D>
__global__ void __launch_bounds__(kDecThreads, D == 64 ? 4 : 3) decode_split_kernel(const DecParams p) {
  using Sh = Shape<D>;
  __shared__ int cols[kDecWarps][2][kCols];
  __shared__ __align__(16) QueryBuf<D> qbuf[kDecWarps];
  extern __shared__ __align__(16) unsigned char ring[];       // [kDecWarps][2] stages
  __shared__ int items[TWIST_MAX_SUBNETS], counts[kCountCache];
  __shared__ int32_t lens[kLenCache], head_cache[kHeadCache], pos_cache[kPosCache];
  __shared__ uint32_t warp_sum[kDecWarps];
  __shared__ __align__(16) uint32_t before[kDecThreads];    // cost of the sequences before each thread's
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int N = p.S * p.n_seqs, per = (N + kDecThreads - 1) / kDecThreads;
  for (int i = threadIdx.x; i < kCountCache; i += kDecThreads) counts[i] = 0;
  griddep_launch_dependents();
  griddep_wait();
  // one round trip: lengths, heads, positions
  copy_words(lens, p.len, min(N, kLenCache));
  const Heads hd = cache_heads(p, head_cache, pos_cache, 0, p.S);
  wait_copies();
  __syncthreads();
  // Items of each subnet.  One row tile: the positions up to the last that a group has.  More (sharing by more than eight
  // heads): as many as the position's kept heads fill, counted, so that no keys are read for an empty row tile.
  const bool counted = p.row_tiles > 1 && hd.idx != p.head_idx && p.S * p.kv_max <= kCountCache;
  if (counted) {
    for (int i = threadIdx.x; i < p.S * p.heads; i += kDecThreads) {
      const int s = i / p.heads;
      atomicAdd(&counts[s * p.kv_max + position_of(p, hd, s, i - s * p.heads)], 1);
    }
    __syncthreads();
  }
  auto count_tiles = [&](int s, int pos) { return min((counts[s * p.kv_max + pos] + kCols - 1) / kCols, p.row_tiles); };
  for (int s = warp; s < p.S; s += kDecWarps) {
    int n = 0;
    if (counted) {
      for (int k = lane; k < p.kv_max; k += 32) n += count_tiles(s, k);
      n = __reduce_add_sync(0xffffffffu, n);
    } else {
      if (p.head_idx) {
        for (int k = lane; k < p.n_kv_heads; k += 32) n = max(n, min(hd.pos[s * p.n_kv_heads + k], p.kv_max - 1));
        n = __reduce_max_sync(0xffffffffu, n);
      } else {
        n = p.kv_max - 1;
      }
      n = (n + 1) * p.row_tiles;
    }
    if (lane == 0) items[s] = n;
  }
  __syncthreads();
  // row tiles of a position (0: none; the position is behind the subnet's last one, or no head reads it)
  auto row_tiles = [&](int s, int pos) { return counted ? count_tiles(s, pos) : (pos * p.row_tiles < items[s] ? p.row_tiles : 0); };
  auto len_of = [&](int i) { return clamped_len(p, i < kLenCache ? lens[i] : p.len[i]); };
  uint32_t mine = 0;
  {
    int i = min(N, (int)threadIdx.x * per), s = i / p.n_seqs, b = i - s * p.n_seqs;
    const int last = min(N, i + per);
#pragma unroll 8
    for (; i < last; ++i) {
      mine += (uint32_t)items[s] * (kItemCost + tiles_of<D>(len_of(i)));
      if (++b == p.n_seqs) { b = 0; ++s; }
    }
  }
  uint32_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  uint32_t mine_at = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) mine_at += warp_sum[w];
    total += warp_sum[w];
  }
  before[threadIdx.x] = mine_at;
  const uint32_t G = min((uint32_t)gridDim.x * kDecWarps, max(1u, total / kMinCost));
  const Cut cut{total / G, total % G};
  __syncthreads();
  const uint32_t c = blockIdx.x * kDecWarps + warp;
  if (!p.by_item && lane == 0) p.desc[c] = make_int4(0, 0, 0, 0);
  if (c >= G) return;
  uint32_t left = cut.begin(c + 1) - cut.begin(c);          // units of the warp behind the current segment
  uint32_t item0;                                            // the line's unit at the beginning of the current item
  Segment now;
  auto enter = [&](Segment& x, int seq, int s) {             // the first item of a sequence
    x.seq = seq;
    x.s = s;
    x.len = len_of(seq);
    x.nt = tiles_of<D>(x.len);
  };
  {
    const uint32_t u = cut.begin(c);
    int owner = -1;                                          // the last thread whose sequences begin at or before u
    for (int k = 0; k < kDecThreads; k += 32) owner += __popc(__ballot_sync(0xffffffffu, before[k + lane] <= u));
    uint32_t base = before[owner], cost;
    int seq = owner * per, s = seq / p.n_seqs, b = seq - s * p.n_seqs;
    for (;;) {
      enter(now, seq, s);
      cost = (uint32_t)items[s] * (now.nt + kItemCost);
      if (u < base + cost) break;
      base += cost;
      ++seq;
      if (++b == p.n_seqs) { b = 0; ++s; }
    }
    const uint32_t one = now.nt + kItemCost;
    int item = (int)((u - base) / one);
    const uint32_t x0 = u - base - item * one, x1 = min(one, x0 + left);
    item0 = u - x0;
    if (!counted) {
      now.pos = item / p.row_tiles;
      now.rt = item - now.pos * p.row_tiles;
    } else {
      for (now.pos = 0; item >= count_tiles(s, now.pos); ++now.pos) item -= count_tiles(s, now.pos);
      now.rt = item;
    }
    now.t0 = max(0, (int)x0 - kItemCost);
    now.t1 = max(0, (int)x1 - kItemCost);
    left -= x1 - x0;
  }
  if (now.t1 <= now.t0) return;                           // the item's own cost is all there is: the next warp has its tiles

  constexpr int AHEAD = 32 / Sh::SUB;
  constexpr bool STAGED = kStaged<D>;
  Stage<D>* stages = reinterpret_cast<Stage<D>*>(ring) + 2 * warp;
  Tile<D> x;
  int ids = fetch_pages<D>(p, now.seq, now.t0, 1, lane);
  int next_ids = fetch_pages<D>(p, now.seq, now.t0 + AHEAD, 1, lane);     // unchecked until it becomes `ids`
  int n = 0;                                        // number of the loaded tile in its window of page ids
  int buf = 0, stage = 0;
  find_heads(p, hd, now.s, now.pos, now.rt, lane, cols[warp][0]);
  prefetch_q<D>(qbuf[warp], p, now.seq, cols[warp][0][g], lane);
  ids = check_pages<D>(p, ids, now.len - 1, now.t0, 1, lane);
  if (now.len > 0) {
    if constexpr (STAGED) stage_k<D>(stages[0], p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_k<D>(p, now.pos, g, t), lane);
    else load_k<D>(x, p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_k<D>(p, now.pos, g, t), g);
  }
  commit_copies();                                  // the queries travel with the first keys
  if (now.len > 0) {
    if constexpr (STAGED) stage_v<D>(stages[0], p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_v<D>(p, now.pos, g, t), lane);
    else load_v<D>(x, p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_v<D>(p, now.pos, g, t), t);
  }
  commit_copies();
  for (;;) {
    uint32_t q[Sh::KCH][Sh::KW];
    if constexpr (STAGED) wait_copies_but<1>();
    else wait_copies();
    take_q<D>(q, qbuf[warp], lane);
    const int hq = cols[warp][buf][g];
    // the segment behind this one: its first pages, its heads and their queries on their way before they are needed
    const bool more = left > (uint32_t)kItemCost;
    Segment next = now;
    int head_ids = 0;
    if (more) {
      next.t0 = 0;
      if (++next.rt >= row_tiles(next.s, next.pos)) {
        next.rt = 0;
        do {
          if (++next.pos == p.kv_max) {
            next.pos = 0;
            enter(next, next.seq + 1, (next.seq + 1) / p.n_seqs);
          }
        } while (row_tiles(next.s, next.pos) == 0);
      }
      next.t1 = (int)min((uint32_t)next.nt, left - kItemCost);
      head_ids = fetch_pages<D>(p, next.seq, 0, 1, lane);
      find_heads(p, hd, next.s, next.pos, next.rt, lane, cols[warp][buf ^ 1]);
      prefetch_q<D>(qbuf[warp], p, next.seq, cols[warp][buf ^ 1][g], lane);          // complete with the next tile's keys
    }
    State<D> st;
    reset<D>(st);
    for (int tile = now.t0; tile < now.t1; ++tile) {
      // the tile to load: the item's next one or the next item's first
      const bool inside = tile + 1 < now.t1;
      const int key0 = inside ? (tile + 1) * Sh::TILE : 0, last_key = inside ? now.len - 1 : next.len - 1, of = inside ? now.pos : next.pos;
      const bool load = (inside || more) && last_key >= 0;
      if (inside) {
        if (++n == AHEAD) {
          ids = check_pages<D>(p, next_ids, now.len - 1, tile + 1, 1, lane);
          next_ids = fetch_pages<D>(p, now.seq, tile + 1 + AHEAD, 1, lane);
          n = 0;
        }
      } else {
        ids = check_pages<D>(p, head_ids, more ? next.len - 1 : -1, 0, 1, lane);
        next_ids = fetch_pages<D>(p, next.seq, AHEAD, 1, lane);
        n = 0;
      }
      float sc[Sh::SUB][4];
      if constexpr (STAGED) {
        Stage<D>& to = stages[stage ^ 1];
        if (load) stage_k<D>(to, p, ids, n, key0, last_key, at_k<D>(p, of, g, t), lane);
        commit_copies();
        if (load) stage_v<D>(to, p, ids, n, key0, last_key, at_v<D>(p, of, g, t), lane);
        commit_copies();
        wait_copies_but<3>();
        take_k<D>(x, stages[stage], lane);
        tile_scores<D>(sc, x, q);
        wait_copies_but<2>();
        take_v<D>(x, stages[stage], lane);
        if (now.len > 0) tile_values<D>(st, sc, x, p.scale_log2, tile * Sh::TILE, now.len, g, t);
        stage ^= 1;
      } else {
        tile_scores<D>(sc, x, q);
        if (load) load_k<D>(x, p, ids, n, key0, last_key, at_k<D>(p, of, g, t), g);
        if (now.len > 0) tile_values<D>(st, sc, x, p.scale_log2, tile * Sh::TILE, now.len, g, t);
        if (load) load_v<D>(x, p, ids, n, key0, last_key, at_v<D>(p, of, g, t), t);
      }
    }
    finish<D>(st, p.scale_log2);
    const bool whole = now.t0 == 0 && now.t1 == now.nt;
    const int h0 = __shfl_sync(0xffffffffu, hq, 8 * t), h1 = __shfl_sync(0xffffffffu, hq, 8 * t + 4);
    if (whole) {
      if (h0 >= 0) store_head<D>(p, st, 0, now.seq, h0, g, now.len);
      if (h1 >= 0) store_head<D>(p, st, 1, now.seq, h1, g, now.len);
    } else {
      float* part = p.part + (2ll * c + (now.t0 == 0)) * kCols * kPartRow(D);
      if (h0 >= 0) store_part<D>(part + 2 * t * kPartRow(D), st, 0, h0, g);
      if (h1 >= 0) store_part<D>(part + (2 * t + 1) * kPartRow(D), st, 1, h1, g);
    }
    if (now.t0 == 0 && (p.by_item || !whole)) {
      const int heads = __popc(__ballot_sync(0xffffffffu, hq >= 0 && t == 0));
      if (lane == 0) {
        const int parts = whole ? 0 : (int)(cut.piece_of(item0 + kItemCost + now.nt - 1) - c);    // further parts of the item
        const int all = p.kv_max * p.row_tiles, item = now.pos * p.row_tiles + now.rt;
        int4* desc = p.desc + (p.by_item ? (long long)now.seq * all : (long long)c);
        desc[p.by_item ? item : 0] = make_int4(now.seq, heads, parts, (int)c);
        if (p.by_item) {                            // the neighbours in the table that are no items
          auto is_item = [&](int k) { return k % p.row_tiles < row_tiles(now.s, k / p.row_tiles); };
          for (int k = item + 1; k < all && !is_item(k); ++k) desc[k] = make_int4(0, 0, 0, 0);
          for (int k = item - 1; k >= 0 && !is_item(k); --k) desc[k] = make_int4(0, 0, 0, 0);
        }
      }
    }
    if (!more) break;
    item0 += now.nt + kItemCost;
    left -= next.t1 + kItemCost;
    now = next;
    buf ^= 1;
  }
}

// Joins the parts of one cut item: its beginning is slot 2c + 1 (c: the warp that has it), the others are 2(c+1), 2(c+2), ...
// A CTA takes blockDim / groups elements of the item's heads; `groups` threads share the parts of each, every one merging
// its own in order, eight at a time; the groups are merged in order through shared memory.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(const DecParams p, int groups) {
  __shared__ float3 sums[kJoinThreads];             // (maximum, sum, element)
  griddep_wait();
  const int4 item = p.desc[blockIdx.x];
  const int heads = item.y, parts = item.z + 1, c = item.w;
  const int elems = blockDim.x / groups, k = blockIdx.y * elems + threadIdx.x % elems, grp = threadIdx.x / elems;
  if (parts <= 1 || (int)(blockIdx.y * elems) >= heads * D) return;
  const int h = k / D, d = k % D;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  if (k < heads * D) {
    for (int e0 = grp; e0 < parts; e0 += 8 * groups) {
      float2 ml[8];
      float y[8];
      float top = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = e0 + j * groups;
        ml[j] = make_float2(-INFINITY, 0.f);
        y[j] = 0.f;
        if (e < parts) {
          const float* row = p.part + ((long long)(e ? 2 * (c + e) : 2 * c + 1) * kCols + h) * kPartRow(D);
          ml[j] = *reinterpret_cast<const float2*>(row + D);
          y[j] = row[d];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
      const float f = part_weight(m, l, top);
      acc *= f;
      l *= f;
      m = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = part_weight(ml[j].x, ml[j].y, top);
        acc += w * y[j];
        l += w * ml[j].y;
      }
    }
  }
  if (groups > 1) {
    sums[threadIdx.x] = make_float3(m, l, acc);
    __syncthreads();
    if (grp > 0) return;
    for (int e = 1; e < groups; ++e) m = fmaxf(m, sums[threadIdx.x + e * elems].x);
    const float f = part_weight(sums[threadIdx.x].x, l, m);
    l *= f;
    acc *= f;
    for (int e = 1; e < groups; ++e) {
      const float3 y = sums[threadIdx.x + e * elems];
      const float w = part_weight(y.x, y.y, m);
      l += w * y.y;
      acc += w * y.z;
    }
  }
  if (k >= heads * D) return;
  const int head = __float_as_int(p.part[((2ll * c + 1) * kCols + h) * kPartRow(D) + D + 2]);
  p.out[((long long)item.x * p.heads + head) * D + d] = __float2bfloat16(acc / l);
  if (d == 0 && p.lse) p.lse[lse_at(p, item.x, head)] = (m + log2f(l)) * kLn2;
}

// Whether the output, dense, lies over one of the rows of queries (which CTAs still read when others write).
bool over_queries(const DecParams& p, int d) {
  const long long rows = (long long)p.S * p.n_seqs, width = 2ll * p.heads * d, stride = 2 * p.q_stride;
  const long long at = (long long)(reinterpret_cast<uintptr_t>(p.out) - reinterpret_cast<uintptr_t>(p.q));     // from the first query
  const long long row = at < width ? 0 : (at - width) / stride + 1;                                            // the first that ends behind it
  return row < rows && row * stride < at + rows * width;
}

size_t max_warps() { return (size_t)sm_count() * kMaxCtasPerSm * kDecWarps; }
size_t desc_bytes() { return (max_warps() * sizeof(int4) + 255) / 256 * 256; }

template <int D>
int run(DecParams& p, long long max_len, cudaStream_t st) {
  const long long items = (long long)p.S * p.n_seqs * p.kv_max * p.row_tiles;
  // the line is counted in 32 bits
  const long long longest = (((long long)p.max_pages << p.page_shift) + Shape<D>::TILE - 1) / Shape<D>::TILE + 1 + kItemCost;
  if (items > 0x7fffffffll / longest) return TWIST_ERR_UNSUPPORTED;
  if (over_queries(p, D)) return TWIST_ERR_SHAPE;
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  static int resident[64] = {0}, join_resident[64];
  const int slot = device_slot();
  if (resident[slot] == 0) {
    int n = 0;
    TWIST_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, decode_join_kernel<D>, kJoinThreads, 0));
    join_resident[slot] = n < 1 ? 1 : n;
    TWIST_CUDA_TRY(cudaFuncSetAttribute(decode_split_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes<D>));
    TWIST_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, decode_split_kernel<D>, kDecThreads, kRingBytes<D>));
    resident[slot] = n < 1 ? 1 : (n > kMaxCtasPerSm ? kMaxCtasPerSm : n);
  }
  const long long grid = (long long)sm_count() * resident[slot];
  // One cluster per item where that needs few turns: two tiles a warp are taken by a single CTA, more by as many CTAs as
  // leave a warp one, if all of them run at once.  Measured (d = 64, one sequence of 8 heads, 1024 keys): 5.0 us against 9.2
  // through the line; 512 items of 512 keys, all at once: 15 against 19.  The line is ahead where a warp would take more
  // than kShortTiles tiles, where the items fill the GPU kShortWork tiles a warp deep (256 ragged items of up to 2048
  // keys: 21 us against 27 to 34), and earlier where they do not run at once (512 items of 256 keys, d = 128: 18.2
  // against 19.6).
  const long long tiles = (max_len + Shape<D>::TILE - 1) / Shape<D>::TILE;
  int cluster = 1;
  if (tiles > 2 * kDecWarps)
    while (cluster < kMaxCluster && 2 * cluster * items <= grid && tiles > kDecWarps * cluster) cluster *= 2;
  if (items <= 2 * grid && tiles <= kShortTiles * kDecWarps * cluster &&
      tiles * items <= (items <= grid ? kShortWork : kShortWaves) * grid * kDecWarps) {
    TWIST_CUDA_TRY(launch_overlapped(decode_whole_kernel<D>, dim3((unsigned)(items * cluster)), dim3(kDecThreads), 0, st, cluster, p));
    return TWIST_OK;
  }
  p.by_item = items <= grid * kDecWarps;
  TWIST_CUDA_TRY(launch_overlapped(decode_split_kernel<D>, dim3((unsigned)grid), dim3(kDecThreads), kRingBytes<D>, st, 1, p));
  // An item of an even batch is cut into about warps / items parts: the fewer items, the more threads share the parts of
  // one, down to eight parts each, as long as all threads of the join run at once.  The whole call, with twice the threads
  // against without: where they fit, four heads on a position, 16 items, d = 16 and 32: 15.9 and 16.5 us against 17.5; one
  // head a position, 64 to 256 items, d = 64: 49.0 against 49.6.  Where they do not (262144 for 151552), eight heads on a
  // position, d = 64, 32 to 256 items: 22.3 to 22.9 against 21.4 to 22.1; four subnets, 256 ragged items: 20.9 against 19.9.
  const int elems = (kCols < p.per_group ? kCols : p.per_group) * D;                   // of the heads that share a position
  const long long at_once = (long long)sm_count() * join_resident[slot] * kJoinThreads;
  int groups = 1;
  while (groups < kJoinThreads / 32 && 8ll * groups * items < grid * kDecWarps && 2ll * groups * items * elems <= at_once) groups *= 2;
  const int block = elems * groups < 32 ? 32 : (elems * groups > kJoinThreads ? kJoinThreads : elems * groups);
  const dim3 join_grid((unsigned)(p.by_item ? items : grid * kDecWarps), (unsigned)((elems * groups + block - 1) / block));
  TWIST_CUDA_TRY(launch_overlapped(decode_join_kernel<D>, join_grid, dim3(block), 0, st, 1, p, groups));
  return TWIST_OK;
}

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" size_t twist_attn_decode_workspace_bytes(int32_t d_head) {
  if (d_head <= 0 || d_head > 128) return 0;
  return desc_bytes() + max_warps() * 2 * kCols * kPartRow(d_head) * sizeof(float);
}

extern "C" int32_t twist_attn_decode(const twist_attn_decode_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->head_keep <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 ||
      a->max_pages <= 0 || a->page_size <= 0 || a->max_len < 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if (dh != 8 && dh != 16 && dh != 32 && dh != 64 && dh != 128) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets > TWIST_MAX_SUBNETS || a->n_heads > 1024 || a->head_keep > 1024) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->n_subnets * a->n_seqs > 65535) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll - 1024) return TWIST_ERR_UNSUPPORTED;   // positions are 32-bit
  if (a->page_stride % 8 != 0 || a->page_stride < (long long)a->kv_max * a->page_size * dh) return TWIST_ERR_SHAPE;
  if (a->q_stride % 8 != 0 || a->q_stride < (long long)a->head_keep * dh) return TWIST_ERR_SHAPE;
  if (a->head_idx) {
    if (!a->kv_pos || a->n_heads <= 0 || a->n_kv_heads <= 0 || a->n_heads % a->n_kv_heads != 0) return TWIST_ERR_SHAPE;
  } else if (a->kv_max != a->head_keep) {
    return TWIST_ERR_SHAPE;
  }
  if (!a->q || !a->k_cache || !a->v_cache || !a->page_table || !a->kv_len || !a->out) return TWIST_ERR_NULL;
  if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->out) || !aligned16(a->ws)) return TWIST_ERR_SHAPE;
  if (!a->ws || a->ws_bytes < twist_attn_decode_workspace_bytes(dh)) return TWIST_ERR_WORKSPACE;
  DecParams p;
  memset(&p, 0, sizeof(p));
  p.q = static_cast<const __nv_bfloat16*>(a->q);
  p.k = static_cast<const __nv_bfloat16*>(a->k_cache);
  p.v = static_cast<const __nv_bfloat16*>(a->v_cache);
  p.table = a->page_table; p.len = a->kv_len; p.head_idx = a->head_idx; p.kv_pos = a->kv_pos;
  p.out = static_cast<__nv_bfloat16*>(a->out);
  p.lse = a->lse;
  p.desc = static_cast<int4*>(a->ws);
  p.part = reinterpret_cast<float*>(static_cast<char*>(a->ws) + desc_bytes());
  p.page_stride = a->page_stride; p.q_stride = a->q_stride;
  p.S = a->n_subnets; p.n_seqs = a->n_seqs; p.heads = a->head_keep; p.kv_max = a->kv_max;
  p.per_group = a->head_idx ? a->n_heads / a->n_kv_heads : 1;
  p.n_kv_heads = a->head_idx ? a->n_kv_heads : a->kv_max;
  p.row_tiles = (p.per_group + kCols - 1) / kCols;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages;
  p.scale_log2 = kLog2e / sqrtf((float)dh);
  const long long table_len = (long long)a->max_pages * a->page_size;
  const long long max_len = a->max_len > 0 && a->max_len < table_len ? a->max_len : table_len;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dh) {
    case 8: return run<8>(p, max_len, st);
    case 16: return run<16>(p, max_len, st);
    case 32: return run<32>(p, max_len, st);
    case 64: return run<64>(p, max_len, st);
    default: return run<128>(p, max_len, st);
  }
}
