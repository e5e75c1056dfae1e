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
// a tile (8 KB) in flight all the time.  (tcgen05 would need 128 rows of queries to fill its smallest tile.)
//
// Softmax in fp32 with a running reference maximum per head that moves only when a score exceeds it by more than 2^8 (one
// vote per tile instead of a reduction).  The probabilities enter the second product as the sum of two bf16 numbers
// (value and remainder: 16 bits), so that rounding them costs nothing against the one rounding of the result.
//
// Splitting.  The work of a call is a line of tiles: sequence after sequence, KV position after KV position.  CTA c of G
// takes the c-th G-th of the line, whatever the lengths are: a ragged batch is balanced on the device.  A CTA writes the
// items it has whole; of an item that a CTA boundary cuts, every CTA writes its unnormalised part (fp32 sums, maximum,
// sum) to the workspace, and a second small launch joins the parts in the order of the CTAs.
#include "common.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kCols = 8;                   // heads per pass over the keys (columns of the MMA tile)
constexpr int kMaxCtasPerSm = 4;
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
  float* part;                // [2 G][kCols][D + 2]: sums, maximum (log2), sum of probabilities
  int4* desc;                 // [G] the item that starts in CTA c and ends behind it: (sequence, KV position, row tile, parts)
  long long page_stride, q_stride;
  int S, n_seqs, heads, kv_max, per_group, n_kv_heads, row_tiles;
  int page_shift, n_pages, max_pages;
  float scale_log2;
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
__device__ inline float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ inline float hi_f(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// `W` 32-bit words (W = 4, 2, 1) of a row that is read once.
template <int W>
__device__ inline void load_words(uint32_t (&r)[W], const __nv_bfloat16* p) {
  if constexpr (W == 4)
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
  else if constexpr (W == 2)
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
  else
    asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(r[0]) : "l"(p));
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
  static constexpr int SUB = D == 128 ? 1 : (D == 64 ? 2 : 4);
  static constexpr int TILE = 16 * SUB;
};

template <int D>
struct Tile {
  using Sh = Shape<D>;
  uint32_t k[Sh::SUB][2][Sh::KCH][Sh::KW];
  uint32_t v[Sh::SUB][4][Sh::VCH][Sh::VW];
};

// A page of the sequence; a bad entry is replaced by page 0 and reported.
__device__ inline long long page_of(const DecParams& p, const int32_t* table, int key) {
  int id = table[key >> p.page_shift];
  if ((unsigned)id >= (unsigned)p.n_pages) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); id = 0; }
  return id * p.page_stride;
}

// Keys behind the end are read as zeros: whatever lies in the unused part of a page must not reach the products.
template <int D>
__device__ inline void load_k(Tile<D>& x, const DecParams& p, const int32_t* table, int key0, int len, long long pos_off, int g, int t) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int kb = key0 + 16 * s;
    const __nv_bfloat16* base = kb < len ? p.k + page_of(p, table, kb) + pos_off : p.k;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int key = kb + g + 8 * r;
      const __nv_bfloat16* row = base + (long long)(key & ((1 << p.page_shift) - 1)) * D + t * 2 * Sh::KW;
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c) {
        if (key < len) {
          load_words<Sh::KW>(x.k[s][r][c], row + c * 8 * Sh::KW);
        } else {
#pragma unroll
          for (int w = 0; w < Sh::KW; ++w) x.k[s][r][c][w] = 0;
        }
      }
    }
  }
}

template <int D>
__device__ inline void load_v(Tile<D>& x, const DecParams& p, const int32_t* table, int key0, int len, long long pos_off, int g, int t) {
  using Sh = Shape<D>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    const int kb = key0 + 16 * s;
    const __nv_bfloat16* base = kb < len ? p.v + page_of(p, table, kb) + pos_off : p.v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = kb + 2 * t + (r & 1) + 8 * (r >> 1);
      const __nv_bfloat16* row = base + (long long)(key & ((1 << p.page_shift) - 1)) * D;
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c) {
        if (key < len) {
          if constexpr (D == 8) x.v[s][r][c][0] = *reinterpret_cast<const unsigned short*>(row + g);
          else load_words<Sh::VW>(x.v[s][r][c], row + c * 64 + g * 2 * Sh::VW);
        } else {
#pragma unroll
          for (int w = 0; w < Sh::VW; ++w) x.v[s][r][c][w] = 0;
        }
      }
    }
  }
}

// Running state of a warp: up to eight heads (columns); the thread's columns are 2t and 2t + 1.
template <int D>
struct State {
  float o[Shape<D>::MT][4];
  float m0, m1, l0, l1;
};

// KV position among the subnet's kept groups that kept head hq reads, checked.
__device__ inline int position_of(const DecParams& p, int s, int hq) {
  if (!p.head_idx) return hq;
  const int h = p.head_idx[(long long)s * p.heads + hq];
  int g = h < 0 ? -1 : h / p.per_group;
  if ((unsigned)g >= (unsigned)p.n_kv_heads) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); g = 0; }
  int pos = p.kv_pos[(long long)s * p.n_kv_heads + g];
  if ((unsigned)pos >= (unsigned)p.kv_max) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); pos = 0; }
  return pos;
}

// The kept heads number 8 rt .. 8 rt + 7 among those that read KV position `pos`, into cols[0..7] (-1: none).  One warp.
__device__ inline void find_heads(const DecParams& p, int s, int pos, int rt, int lane, int* cols) {
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
    const bool mine = hq < p.heads && position_of(p, s, hq) == pos;
    const unsigned vote = __ballot_sync(0xffffffffu, mine);
    const int rank = seen + __popc(vote & ((1u << lane) - 1)) - kCols * rt;
    if (mine && rank >= 0 && rank < kCols) cols[rank] = hq;
    seen += __popc(vote);
  }
  if (lane == 0 && rt == 0 && seen > kCols * p.row_tiles) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
  __syncwarp();
}

// All tiles t0 + warp, t0 + warp + kDecWarps, ... < t1 of one item.
template <int D>
__device__ inline void run_tiles(State<D>& st, const DecParams& p, const int32_t* table, int len, long long pos_off,
                                 const uint32_t (&q)[Shape<D>::KCH][Shape<D>::KW], int t0, int t1, int warp, int lane) {
  using Sh = Shape<D>;
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < Sh::MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[i][e] = 0.f;
  st.m0 = st.m1 = -INFINITY;
  st.l0 = st.l1 = 0.f;
  int tile = t0 + warp;
  if (tile >= t1) return;
  Tile<D> x;
  load_k<D>(x, p, table, tile * Sh::TILE, len, pos_off, g, t);
  load_v<D>(x, p, table, tile * Sh::TILE, len, pos_off, g, t);
  for (; tile < t1; tile += kDecWarps) {
    const int key0 = tile * Sh::TILE;
    const bool more = tile + kDecWarps < t1;
    float sc[Sh::SUB][4];
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
    if (more) load_k<D>(x, p, table, key0 + kDecWarps * Sh::TILE, len, pos_off, g, t);
    // scores in log2 units; keys behind the end count for nothing
    float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
    for (int s = 0; s < Sh::SUB; ++s) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool live = key0 + 16 * s + g + 8 * (e >> 1) < len;
        sc[s][e] = live ? sc[s][e] * p.scale_log2 : -INFINITY;
      }
      mx0 = fmaxf(mx0, fmaxf(sc[s][0], sc[s][2]));
      mx1 = fmaxf(mx1, fmaxf(sc[s][1], sc[s][3]));
    }
    if (__any_sync(0xffffffffu, mx0 > st.m0 + kSlack || mx1 > st.m1 + kSlack)) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
      }
      const float n0 = fmaxf(st.m0, mx0), n1 = fmaxf(st.m1, mx1);
      const float f0 = st.m0 == -INFINITY ? 0.f : ex2(st.m0 - n0), f1 = st.m1 == -INFINITY ? 0.f : ex2(st.m1 - n1);
      st.m0 = n0; st.m1 = n1;
      st.l0 *= f0; st.l1 *= f1;
#pragma unroll
      for (int i = 0; i < Sh::MT; ++i) { st.o[i][0] *= f0; st.o[i][1] *= f1; st.o[i][2] *= f0; st.o[i][3] *= f1; }
    }
    const float r0 = st.m0 == -INFINITY ? 0.f : st.m0, r1 = st.m1 == -INFINITY ? 0.f : st.m1;
#pragma unroll
    for (int s = 0; s < Sh::SUB; ++s) {
      float pr[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) pr[e] = ex2(sc[s][e] - ((e & 1) ? r1 : r0));
      st.l0 += pr[0] + pr[2];
      st.l1 += pr[1] + pr[3];
      const uint32_t h0 = pack_bf16(pr[0], pr[1]), h1 = pack_bf16(pr[2], pr[3]);
      const uint32_t e0 = pack_bf16(pr[0] - lo_f(h0), pr[1] - hi_f(h0)), e1 = pack_bf16(pr[2] - lo_f(h1), pr[3] - hi_f(h1));
      const uint32_t b0 = transpose8x8(h0), b1 = transpose8x8(h1), c0 = transpose8x8(e0), c1 = transpose8x8(e1);
#pragma unroll
      for (int i = 0; i < Sh::MT; ++i) {
        uint32_t a[4];                             // (rows g, g + 8) x (keys 2t, 2t+1 | 2t+8, 2t+9): element 2i and 2i + 1
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
        mma16816(st.o[i], a[0], a[1], a[2], a[3], b0, b1);
        mma16816(st.o[i], a[0], a[1], a[2], a[3], c0, c1);
      }
    }
    if (more) load_v<D>(x, p, table, key0 + kDecWarps * Sh::TILE, len, pos_off, g, t);
  }
}

// Element of the head that accumulator row (i, half) of thread g holds (half: rows g / g + 8 of the MMA tile).
template <int D>
__device__ inline int elem_of(int i, int half, int g) {
  if constexpr (D == 8) return half ? -1 : g;
  const int e = 2 * i + half;
  if constexpr (D == 128) return (e / 8) * 64 + g * 8 + e % 8;
  return g * (D / 8) + e;
}

__device__ inline int clamped_len(const DecParams& p, long long seq) {
  const int most = p.max_pages << p.page_shift;
  int n = p.len[seq];
  if (n < 0 || n > most) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); n = n < 0 ? 0 : most; }
  return n;
}

// One segment (tiles t0 .. t1 of the item (seq, pos, row tile)); `slot` >= 0: a part, written to the workspace.
template <int D>
__device__ inline void run_segment(const DecParams& p, float* sm, int (*cols)[kCols], long long seq, int pos, int rt, int len,
                                   int t0, int t1, int slot) {
  using Sh = Shape<D>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int s = (int)(seq / p.n_seqs);
  const long long pos_off = ((long long)pos << p.page_shift) * D;
  const int32_t* table = p.table + seq * p.max_pages;
  find_heads(p, s, pos, rt, lane, cols[warp]);
  if (cols[warp][0] < 0) return;                    // no head reads this position: nothing to do (the same in every warp)
  State<D> st;
  uint32_t q[Sh::KCH][Sh::KW];
  const int hq = cols[warp][g];
  const __nv_bfloat16* qrow = p.q + seq * p.q_stride + (long long)(hq < 0 ? 0 : hq) * D + t * 2 * Sh::KW;
#pragma unroll
  for (int c = 0; c < Sh::KCH; ++c) {
    if (hq >= 0) load_words<Sh::KW>(q[c], qrow + c * 8 * Sh::KW);
    else
#pragma unroll
      for (int w = 0; w < Sh::KW; ++w) q[c][w] = 0;
  }
  run_tiles<D>(st, p, table, len, pos_off, q, t0, t1, warp, lane);
  // the warps' states side by side in shared memory: [warp][head][D + 2]
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    st.l0 += __shfl_xor_sync(0xffffffffu, st.l0, o);
    st.l1 += __shfl_xor_sync(0xffffffffu, st.l1, o);
  }
  float* mine = sm + warp * kCols * (D + 2);
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
  for (int k = threadIdx.x; k < kCols * D; k += kDecThreads) {
    const int h = k / D, d = k % D, head = cols[warp][h];
    if (head < 0) continue;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) m = fmaxf(m, sm[(w * kCols + h) * (D + 2) + D]);
    float acc = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      const float* x = sm + (w * kCols + h) * (D + 2);
      const float f = x[D] == -INFINITY ? (x[D + 1] == 0.f ? 0.f : 1.f) : ex2(x[D] - m);
      acc += f * x[d];
      l += f * x[D + 1];
    }
    if (slot >= 0) {
      float* dst = p.part + ((long long)slot * kCols + h) * (D + 2);
      dst[d] = acc;
      if (d == 0) { dst[D] = m; dst[D + 1] = l; }
    } else {
      p.out[(seq * p.heads + head) * D + d] = __float2bfloat16(len == 0 ? 0.f : acc / l);
      if (d == 0 && p.lse)
        p.lse[((long long)s * p.heads + head) * p.n_seqs + seq % p.n_seqs] = len == 0 ? -INFINITY : (m + log2f(l)) * kLn2;
    }
  }
  __syncthreads();
}

// Whole items only: one CTA per (sequence, KV position, row tile).
template <int D>
__global__ void __launch_bounds__(kDecThreads) decode_whole_kernel(const DecParams p) {
  __shared__ float sm[kDecWarps * kCols * (D + 2)];
  __shared__ int cols[kDecWarps][kCols];
  const int items = p.kv_max * p.row_tiles;
  const long long seq = blockIdx.x / items;
  const int rest = (int)(blockIdx.x - seq * items);
  const int len = clamped_len(p, seq);
  run_segment<D>(p, sm, cols, seq, rest / p.row_tiles, rest % p.row_tiles, len, 0, (len + Shape<D>::TILE - 1) / Shape<D>::TILE, -1);
}

// The line of tiles.  Units of sequence i: held(s) * row_tiles * max(1, tiles of its keys).
template <int D>
__device__ inline int tiles_of(int len) { return max(1, (len + Shape<D>::TILE - 1) / Shape<D>::TILE); }

template <int D>
__global__ void __launch_bounds__(kDecThreads) decode_split_kernel(const DecParams p) {
  __shared__ float sm[kDecWarps * kCols * (D + 2)];
  __shared__ int cols[kDecWarps][kCols];
  __shared__ int held[TWIST_MAX_SUBNETS];
  __shared__ long long warp_sum[kDecWarps];
  __shared__ long long start_base;
  __shared__ long long start_seq;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // KV positions of each subnet that some head reads: 1 + the largest entry of kv_pos
  for (int s = warp; s < p.S; s += kDecWarps) {
    int top = 0;
    if (p.head_idx) {
      for (int k = lane; k < p.n_kv_heads; k += 32) top = max(top, min(p.kv_pos[s * p.n_kv_heads + k], p.kv_max - 1));
      for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    } else {
      top = p.kv_max - 1;
    }
    if (lane == 0) held[s] = top + 1;
  }
  __syncthreads();
  const int N = p.S * p.n_seqs, per = (N + kDecThreads - 1) / kDecThreads;
  const int first = min(N, (int)threadIdx.x * per), last = min(N, first + per);
  long long mine = 0;
  for (int i = first; i < last; ++i) mine += (long long)held[i / p.n_seqs] * p.row_tiles * tiles_of<D>(clamped_len(p, i));
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  long long before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  // as many CTAs as get a tile for each of their warps
  const long long G = min((long long)gridDim.x, (total + kDecWarps - 1) / kDecWarps);
  const int c = blockIdx.x;
  if (threadIdx.x == 0) p.desc[c] = make_int4(0, 0, 0, 0);
  if (c >= G) return;
  const long long u0 = total * c / G, u1 = total * (c + 1) / G;
  if (u0 >= before && u0 < before + mine) {
    long long base = before;
    int i = first;
    for (;; ++i) {
      const long long n = (long long)held[i / p.n_seqs] * p.row_tiles * tiles_of<D>(clamped_len(p, i));
      if (u0 < base + n) break;
      base += n;
    }
    start_seq = i;
    start_base = base;
  }
  __syncthreads();
  long long seq = start_seq, base = start_base, u = u0;
  while (u < u1) {
    const int len = clamped_len(p, seq), nt = tiles_of<D>(len);
    const int s = (int)(seq / p.n_seqs);
    const long long units = (long long)held[s] * p.row_tiles * nt;
    while (u < u1 && u < base + units) {
      const int item = (int)((u - base) / nt);
      const long long item0 = base + (long long)item * nt;
      const int t0 = (int)(u - item0), t1 = (int)min((long long)nt, u1 - item0);
      int slot = -1;
      if (t0 > 0) slot = 2 * c;
      else if (t1 < nt) {
        slot = 2 * c + 1;
        // the CTA that holds the item's last tile: the largest e with total * e / G <= that tile
        const long long end = item0 + nt - 1;
        long long e = end * G / total;
        while (total * (e + 1) / G <= end) ++e;
        while (total * e / G > end) --e;
        if (threadIdx.x == 0) p.desc[c] = make_int4((int)seq, item / p.row_tiles, item % p.row_tiles, (int)(e - c));
      }
      run_segment<D>(p, sm, cols, seq, item / p.row_tiles, item % p.row_tiles, len, t0, t1, slot);
      u = item0 + t1;
    }
    base += units;
    ++seq;
  }
}

// Joins the parts of one cut item: CTA c's own (the item's beginning, slot 2c + 1) and slots 2(c+1), 2(c+2), ...
template <int D>
__global__ void __launch_bounds__(kDecThreads) decode_join_kernel(const DecParams p) {
  __shared__ int cols[kCols];
  griddep_wait();
  const int c = blockIdx.x;
  const int4 item = p.desc[c];
  if (item.w <= 0) return;
  const long long seq = item.x;
  const int s = (int)(seq / p.n_seqs);
  if (threadIdx.x < 32) find_heads(p, s, item.y, item.z, threadIdx.x, cols);
  __syncthreads();
  for (int k = threadIdx.x; k < kCols * D; k += kDecThreads) {
    const int h = k / D, d = k % D, head = cols[h];
    if (head < 0) continue;
    float m = -INFINITY;
    for (int e = 0; e <= item.w; ++e)
      m = fmaxf(m, p.part[((long long)(e ? 2 * (c + e) : 2 * c + 1) * kCols + h) * (D + 2) + D]);
    float acc = 0.f, l = 0.f;
    for (int e = 0; e <= item.w; ++e) {
      const float* x = p.part + ((long long)(e ? 2 * (c + e) : 2 * c + 1) * kCols + h) * (D + 2);
      const float f = x[D] == -INFINITY ? (x[D + 1] == 0.f ? 0.f : 1.f) : ex2(x[D] - m);
      acc += f * x[d];
      l += f * x[D + 1];
    }
    p.out[(seq * p.heads + head) * D + d] = __float2bfloat16(acc / l);
    if (d == 0 && p.lse) p.lse[((long long)s * p.heads + head) * p.n_seqs + seq % p.n_seqs] = (m + log2f(l)) * kLn2;
  }
}

size_t desc_bytes() { return ((size_t)sm_count() * kMaxCtasPerSm * sizeof(int4) + 255) / 256 * 256; }

template <int D>
int run(DecParams& p, long long max_len, cudaStream_t st) {
  const long long items = (long long)p.S * p.n_seqs * p.kv_max * p.row_tiles;
  if (max_len <= 512 && items <= 0x7fffffffll) {
    decode_whole_kernel<D><<<(unsigned)items, kDecThreads, 0, st>>>(p);
    TWIST_LAUNCH_CHECK();
    return TWIST_OK;
  }
  static int ctas[64] = {0};
  const int slot = device_slot();
  if (ctas[slot] == 0) {
    int n = 0;
    TWIST_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, decode_split_kernel<D>, kDecThreads, 0));
    ctas[slot] = n < 1 ? 1 : (n > kMaxCtasPerSm ? kMaxCtasPerSm : n);
  }
  const unsigned grid = (unsigned)(sm_count() * ctas[slot]);
  decode_split_kernel<D><<<grid, kDecThreads, 0, st>>>(p);
  TWIST_LAUNCH_CHECK();
  decode_join_kernel<D><<<grid, kDecThreads, 0, st>>>(p);
  TWIST_LAUNCH_CHECK();
  return TWIST_OK;
}

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" size_t twist_attn_decode_workspace_bytes(int32_t d_head) {
  if (d_head <= 0 || d_head > 128) return 0;
  return desc_bytes() + (size_t)sm_count() * kMaxCtasPerSm * 2 * kCols * ((size_t)d_head + 2) * sizeof(float);
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
  if ((long long)a->n_subnets * a->n_seqs > (1 << 24)) return TWIST_ERR_UNSUPPORTED;
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
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
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
