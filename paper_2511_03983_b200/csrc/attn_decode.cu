// twist_attn_decode and twist_attn_decode_q8: attention of one new token per sequence over a paged key-value cache,
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
// 8 bits (B = 1): the same, the numbers widened to fp16 between load and product (exact), K's scales multiplied into the scores and
// V's into the probabilities.  A byte then costs twice the instructions, and a tile in registers is too little in flight: tiles
// come through rings in shared memory, filled by bulk copies (see Ring).
//
// Calls whose length and number of items leave little to balance take a shorter way instead: one cluster of 1 to 8 CTAs
// per item, whose warps take the item's tiles in turn and join through (distributed) shared memory: one launch, no
// workspace.
#include <cooperative_groups.h>

#include "decode_tiles.cuh"

namespace twist {
namespace {

constexpr int kMaxCtasPerSm = 4;
// What changing to the next item costs a warp, in tiles.  8 bits, 1 / 2 / 3 / 5: 952 ragged sequences of up to 274 keys on 4
// positions of d = 128 58.0 / 51.9 / 49.7 / 50.0 us, eight subnets of long ones 200 / 200 / 191 / 189.
template <int B>
constexpr int kItemCost = B == 1 ? 3 : 1;
constexpr int kMinCost = 2;                // least work of a warp, in tiles
constexpr int kJoinThreads = 512;
// The short way, one cluster per item (see run).
constexpr int kMaxCluster = 8, kShortTiles = 8, kShortWork = 8, kShortWaves = 4;
constexpr float kSlack = 8.0f;             // log2 headroom of the lazily moved reference maximum

// Row of a part: d sums, then maximum (log2), sum of probabilities, head, padding.
__host__ __device__ constexpr int kPartRow(int d) { return d + 4; }
// Weight of a part with maximum x (log2) and sum l against the maximum m of all parts.  A part without a reference maximum
// has no finite score: it counts for nothing, unless its sum is NaN.
__device__ inline float part_weight(float x, float l, float m) { return x == -INFINITY ? (l == 0.f ? 0.f : 1.f) : ex2(x - m); }

// Running state of a warp: up to eight heads (columns); the thread's columns are 2t and 2t + 1.
template <int D, int B>
struct State {
  float o[Shape<D, B>::MT][4];
  float m0, m1, l0, l1;
  float c0, c1, e0, e1;       // 8 bits: the sums o are c times what they stand for, c = 2^e
};
constexpr float kMostUp = 124.f;           // e at most: a probability of 1 beside the smallest scale of an append becomes 2^14

template <int D, int B>
__device__ inline void reset(State<D, B>& st) {
#pragma unroll
  for (int i = 0; i < Shape<D, B>::MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[i][e] = 0.f;
  st.m0 = st.m1 = -INFINITY;
  st.l0 = st.l1 = 0.f;
  st.e0 = st.e1 = kMostUp;
  st.c0 = st.c1 = 0x1p124f;
}

// Values of keys behind the end of `len` keys, cleared (see kClamp).
template <int D, int B>
__device__ inline void clear_behind(Tile<D, B>& x, int key0, int len, int t) {
  using Sh = Shape<D, B>;
  if (!kClamp<D, B> && key0 + Sh::TILE > len) {
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
}

// A step's probabilities from the scores against the reference r0, r1.
__device__ inline void probabilities(float (&pr)[4], const float (&sc)[4], float scale_log2, float r0, float r1) {
#pragma unroll
  for (int e = 0; e < 4; ++e) pr[e] = ex2(fmaf(sc[e], scale_log2, (e & 1) ? -r1 : -r0));
}

// 8 bits: brings the sums to units in which the tile's products of probability and V's scale are below 2^15 for each head again.
// Units only grow here, so nothing overflows.
template <int D>
__device__ inline void grow_units(State<D, 1>& st, const float (&sc)[Shape<D, 1>::SUB][4], const Scales<D, 1>& scale, float scale_log2, float r0, float r1, int steps) {
  auto exponent = [](float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; };
  int k0 = -1000, k1 = -1000, top = -1000;
#pragma unroll
  for (int s = 0; s < Shape<D, 1>::SUB; ++s) {
    if (s > 0 && s >= steps) break;
    float pr[4];
    probabilities(pr, sc[s], scale_log2, r0, r1);
    const int e = exponent(scale.of[s].y);
    k0 = max(k0, e + exponent(fmaxf(pr[0], pr[2])));                   // (NaN beside a number counts for nothing)
    k1 = max(k1, e + exponent(fmaxf(pr[1], pr[3])));
    top = max(top, e);
  }
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    k0 = max(k0, __shfl_xor_sync(0xffffffffu, k0, o));
    k1 = max(k1, __shfl_xor_sync(0xffffffffu, k1, o));
  }
  const float n0 = fminf(st.e0, (float)min(13 - k0, 125 - top)), n1 = fminf(st.e1, (float)min(13 - k1, 125 - top));
  const float f0 = ex2(n0 - st.e0), f1 = ex2(n1 - st.e1);
#pragma unroll
  for (int i = 0; i < Shape<D, 1>::MT; ++i) { st.o[i][0] *= f0; st.o[i][1] *= f1; st.o[i][2] *= f0; st.o[i][3] *= f1; }
  st.e0 = n0; st.e1 = n1;
  st.c0 = ex2(n0); st.c1 = ex2(n1);
}
// Whether one of the four is above 2^15 or NaN.
__device__ inline bool beyond(uint32_t a, uint32_t b) {
  const __half2 most = __hmax2_nan(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return !__hble2(most, __half2half2(__ushort_as_half(0x7800)));
}

// The second half of tile_values for an 8-bit cache: probabilities from the scores against the reference r0, r1, and
// O^T += V^T P^T.  The probabilities enter the product as fp16 (11 bits: half a step is 2^-11, an eighth of the result's own rounding, and
// V has four bits; a second term would cost as many MMA instructions again), times the step's scale of V, in units of each head's own:
// the largest product of the two so far was 2^13 to 2^15 when it came, whichever of them made it large, and none is above 2^15.
// What is 2^27 below it or less loses bits (to 2^-38 of it): a long tail behind a key that takes nearly all of the weight counts in
// full, and blocks whose scales are any powers of two apart can neither overflow nor hide each other.  One check a tile, on the
// packed products (a check a step keeps the steps apart: d = 16 36.6 us against 34.8, d = 32 40.2 against 39.2, for 64 sequences of up to
// 16000 keys; in logarithms of the scores, before the tile's vote on the maximum, 34.8 and 38.7, but d = 64 57.6 against 55.6).
template <int D>
__device__ inline void add_values8(State<D, 1>& st, const float (&sc)[Shape<D, 1>::SUB][4], Tile<D, 1>& x, const Scales<D, 1>& scale, float scale_log2,
                                   float r0, float r1, int key0, int len, int t) {
  using Sh = Shape<D, 1>;
  const int steps = (len - key0 + 15) >> 4;        // of the tile that have been copied
  uint32_t h[Sh::SUB][2];
  auto products = [&](bool sums) {                 // whether one of them is above 2^15 (or not a number: a factor beyond fp32 and a zero)
    bool over = false;
#pragma unroll
    for (int s = 0; s < Sh::SUB; ++s) {
      float pr[4];
      probabilities(pr, sc[s], scale_log2, r0, r1);
      if (sums) {
        st.l0 += pr[0] + pr[2];
        st.l1 += pr[1] + pr[3];
      }
      const float unit = s > 0 && s >= steps ? 0.f : scale.of[s].y, f0 = unit * st.c0, f1 = unit * st.c1;
      h[s][0] = pack_f16(pr[0] * f0, pr[1] * f1);
      h[s][1] = pack_f16(pr[2] * f0, pr[3] * f1);
      over |= beyond(h[s][0], h[s][1]);
    }
    return over;
  };
  if (__any_sync(0xffffffffu, products(true))) {
    grow_units<D>(st, sc, scale, scale_log2, r0, r1, steps);
    products(false);
  }
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s) {
    if (s > 0 && s >= steps) break;
    const uint32_t b0 = transpose8x8(h[s][0]), b1 = transpose8x8(h[s][1]);
    if (s == 0) clear_behind(x, key0, len, t);
#pragma unroll
    for (int c = 0; c < Sh::VCH; ++c)
#pragma unroll
      for (int w = 0; w < Sh::VW; ++w) {
        // (rows g, g + 8) x (keys 2t, 2t+1 | 2t+8, 2t+9): elements 2i and 2i + 1 of the thread's
        uint32_t a[4];
        widen(__byte_perm(x.v[s][0][c][w], x.v[s][1][c][w], 0x5140), a[0], a[1]);
        widen(__byte_perm(x.v[s][2][c][w], x.v[s][3][c][w], 0x5140), a[2], a[3]);
        mma16816_f16(st.o[2 * (c * Sh::VW + w)], a[0], a[1], a[2], a[3], b0, b1);
        if constexpr (!Sh::HALF_V) {
          widen(__byte_perm(x.v[s][0][c][w], x.v[s][1][c][w], 0x7362), a[0], a[1]);
          widen(__byte_perm(x.v[s][2][c][w], x.v[s][3][c][w], 0x7362), a[2], a[3]);
          mma16816_f16(st.o[2 * (c * Sh::VW + w) + 1], a[0], a[1], a[2], a[3], b0, b1);
        }
      }
  }
}

// 8 bits: the reference rises by `up` (log2), and c may be 2^most.  c rises as far as it may with the reference, so that the sums keep
// their size (nothing is lost when keys without values take the weight); returns the factor for the sums that is left, at most 1.
__device__ inline float move_unit(float& e, float& c, float up, float most) {
  const float n = fminf(e + up, fminf(most, kMostUp)), f = ex2(n - e - up);
  e = n;
  c = ex2(n);
  return f;
}

// Softmax step and O^T += V^T P^T of the tile that begins at key0 of `len` keys.
template <int D, int B>
__device__ inline void tile_values(State<D, B>& st, float (&sc)[Shape<D, B>::SUB][4], Tile<D, B>& x, const Scales<D, B>& scale, float scale_log2, int key0, int len, int g, int t) {
  using Sh = Shape<D, B>;
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
    float f0 = st.m0 == -INFINITY ? 0.f : ex2((st.m0 - n0) * scale_log2);
    float f1 = st.m1 == -INFINITY ? 0.f : ex2((st.m1 - n1) * scale_log2);
    st.l0 *= f0; st.l1 *= f1;
    if constexpr (B == 1) {                          // units, by the largest product of probability and scale (log2), and the largest scale
      float w0 = -INFINITY, w1 = -INFINITY, top = -INFINITY;
#pragma unroll
      for (int s = 0; s < Sh::SUB; ++s) {
        const float unit = s > 0 && key0 + 16 * s >= len ? -INFINITY : __log2f(scale.of[s].y);
        w0 = fmaxf(w0, fmaf(fmaxf(sc[s][0], sc[s][2]), scale_log2, unit));
        w1 = fmaxf(w1, fmaf(fmaxf(sc[s][1], sc[s][3]), scale_log2, unit));
        top = fmaxf(top, unit);
      }
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        w0 = fmaxf(w0, __shfl_xor_sync(0xffffffffu, w0, o));
        w1 = fmaxf(w1, __shfl_xor_sync(0xffffffffu, w1, o));
      }
      // (no reference yet: no sums)
      const float g0 = move_unit(st.e0, st.c0, st.m0 == -INFINITY ? 0.f : (n0 - st.m0) * scale_log2, fminf(14.f - fmaf(-n0, scale_log2, w0), 125.f - top));
      const float g1 = move_unit(st.e1, st.c1, st.m1 == -INFINITY ? 0.f : (n1 - st.m1) * scale_log2, fminf(14.f - fmaf(-n1, scale_log2, w1), 125.f - top));
      f0 = st.m0 == -INFINITY ? 0.f : g0;
      f1 = st.m1 == -INFINITY ? 0.f : g1;
    }
    st.m0 = n0; st.m1 = n1;
#pragma unroll
    for (int i = 0; i < Sh::MT; ++i) { st.o[i][0] *= f0; st.o[i][1] *= f1; st.o[i][2] *= f0; st.o[i][3] *= f1; }
  }
  const float r0 = st.m0 == -INFINITY ? 0.f : st.m0 * scale_log2, r1 = st.m1 == -INFINITY ? 0.f : st.m1 * scale_log2;
  if constexpr (B == 1) {
    add_values8<D>(st, sc, x, scale, scale_log2, r0, r1, key0, len, t);
  } else {
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
    clear_behind(x, key0, len, t);
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
}

// The sums of the eight thread rows; maxima in log2 units from here on.
template <int D, int B>
__device__ inline void finish(State<D, B>& st, float scale_log2) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    st.l0 += __shfl_xor_sync(0xffffffffu, st.l0, o);
    st.l1 += __shfl_xor_sync(0xffffffffu, st.l1, o);
  }
  st.m0 *= scale_log2;
  st.m1 *= scale_log2;
  if constexpr (B == 1) {
    const float u0 = ex2(-st.e0), u1 = ex2(-st.e1);
#pragma unroll
    for (int i = 0; i < Shape<D, B>::MT; ++i) { st.o[i][0] *= u0; st.o[i][1] *= u1; st.o[i][2] *= u0; st.o[i][3] *= u1; }
  }
}

// Element of the head that accumulator row (i, half) of thread g holds (half: rows g / g + 8 of the MMA tile).
template <int D, int B>
__device__ inline int elem_of(int i, int half, int g) {
  if constexpr (D == 8) return half ? -1 : g;
  const int e = 2 * i + half;
  if constexpr (D == 128 && B == 2) return (e / 8) * 64 + g * 8 + e % 8;
  return g * (D / 8) + e;
}

__device__ inline long long lse_at(const DecParams& p, long long seq, int head) {
  const long long s = seq / p.n_seqs;
  return (s * p.heads + head) * p.n_seqs + (seq - s * p.n_seqs);
}

// The thread's elements of a head: OCH runs of OW words (pairs of elements, accumulators 2i and 2i + 1), run c from element
// out_elem(c, g) on.
template <int D, int B>
struct Out {
  static constexpr int OW = Shape<D, B>::MT < 4 ? Shape<D, B>::MT : 4, OCH = Shape<D, B>::MT / OW;
};
template <int D, int B>
__device__ inline int out_elem(int c, int g) { return D == 128 && B == 2 ? c * 64 + g * 8 : g * (D / 8) + c * 8; }

// A warp's result for one of the thread's two heads (col 0, 1): the finished row, or a part.
template <int D, int B>
__device__ inline void store_head(const DecParams& p, const State<D, B>& st, int col, long long seq, int head, int g, int len) {
  using O = Out<D, B>;
  const float l = col ? st.l1 : st.l0, m = col ? st.m1 : st.m0, inv = len == 0 ? 0.f : 1.f / l;
  __nv_bfloat16* out = p.out + (seq * p.heads + head) * D;
  if constexpr (D == 8) {
    out[g] = __float2bfloat16(st.o[0][col] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < O::OCH; ++c) {
      uint32_t w[O::OW];
#pragma unroll
      for (int j = 0; j < O::OW; ++j) w[j] = pack_bf16(st.o[c * O::OW + j][col] * inv, st.o[c * O::OW + j][2 + col] * inv);
      __nv_bfloat16* dst = out + out_elem<D, B>(c, g);
      if constexpr (O::OW == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      else if constexpr (O::OW == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
  }
  if (g == 0 && p.lse) p.lse[lse_at(p, seq, head)] = len == 0 ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int D, int B>
__device__ inline void store_part(float* row, const State<D, B>& st, int col, int head, int g) {
  using O = Out<D, B>;
  if constexpr (D == 8) {
    row[g] = st.o[0][col];
  } else {
#pragma unroll
    for (int c = 0; c < O::OCH; ++c)
#pragma unroll
      for (int j = 0; j < O::OW; ++j)
        *reinterpret_cast<float2*>(row + out_elem<D, B>(c, g) + 2 * j) = make_float2(st.o[c * O::OW + j][col], st.o[c * O::OW + j][2 + col]);
  }
  if (g == 0)
    *reinterpret_cast<float4*>(row + D) = make_float4(col ? st.m1 : st.m0, col ? st.l1 : st.l0, __int_as_float(head), 0.f);
}

// Whole items, one cluster of CTAs per (sequence, KV position, row tile): its warps take the item's tiles in turn; the warps
// of a CTA join in shared memory, the CTAs in the others' shared memory, every one for its share of the result.
template <int D, int B>
__global__ void __launch_bounds__(kDecThreads, D == 128 ? 3 : (D >= 32 ? 4 : 5)) decode_whole_kernel(const DecParams p) {
  using Sh = Shape<D, B>;
  __shared__ float sm[kDecWarps * kCols * (D + 2)];
  __shared__ float joined[kCols * (D + 2)];
  __shared__ int cols[kDecWarps][kCols];
  __shared__ __align__(16) QueryBuf<D, B> qbuf[kDecWarps];
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
  int ids = fetch_pages<Sh::SUB>(p, seq, first, stride, lane);
  const int len = clamped_len(p, p.len[seq]), tiles = (len + Sh::TILE - 1) / Sh::TILE;
  ids = check_pages<Sh::SUB>(p, ids, len - 1, first, stride, lane);
  wait_copies();
  const long long k_at = at_k<D, B>(p, pos, g, t), v_at = at_v<D, B>(p, pos, g, t);
  constexpr int AHEAD = 32 / Sh::SUB;
  State<D, B> st;
  reset<D, B>(st);
  Tile<D, B> x;
  int key0 = first * Sh::TILE;
  if (first < tiles) {
    load_k<D, B>(x, p, ids, 0, key0, len - 1, pos, k_at, lane);
    load_v<D, B>(x, p, ids, 0, key0, len - 1, v_at, lane);
  }
  __syncthreads();
  find_heads(p, hd, s, pos, rt, lane, cols[warp]);
  if (cols[warp][0] < 0) return;                   // no head reads this position (the same in the whole cluster)
  Query<D, B> q;
  prefetch_q<D, B>(qbuf[warp], p, seq, cols[warp][g], lane);
  wait_copies();
  take_q<D, B>(q, qbuf[warp], lane);
  for (int tile = first, n = 0; tile < tiles; tile += stride, key0 += stride * Sh::TILE) {
    const bool more = tile + stride < tiles;
    const int next0 = key0 + stride * Sh::TILE;
    float sc[Sh::SUB][4];
    const Scales<D, B> scale = gather_scales(x);
    tile_scores<D, B>(sc, x, q, scale);
    if (more) {
      if (++n == AHEAD) {
        ids = check_pages<Sh::SUB>(p, fetch_pages<Sh::SUB>(p, seq, tile + stride, stride, lane), len - 1, tile + stride, stride, lane);
        n = 0;
      }
      load_k<D, B>(x, p, ids, n, next0, len - 1, pos, k_at, lane);
    }
    tile_values<D, B>(st, sc, x, scale, p.scale_log2, key0, len, g, t);
    if (more) load_v<D, B>(x, p, ids, n, next0, len - 1, v_at, lane);
  }
  finish<D, B>(st, p.scale_log2);
  float* mine = sm + warp * kCols * (D + 2);       // [head][D + 2]
#pragma unroll
  for (int i = 0; i < Sh::MT; ++i)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = elem_of<D, B>(i, half, g);
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
template <int D, int B>
__device__ inline int tiles_of(int len) { return max(1, (len + Shape<D, B>::TILE - 1) / Shape<D, B>::TILE); }

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

// An 8-bit cache's tiles in the split kernel: a ring of them per warp, filled by bulk copies (the 16 rows of a step lie next to
// each other in their page: one copy for K, one for V).  Half the bytes for the same arithmetic: with the next tile in
// registers, as in 16 bits, the loads in flight do not cover a tile's time (eight subnets of d = 128 246 us, 64 ragged sequences
// with 32 heads on 4 positions of d = 64 75; through rings, at first, 205 and 60).  Three tiles of 16 keys and 12 warps an SM at d = 128
// (two: 193 us against 191; two of 32 keys and 8 warps, at 195: 204), two of 32 keys and 16 warps at d = 64 (three and 12 warps:
// 57.6 against 55.1; two of 64 keys and 12 warps and three of 16, at 58: 63 and 63 to 70).
template <int D>
constexpr int kRing = D == 128 ? 3 : 2;
template <int D>
struct Ring {
  using Sh = Shape<D, 1>;
  struct alignas(16) {
    uint8_t k[Sh::TILE * D], v[Sh::TILE * D];
  } tile[kRing<D>];
  float2 scale[kRing<D>][Sh::SUB];
  alignas(16) uint64_t full[kRing<D>];           // 2 SUB arrivals: of every step, its bytes to expect and its scales
};

template <int D>
__device__ inline void take_values(Tile<D, 1>& x, const uint8_t* v, int g, int t) {
  using Sh = Shape<D, 1>;
#pragma unroll
  for (int s = 0; s < Sh::SUB; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < Sh::VCH; ++c) {
        const uint8_t* row = v + (16 * s + 2 * t + (r & 1) + 8 * (r >> 1)) * D;
        if constexpr (Sh::HALF_V) x.v[s][r][c][0] = *reinterpret_cast<const unsigned short*>(row + 2 * g);
        else take_words<Sh::VW>(x.v[s][r][c], row + 4 * Sh::VW * (8 * c + g));
      }
}

// Tiles that go through shared memory in the split kernel.
template <int D, int B>
constexpr bool kStaged = B == 2 && (D == 16 || D == 32);

template <int D, int B>
constexpr int kRingBytes = B == 1 ? kDecWarps * (int)sizeof(Ring<D>) : (kStaged<D, B> ? 2 * kDecWarps * (int)sizeof(Stage<D, B>) : 0);

constexpr int kCountCache = 256;      // KV positions of all subnets whose heads a CTA counts

// QUITS: for the self-test of the way out that a warp takes when a wait of it has run out.
template <int D, int B, bool QUITS = false>
__global__ void __launch_bounds__(kDecThreads, D == 64 ? 4 : 3) decode_split_kernel(const DecParams p) {
  using Sh = Shape<D, B>;
  __shared__ int cols[kDecWarps][2][kCols];
  __shared__ __align__(16) QueryBuf<D, B> qbuf[kDecWarps];
  extern __shared__ __align__(16) unsigned char ring[];       // [kDecWarps][2] stages, or [kDecWarps] rings
  __shared__ int items[TWIST_MAX_SUBNETS], counts[kCountCache];
  __shared__ int32_t lens[kLenCache], head_cache[kHeadCache], pos_cache[kPosCache];
  __shared__ uint32_t warp_sum[kDecWarps];
  __shared__ __align__(16) uint32_t before[kDecThreads];    // cost of the sequences before each thread's
  __shared__ volatile int abort_flag;                       // a wait for a copy ran out
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int N = p.S * p.n_seqs, per = (N + kDecThreads - 1) / kDecThreads;
  for (int i = threadIdx.x; i < kCountCache; i += kDecThreads) counts[i] = 0;
  if (B == 1 && threadIdx.x == 0) abort_flag = 0;
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
      mine += (uint32_t)items[s] * (kItemCost<B> + tiles_of<D, B>(len_of(i)));
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
    x.nt = tiles_of<D, B>(x.len);
  };
  {
    const uint32_t u = cut.begin(c);
    int owner = -1;                                          // the last thread whose sequences begin at or before u
    for (int k = 0; k < kDecThreads; k += 32) owner += __popc(__ballot_sync(0xffffffffu, before[k + lane] <= u));
    uint32_t base = before[owner], cost;
    int seq = owner * per, s = seq / p.n_seqs, b = seq - s * p.n_seqs;
    for (;;) {
      enter(now, seq, s);
      cost = (uint32_t)items[s] * (now.nt + kItemCost<B>);
      if (u < base + cost) break;
      base += cost;
      ++seq;
      if (++b == p.n_seqs) { b = 0; ++s; }
    }
    const uint32_t one = now.nt + kItemCost<B>;
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
    now.t0 = max(0, (int)x0 - kItemCost<B>);
    now.t1 = max(0, (int)x1 - kItemCost<B>);
    left -= x1 - x0;
  }
  if (now.t1 <= now.t0) return;                           // the item's own cost is all there is: the next warp has its tiles

  constexpr int AHEAD = 32 / Sh::SUB;
  // the item behind another one (its t1 is the caller's)
  auto following = [&](Segment x) {
    x.t0 = 0;
    if (++x.rt >= row_tiles(x.s, x.pos)) {
      x.rt = 0;
      do {
        if (++x.pos == p.kv_max) {
          x.pos = 0;
          enter(x, x.seq + 1, (x.seq + 1) / p.n_seqs);
        }
      } while (row_tiles(x.s, x.pos) == 0);
    }
    return x;
  };
  // the entry of the item that begins with segment x
  auto describe = [&](const Segment& x, int4 entry) {
    if (lane != 0) return;
    if (!p.by_item) {
      p.desc[c] = entry;
      return;
    }
    const int all = p.kv_max * p.row_tiles, item = x.pos * p.row_tiles + x.rt;
    int4* desc = p.desc + (long long)x.seq * all;
    desc[item] = entry;
    // the neighbours in the table that are no items
    auto is_item = [&](int k) { return k % p.row_tiles < row_tiles(x.s, k / p.row_tiles); };
    for (int k = item + 1; k < all && !is_item(k); ++k) desc[k] = make_int4(0, 0, 0, 0);
    for (int k = item - 1; k >= 0 && !is_item(k); --k) desc[k] = make_int4(0, 0, 0, 0);
  };
  // a segment's result
  auto store = [&](const State<D, B>& st, const Segment& now, int hq) {
    const bool whole = now.t0 == 0 && now.t1 == now.nt;
    const int h0 = __shfl_sync(0xffffffffu, hq, 8 * t), h1 = __shfl_sync(0xffffffffu, hq, 8 * t + 4);
    if (whole) {
      if (h0 >= 0) store_head<D, B>(p, st, 0, now.seq, h0, g, now.len);
      if (h1 >= 0) store_head<D, B>(p, st, 1, now.seq, h1, g, now.len);
    } else {
      float* part = p.part + (2ll * c + (now.t0 == 0)) * kCols * kPartRow(D);
      if (h0 >= 0) store_part<D, B>(part + 2 * t * kPartRow(D), st, 0, h0, g);
      if (h1 >= 0) store_part<D, B>(part + (2 * t + 1) * kPartRow(D), st, 1, h1, g);
    }
    if (now.t0 == 0 && (p.by_item || !whole)) {
      const int heads = __popc(__ballot_sync(0xffffffffu, hq >= 0 && t == 0));
      const int parts = whole ? 0 : (int)(cut.piece_of(item0 + kItemCost<B> + now.nt - 1) - c);          // further parts of the item
      describe(now, make_int4(now.seq, heads, parts, (int)c));
    }
  };
  if constexpr (B == 1) {
    Ring<D>& ring8 = reinterpret_cast<Ring<D>*>(ring)[warp];
    if (lane == 0) {
      for (int i = 0; i < kRing<D>; ++i) mbar_init(smem_u32(&ring8.full[i]), 2 * Sh::SUB);
      fence_async_smem();
    }
    __syncwarp();
    // The filling side walks the line by itself, kRing tiles ahead of the other: its segment, the one behind it, and where the
    // lane's step of the current AHEAD tiles lies (lane l: step l % SUB of the l / SUB-th).
    Segment at = now, behind = now;
    uint32_t at_left = left;
    bool at_more = false, live = false;
    int tile = now.t0, n = 0, head_ids = 0, to = 0;
    long long from = 0, scale_from = 0;
    int next_ids = fetch_pages<Sh::SUB>(p, now.seq, now.t0, 1, lane);
    auto window = [&](int ids) {                     // the page ids of the AHEAD tiles from `tile` on have come
      ids = check_pages<Sh::SUB>(p, ids, at.len - 1, tile, 1, lane);
      next_ids = fetch_pages<Sh::SUB>(p, at.seq, tile + AHEAD, 1, lane);
      const int key = (int)step_key<Sh::SUB>(tile, 1, lane), in_page = key & ((1 << p.page_shift) - 1);
      live = key < at.len;
      from = ids * p.page_stride + (((long long)at.pos << p.page_shift) + in_page) * D;
      scale_from = (((long long)ids * p.kv_max + at.pos) << (p.page_shift - 4)) + (in_page >> 4);
      n = 0;
    };
    auto look = [&] {
      at_more = at_left > (uint32_t)kItemCost<B>;
      if (at_more) {
        behind = following(at);
        behind.t1 = (int)min((uint32_t)behind.nt, at_left - kItemCost<B>);
        head_ids = fetch_pages<Sh::SUB>(p, behind.seq, 0, 1, lane);
      }
    };
    auto fill = [&] {                                // a group of copies, empty behind the last tile
      while (tile >= at.t1 || at.len == 0) {
        if (!at_more) { commit_copies(); return; }
        at_left -= behind.t1 + kItemCost<B>;
        at = behind;
        tile = 0;
        window(head_ids);
        look();
      }
      if (n == AHEAD) window(next_ids);
      if (lane / Sh::SUB == n) {
        const int step = lane % Sh::SUB;
        const uint32_t bar = smem_u32(&ring8.full[to]);
        if (live) {
          mbar_expect_tx(bar, 32 * D);
          bulk_load(smem_u32(ring8.tile[to].k + 16 * D * step), static_cast<const uint8_t*>(p.k) + from, 16 * D, bar);
          bulk_load(smem_u32(ring8.tile[to].v + 16 * D * step), static_cast<const uint8_t*>(p.v) + from, 16 * D, bar);
          copy_async<8>(&ring8.scale[to][step], p.scales + scale_from);
          asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
        } else {                                       // a step behind the end
          mbar_arrive(bar);
          mbar_arrive(bar);
        }
      }
      commit_copies();
      to = to + 1 == kRing<D> ? 0 : to + 1;
      ++tile;
      ++n;
    };
    find_heads(p, hd, now.s, now.pos, now.rt, lane, cols[warp][0]);
    prefetch_q<D, B>(qbuf[warp], p, now.seq, cols[warp][0][g], lane);
    commit_copies();
    window(next_ids);
    look();
#pragma unroll 1
    for (int i = 0; i < kRing<D>; ++i) fill();
    auto quits = [&](int tile) {
      if (c % (uint32_t)p.quit_every != 0 || tile < p.quit_tile) return false;
      if (lane == 0) {
        abort_flag = 1;
        note_status(p.status, (int)TWIST_ERR_DEVICE_TIMEOUT);
      }
      return true;
    };
    int buf = 0, slot = 0, since = kRing<D>;
    uint32_t parity = 0;
    bool ok = true;
    for (;;) {
      // the queries: their group is older than those of the tiles filled since, of which the newest need not have come
      Query<D, B> q;
      if (since >= 2) wait_copies_but<2>();
      else wait_copies();
      take_q<D, B>(q, qbuf[warp], lane);
      const int hq = cols[warp][buf][g];
      const bool more = left > (uint32_t)kItemCost<B>;
      Segment next = now;
      if (more) {
        next = following(now);
        next.t1 = (int)min((uint32_t)next.nt, left - kItemCost<B>);
        find_heads(p, hd, next.s, next.pos, next.rt, lane, cols[warp][buf ^ 1]);
        prefetch_q<D, B>(qbuf[warp], p, next.seq, cols[warp][buf ^ 1][g], lane);
      }
      commit_copies();
      since = now.len > 0 ? now.t1 - now.t0 : 0;
      State<D, B> st;
      reset<D, B>(st);
      if (now.len > 0) {
        for (int i = now.t0; i < now.t1; ++i) {
          ok = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&ring8.full[slot]), parity, &abort_flag, p.status));
          if constexpr (QUITS) ok = ok && !quits(i - now.t0);
          if (!ok) break;
          Tile<D, B> x;
          Scales<D, B> scale;
          float sc[Sh::SUB][4];
#pragma unroll
          for (int s = 0; s < Sh::SUB; ++s) scale.of[s] = ring8.scale[slot][s];
#pragma unroll
          for (int s = 0; s < Sh::SUB; ++s) take_keys<D, B>(x.k[s], ring8.tile[slot].k + 16 * D * s, g, t);
          tile_scores<D, B>(sc, x, q, scale);
          take_values<D>(x, ring8.tile[slot].v, g, t);
          tile_values<D, B>(st, sc, x, scale, p.scale_log2, i * Sh::TILE, now.len, g, t);
          __syncwarp();                                // the tile has been read
          if (++slot == kRing<D>) { slot = 0; parity ^= 1; }
          fill();
        }
      }
      if (!ok) break;
      finish<D, B>(st, p.scale_log2);
      store(st, now, hq);
      if (!more) break;
      item0 += now.nt + kItemCost<B>;
      left -= next.t1 + kItemCost<B>;
      now = next;
      buf ^= 1;
    }
    if (!ok) {
      // the join will read an entry of every item: those that were to begin here get empty ones
      while (p.by_item) {
        if (now.t0 == 0) describe(now, make_int4(0, 0, 0, 0));
        if (left <= (uint32_t)kItemCost<B>) break;
        now = following(now);
        now.t1 = (int)min((uint32_t)now.nt, left - kItemCost<B>);
        left -= now.t1 + kItemCost<B>;
      }
      drain_after_abort(&abort_flag);
    }
    return;
  } else {
  constexpr bool STAGED = kStaged<D, B>;
  const Scales<D, B> none{};
  Stage<D, B>* stages = reinterpret_cast<Stage<D, B>*>(ring) + 2 * warp;
  Tile<D, B> x;
  int ids = fetch_pages<Sh::SUB>(p, now.seq, now.t0, 1, lane);
  int next_ids = fetch_pages<Sh::SUB>(p, now.seq, now.t0 + AHEAD, 1, lane);     // unchecked until it becomes `ids`
  int n = 0;                                        // number of the loaded tile in its window of page ids
  int buf = 0, stage = 0;
  find_heads(p, hd, now.s, now.pos, now.rt, lane, cols[warp][0]);
  prefetch_q<D, B>(qbuf[warp], p, now.seq, cols[warp][0][g], lane);
  ids = check_pages<Sh::SUB>(p, ids, now.len - 1, now.t0, 1, lane);
  if (now.len > 0) {
    if constexpr (STAGED) stage_k<D, B>(stages[0], p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_k<D, B>(p, now.pos, g, t), lane);
    else load_k<D, B>(x, p, ids, 0, now.t0 * Sh::TILE, now.len - 1, now.pos, at_k<D, B>(p, now.pos, g, t), lane);
  }
  commit_copies();                                  // the queries travel with the first keys
  if (now.len > 0) {
    if constexpr (STAGED) stage_v<D, B>(stages[0], p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_v<D, B>(p, now.pos, g, t), lane);
    else load_v<D, B>(x, p, ids, 0, now.t0 * Sh::TILE, now.len - 1, at_v<D, B>(p, now.pos, g, t), lane);
  }
  commit_copies();
  for (;;) {
    Query<D, B> q;
    if constexpr (STAGED) wait_copies_but<1>();
    else wait_copies();
    take_q<D, B>(q, qbuf[warp], lane);
    const int hq = cols[warp][buf][g];
    // the segment behind this one: its first pages, its heads and their queries on their way before they are needed
    const bool more = left > (uint32_t)kItemCost<B>;
    Segment next = now;
    int head_ids = 0;
    if (more) {
      next = following(now);
      next.t1 = (int)min((uint32_t)next.nt, left - kItemCost<B>);
      head_ids = fetch_pages<Sh::SUB>(p, next.seq, 0, 1, lane);
      find_heads(p, hd, next.s, next.pos, next.rt, lane, cols[warp][buf ^ 1]);
      prefetch_q<D, B>(qbuf[warp], p, next.seq, cols[warp][buf ^ 1][g], lane);          // complete with the next tile's keys
    }
    State<D, B> st;
    reset<D, B>(st);
    for (int tile = now.t0; tile < now.t1; ++tile) {
      // the tile to load: the item's next one or the next item's first
      const bool inside = tile + 1 < now.t1;
      const int key0 = inside ? (tile + 1) * Sh::TILE : 0, last_key = inside ? now.len - 1 : next.len - 1, of = inside ? now.pos : next.pos;
      const bool load = (inside || more) && last_key >= 0;
      if (inside) {
        if (++n == AHEAD) {
          ids = check_pages<Sh::SUB>(p, next_ids, now.len - 1, tile + 1, 1, lane);
          next_ids = fetch_pages<Sh::SUB>(p, now.seq, tile + 1 + AHEAD, 1, lane);
          n = 0;
        }
      } else {
        ids = check_pages<Sh::SUB>(p, head_ids, more ? next.len - 1 : -1, 0, 1, lane);
        next_ids = fetch_pages<Sh::SUB>(p, next.seq, AHEAD, 1, lane);
        n = 0;
      }
      float sc[Sh::SUB][4];
      if constexpr (STAGED) {
        Stage<D, B>& to = stages[stage ^ 1];
        if (load) stage_k<D, B>(to, p, ids, n, key0, last_key, at_k<D, B>(p, of, g, t), lane);
        commit_copies();
        if (load) stage_v<D, B>(to, p, ids, n, key0, last_key, at_v<D, B>(p, of, g, t), lane);
        commit_copies();
        wait_copies_but<3>();
        take_k<D, B>(x, stages[stage], lane);
        tile_scores<D, B>(sc, x, q, none);
        wait_copies_but<2>();
        take_v<D, B>(x, stages[stage], lane);
        if (now.len > 0) tile_values<D, B>(st, sc, x, none, p.scale_log2, tile * Sh::TILE, now.len, g, t);
        stage ^= 1;
      } else {
        tile_scores<D, B>(sc, x, q, none);
        if (load) load_k<D, B>(x, p, ids, n, key0, last_key, of, at_k<D, B>(p, of, g, t), lane);
        if (now.len > 0) tile_values<D, B>(st, sc, x, none, p.scale_log2, tile * Sh::TILE, now.len, g, t);
        if (load) load_v<D, B>(x, p, ids, n, key0, last_key, at_v<D, B>(p, of, g, t), lane);
      }
    }
    finish<D, B>(st, p.scale_log2);
    store(st, now, hq);
    if (!more) break;
    item0 += now.nt + kItemCost<B>;
    left -= next.t1 + kItemCost<B>;
    now = next;
    buf ^= 1;
  }
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

template <int D, int B, bool QUITS = false>
int run(DecParams& p, long long max_len, cudaStream_t st) {
  const long long items = (long long)p.S * p.n_seqs * p.kv_max * p.row_tiles;
  // the line is counted in 32 bits
  const long long longest = (((long long)p.max_pages << p.page_shift) + Shape<D, B>::TILE - 1) / Shape<D, B>::TILE + 1 + kItemCost<B>;
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
    TWIST_CUDA_TRY(cudaFuncSetAttribute(decode_split_kernel<D, B, QUITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes<D, B>));
    TWIST_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, decode_split_kernel<D, B, QUITS>, kDecThreads, kRingBytes<D, B>));
    resident[slot] = n < 1 ? 1 : (n > kMaxCtasPerSm ? kMaxCtasPerSm : n);
  }
  const long long grid = (long long)sm_count() * resident[slot];
  // One cluster per item where that needs few turns: two tiles a warp are taken by a single CTA, more by as many CTAs as
  // leave a warp one, if all of them run at once.  Measured (d = 64, one sequence of 8 heads, 1024 keys): 5.0 us against 9.2
  // through the line; 512 items of 512 keys, all at once: 15 against 19.  The line is ahead where a warp would take more
  // than kShortTiles tiles, where the items fill the GPU kShortWork tiles a warp deep (256 ragged items of up to 2048
  // keys: 21 us against 27 to 34), and earlier where they do not run at once (512 items of 256 keys, d = 128: 18.2
  // against 19.6).  An 8-bit cache is counted in the same 16 keys from d = 64 on (256 ragged items of up to 2048 keys, d = 64:
  // 17.0 us through the line, 22.7 the short way; 512 items of 512 keys 13.2 the short way, 15.5 through the line).
  constexpr int UNIT = D >= 64 ? 16 : Shape<D, B>::TILE;
  const long long tiles = (max_len + UNIT - 1) / UNIT;
  int cluster = 1;
  if (tiles > 2 * kDecWarps)
    while (cluster < kMaxCluster && 2 * cluster * items <= grid && tiles > kDecWarps * cluster) cluster *= 2;
  if (!QUITS && items <= 2 * grid && tiles <= kShortTiles * kDecWarps * cluster &&
      tiles * items <= (items <= grid ? kShortWork : kShortWaves) * grid * kDecWarps) {
    TWIST_CUDA_TRY(launch_overlapped(decode_whole_kernel<D, B>, dim3((unsigned)(items * cluster)), dim3(kDecThreads), 0, st, cluster, p));
    return TWIST_OK;
  }
  p.by_item = items <= grid * kDecWarps;
  TWIST_CUDA_TRY(launch_overlapped(decode_split_kernel<D, B, QUITS>, dim3((unsigned)grid), dim3(kDecThreads), kRingBytes<D, B>, st, 1, p));
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

namespace {

// The checks and the parameters that both caches share; A: twist_attn_decode_args or twist_attn_decode_q8_args.
template <typename A>
int set_up(const A* a, DecParams& p, int row_unit) {
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->head_keep <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 ||
      a->max_pages <= 0 || a->page_size <= 0 || a->max_len < 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if ((dh != 8 || row_unit > 8) && dh != 16 && dh != 32 && dh != 64 && dh != 128) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets > TWIST_MAX_SUBNETS || a->n_heads > 1024 || a->head_keep > 1024) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->n_subnets * a->n_seqs > 65535) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll - 1024) return TWIST_ERR_UNSUPPORTED;   // positions are 32-bit
  if (a->page_stride % row_unit != 0 || a->page_stride < (long long)a->kv_max * a->page_size * dh) return TWIST_ERR_SHAPE;
  if (a->q_stride % 8 != 0 || a->q_stride < (long long)a->head_keep * dh) return TWIST_ERR_SHAPE;
  if (a->head_idx) {
    if (!a->kv_pos || a->n_heads <= 0 || a->n_kv_heads <= 0 || a->n_heads % a->n_kv_heads != 0) return TWIST_ERR_SHAPE;
  } else if (a->kv_max != a->head_keep) {
    return TWIST_ERR_SHAPE;
  }
  if (!a->q || !a->k_cache || !a->v_cache || !a->page_table || !a->kv_len || !a->out) return TWIST_ERR_NULL;
  if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->out) || !aligned16(a->ws)) return TWIST_ERR_SHAPE;
  if (!a->ws || a->ws_bytes < twist_attn_decode_workspace_bytes(dh)) return TWIST_ERR_WORKSPACE;
  memset(&p, 0, sizeof(p));
  p.q = static_cast<const __nv_bfloat16*>(a->q);
  p.k = a->k_cache;
  p.v = a->v_cache;
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
  return TWIST_OK;
}

template <typename A>
long long bound_of(const A* a) {
  const long long table_len = (long long)a->max_pages * a->page_size;
  return a->max_len > 0 && a->max_len < table_len ? a->max_len : table_len;
}

int set_up_q8(const twist_attn_decode_q8_args* a, DecParams& p) {
  const int rc = set_up(a, p, 16);
  if (rc != TWIST_OK) return rc;
  if (!a->scales) return TWIST_ERR_NULL;
  if (!aligned16(a->scales)) return TWIST_ERR_SHAPE;
  p.scales = reinterpret_cast<const float2*>(a->scales);
  return TWIST_OK;
}

}  // namespace

extern "C" int32_t twist_attn_decode(const twist_attn_decode_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  DecParams p;
  const int rc = set_up(a, p, 8);
  if (rc != TWIST_OK) return rc;
  const long long max_len = bound_of(a);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (a->d_head) {
    case 8: return run<8, 2>(p, max_len, st);
    case 16: return run<16, 2>(p, max_len, st);
    case 32: return run<32, 2>(p, max_len, st);
    case 64: return run<64, 2>(p, max_len, st);
    default: return run<128, 2>(p, max_len, st);
  }
}

extern "C" int32_t twist_attn_decode_q8(const twist_attn_decode_q8_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  DecParams p;
  const int rc = set_up_q8(a, p);
  if (rc != TWIST_OK) return rc;
  const long long max_len = bound_of(a);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (a->d_head) {
    case 16: return run<16, 1>(p, max_len, st);
    case 32: return run<32, 1>(p, max_len, st);
    case 64: return run<64, 1>(p, max_len, st);
    default: return run<128, 1>(p, max_len, st);
  }
}

extern "C" int32_t twist_selftest_decode_quit(const twist_attn_decode_q8_args* a, int32_t every, int32_t tile, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (every <= 0 || tile < 0) return TWIST_ERR_SHAPE;
  if (a->d_head != 64) return TWIST_ERR_UNSUPPORTED;
  DecParams p;
  const int rc = set_up_q8(a, p);
  if (rc != TWIST_OK) return rc;
  p.quit_every = every;
  p.quit_tile = tile;
  return run<64, 1, true>(p, bound_of(a), static_cast<cudaStream_t>(stream));
}
