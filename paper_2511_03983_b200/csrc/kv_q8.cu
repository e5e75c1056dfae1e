// twist_kv_append_q8: new K and V rows into a paged cache of 8-bit numbers, K rotated by position on the way, and the
// rotated Q.
//
// A block is 16 slots of a KV position; its numbers are e4m3, value = number * scale with a power-of-two scale:
//     scale = max(scale of the tokens it holds already, smallest 2^e with max |x| <= 448 * 2^e over the new ones).
// The scale is known only when the whole block has been seen, and a block that holds tokens may have to be rounded again,
// so a block's new tokens belong to one warp: it rotates 16 rows of a head in registers (fp32), finds the largest
// magnitude with one shuffle reduction, and writes each number once.  The work is moving bytes (2 read and 1 written
// per element of K and V, 2 and 2 for Q): HBM-bound for prompts, latency-bound for the rows of a decoding step.
//
// A CTA takes the new tokens of one block of one sequence, all heads: the tokens are neighbouring rows at neighbouring
// positions, so the index data of a CTA is found once, and one table of (cos, sin) serves its heads (angles as in
// positions.cu: reduced in 64 bits).  A warp takes a head at a time, the rows of its next one on their way, and hands the
// elements of a pair from lane to lane; rotating in place is safe because a head's rows are read by one warp before it writes
// any of them.  Magnitudes are compared as integers, which finds what is not finite on the way: only then is every value looked at.
//
// One token of every sequence has a kernel of its own: D / 8 lanes a head, all heads at once, and one round trip for everything
// that does not hang on the page (512 tokens of 16 + 2 * 4 heads of 64: 10.3 us by blocks, 3.6).
#include "common.cuh"
#include "e4m3.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kAppThreads = 256, kAppWarps = kAppThreads / 32;
constexpr double kInvTwoPi = 0.15915494309189533577;

struct AppendParams {
  const __nv_bfloat16* in;       // [S * T][width]
  __nv_bfloat16* q_out;          // rows q_stride apart, or null
  uint8_t* k_cache;
  uint8_t* v_cache;
  float* scales;                 // [n_pages][kv][page / 16][2]
  const double* inv_freq;
  const int32_t *page_table, *kv_len, *seen, *new_begin, *new_len, *kv_count;
  long long q_stride, page_stride;
  int T, heads, kv, width, rot, half;
  int n_seqs, rows_per_seq, per_seq, per_subnet;      // CTAs of a sequence (padded rows) / of a subnet
  int page_shift, n_pages, max_pages;
  int* status;
};

// What a CTA appends: `count` rows from row `row` of [S * T] on to the slots first .. of the block that begins at slot in_page of
// the page; the first is at position `pos` of its sequence.  held: KV positions to write.
struct Run {
  long long row, page;
  int count, first, in_page, pos, held;
};

__device__ inline void report(const AppendParams& p, bool mine) {
  if (mine) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
}

// Blocks that the n new tokens at the end of `len` slots span; 0 if the sequence's numbers contradict each other.
__device__ inline int blocks_of(const AppendParams& p, int n, int len, int seen, bool& bad) {
  bad = n > 0 && (len < n || (long long)len > ((long long)p.max_pages << p.page_shift) || seen < len);
  return n <= 0 || bad ? 0 : (((len - n) & 15) + n + 15) >> 4;
}

// One warp.  count == 0: nothing to do.
__device__ inline Run find_run(const AppendParams& p, int lane) {
  Run r;
  r.count = 0;
  const int s = blockIdx.x / p.per_subnet;
  int j = blockIdx.x - s * p.per_subnet, b, n, len, seen, begin;
  const int32_t* lens = p.kv_len + (long long)s * p.n_seqs;
  const int32_t* seens = p.seen ? p.seen + (long long)s * p.n_seqs : lens;
  const int held = p.kv_count ? p.kv_count[s] : p.kv;
  if (p.new_begin) {
    // the sequence in whose blocks number j falls: lanes take sequences, a running sum over them
    const int32_t* nb = p.new_begin + (long long)s * (p.n_seqs + 1);
    int before = 0;
    bool found = false, broken = false;
    b = n = len = seen = begin = 0;
    for (int k0 = 0; k0 < p.n_seqs; k0 += 32) {
      const int k = k0 + lane;
      int x = 0, y = 0, l = 0, sn = 0, blocks = 0;
      if (k < p.n_seqs) {
        x = nb[k]; y = nb[k + 1]; l = lens[k]; sn = seens[k];
        if (x < 0 || y < x || y > p.T) {
          broken = true;
        } else {
          bool bad;
          blocks = blocks_of(p, y - x, l, sn, bad);
          report(p, bad);
        }
      }
      int upto = blocks;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const int from = before + upto - blocks;
      const unsigned hit = __ballot_sync(0xffffffffu, j >= from && j < from + blocks);
      if (hit && !found) {
        const int at = __ffs(hit) - 1;
        found = true;
        b = k0 + at;
        begin = __shfl_sync(0xffffffffu, x, at);
        n = __shfl_sync(0xffffffffu, y, at) - begin;
        len = __shfl_sync(0xffffffffu, l, at);
        seen = __shfl_sync(0xffffffffu, sn, at);
        j -= __shfl_sync(0xffffffffu, from, at);
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (__any_sync(0xffffffffu, broken)) {            // not ascending, or rows that the call does not have
      report(p, lane == 0);
      return r;
    }
    if (!found) return r;
  } else {
    b = j / p.per_seq;
    j -= b * p.per_seq;
    begin = b * p.rows_per_seq;
    n = p.new_len ? p.new_len[(long long)s * p.n_seqs + b] : p.rows_per_seq;
    len = lens[b];
    seen = seens[b];
    bool bad = n < 0 || n > p.rows_per_seq, bad2 = false;
    if (!bad && j >= blocks_of(p, n, len, seen, bad2)) {
      report(p, bad2 && lane == 0);
      return r;
    }
    if (bad) {
      report(p, lane == 0);
      return r;
    }
  }
  const int slot0 = len - n, block0 = ((slot0 >> 4) + j) << 4;
  const int page = p.page_table[((long long)s * p.n_seqs + b) * p.max_pages + (block0 >> p.page_shift)];
  if ((unsigned)page >= (unsigned)p.n_pages) {
    report(p, lane == 0);
    return r;
  }
  r.first = max(slot0 - block0, 0);
  const int i = max(block0 - slot0, 0);               // the first token's number among the new ones
  r.count = min(16 - r.first, n - i);
  r.row = (long long)s * p.T + begin + i;
  r.pos = seen - n + i;
  r.held = max(0, min(p.kv, held));
  r.page = page;
  r.in_page = block0 & ((1 << p.page_shift) - 1);
  return r;
}

__device__ inline float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ inline float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ inline void spread(float (&x)[8], const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf_lo(w[i]); x[2 * i + 1] = bf_hi(w[i]); }
}

enum { MODE_HALF = 0, MODE_PAIRS = 1, MODE_SLOW_HALF = 2, MODE_SLOW_PAIRS = 3 };

// 16 rows of a head: lane's item i is the eight elements from 8 * c on of row r, c = (32 i + lane) % (D / 8).
template <int D>
struct Rows {
  static constexpr int CHUNKS = D / 8, ITEMS = D / 16;
};

// Where a row's table of (cos, sin) has pair j.  Lanes that own neighbouring chunks of a head read 16 bytes (two pairs) each at a
// time: those lie next to each other.
template <int MODE>
__device__ inline int pair_at(int j, int half) {
  if constexpr (MODE == MODE_HALF || MODE == MODE_PAIRS) {
    constexpr int PER = MODE == MODE_HALF ? 8 : 4;    // pairs of a chunk
    return 2 * (j % PER / 2 * (half / PER) + j / PER) + j % 2;
  }
  return j;
}

// Eight elements of row r's head, rotated where the head is: `own` holds them.  other: the eight that they are paired with, half a
// rotation away (MODE_HALF).
template <int MODE>
__device__ inline void rotate(float (&x)[8], const AppendParams& p, const uint4& own, const uint4& other, const __nv_bfloat16* row, const float2* cs, int c) {
  spread(x, own);
  if (8 * c >= p.rot) return;
  if constexpr (MODE == MODE_HALF) {
    float z[8];
    spread(z, other);
    const bool low = 8 * c < p.half;
    const float4* at = reinterpret_cast<const float4*>(cs) + (low ? c : c - p.half / 8);
    const float sign = low ? -1.f : 1.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float4 a = at[e / 2 * (p.half / 8)];      // (cos, sin) of two pairs
      x[e] = fmaf(sign * z[e], a.y, x[e] * a.x);
      x[e + 1] = fmaf(sign * z[e + 1], a.w, x[e + 1] * a.z);
    }
  } else if constexpr (MODE == MODE_PAIRS) {
    const float4* at = reinterpret_cast<const float4*>(cs) + c;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 a = at[e / 4 * (p.half / 4)];
      const float u = x[e], v = x[e + 1], y = x[e + 2], z = x[e + 3];
      x[e] = u * a.x - v * a.y;
      x[e + 1] = u * a.y + v * a.x;
      x[e + 2] = y * a.z - z * a.w;
      x[e + 3] = y * a.w + z * a.z;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int el = 8 * c + e;
      if (el < p.rot) {
        const bool low = MODE == MODE_SLOW_HALF ? el < p.half : el % 2 == 0;
        const int pair = MODE == MODE_SLOW_HALF ? (low ? el : el - p.half) : el / 2;
        const int mate = MODE == MODE_SLOW_HALF ? (low ? el + p.half : el - p.half) : el ^ 1;
        const float z = __bfloat162float(row[mate]);
        const float2 a = cs[pair];
        x[e] = low ? x[e] * a.x - z * a.y : z * a.y + x[e] * a.x;
      }
    }
  }
}

__device__ inline uint4 pack_bf16x8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight values as numbers.  FINITE: all of them are.
template <bool FINITE>
__device__ inline uint2 numbers(const float (&x)[8], float inv) {
  if constexpr (FINITE) {
    return make_uint2(narrow4_finite(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), narrow4_finite(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
  } else {
    return make_uint2(narrow4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), narrow4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
  }
}
constexpr uint32_t kInfinity = 0x7f800000u;

// The scale of a block from the largest magnitude of its new tokens, and the tokens that it holds rounded to it.  `lanes` lanes
// take part, this one is number `lane` of them.
template <int D>
__device__ inline float rescale(uint8_t* cache, float* scale, float old, float top, int first, int lane, int lanes) {
  const float now = fmaxf(scale_for(top), scale_above(old));
  if (first > 0 && now != old) {
    const float f = old * inverse_scale(now);
    for (int k = lane; k < first * D / 8; k += lanes) {
      uint2* at = reinterpret_cast<uint2*>(cache) + k;
      const uint2 v = *at;
      uint32_t w[2] = {v.x, v.y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float a[4];
        widen4(a, w[i]);
        w[i] = narrow4(a[0] * f, a[1] * f, a[2] * f, a[3] * f);
      }
      *at = make_uint2(w[0], w[1]);
    }
  }
  if (lane == 0) *scale = now;
  return now;
}

// Positions first .. of `count` rows as (cos, sin).
template <int MODE>
__device__ inline void fill_table(const AppendParams& p, float2* table, int pos, int count) {
  for (int k = threadIdx.x; k < count * p.half; k += blockDim.x) {
    const int r = k / p.half, j = k - r * p.half;
    double turns = (double)(pos + r) * (p.inv_freq[j] * kInvTwoPi);
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    table[r * p.half + pair_at<MODE>(j, p.half)] = make_float2(c, s);
  }
}

template <int D, int MODE>
__global__ void __launch_bounds__(kAppThreads, D == 128 ? 2 : 3) append_q8_kernel(const AppendParams p) {
  using R = Rows<D>;
  __shared__ Run shared;
  extern __shared__ __align__(16) float2 table[];     // [16][half]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  griddep_launch_dependents();
  griddep_wait();
  if (warp == 0) {
    const Run r = find_run(p, lane);
    if (lane == 0) shared = r;
  }
  __syncthreads();
  const Run run = shared;
  if (run.count == 0) return;
  const __nv_bfloat16* rows = p.in + run.row * p.width;
  const int units = 2 * p.kv + (p.q_out ? p.heads : 0);
  // heads in the order K, V, Q; the first one's rows travel while the table is filled, the next one's while one is worked on
  auto column = [&](int u) { return (u < 2 * p.kv ? p.heads + u : u - 2 * p.kv) * D; };
  auto load = [&](uint4 (&own)[R::ITEMS], int u) {
#pragma unroll
    for (int i = 0; i < R::ITEMS; ++i) {
      const int k = 32 * i + lane, r = k / R::CHUNKS, c = k % R::CHUNKS;
      own[i] = make_uint4(0, 0, 0, 0);
      if (r < run.count) own[i] = *reinterpret_cast<const uint4*>(rows + (r * p.width + column(u) + 8 * c));
    }
  };
  uint4 own[R::ITEMS];
  if (warp < units) load(own, warp);
  fill_table<MODE>(p, table, run.pos, run.count);
  __syncthreads();
#pragma unroll 1
  for (int u = warp; u < units; u += kAppWarps) {
    uint4 next[R::ITEMS];
    const bool is_q = u >= 2 * p.kv, is_k = u < p.kv;
    const int group = is_q ? -1 : (is_k ? u : u - p.kv);
    if (u + kAppWarps < units) load(next, u + kAppWarps);
    // the eight elements that an item is paired with: another lane has them
    auto paired = [&](const uint4& v) {
      if constexpr (MODE != MODE_HALF) return v;
      const int c = lane % R::CHUNKS, hop = p.half / 8, from = 8 * c >= p.rot ? lane : (c < hop ? lane + hop : lane - hop);
      return make_uint4(__shfl_sync(0xffffffffu, v.x, from), __shfl_sync(0xffffffffu, v.y, from), __shfl_sync(0xffffffffu, v.z, from),
                        __shfl_sync(0xffffffffu, v.w, from));
    };
    if (is_q) {
      __nv_bfloat16* out = p.q_out + run.row * p.q_stride + (u - 2 * p.kv) * D;
      if (MODE == MODE_SLOW_HALF || MODE == MODE_SLOW_PAIRS) {
        uint4 y[R::ITEMS];                            // reads its rows once more
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS, c = k % R::CHUNKS;
          float x[8];
          if (r < run.count) {
            rotate<MODE>(x, p, own[i], own[i], rows + r * p.width + column(u), table + r * p.half, c);
            y[i] = pack_bf16x8(x);
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS, c = k % R::CHUNKS;
          if (r < run.count) *reinterpret_cast<uint4*>(out + r * p.q_stride + 8 * c) = y[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS, c = k % R::CHUNKS;
          float x[8];
          const uint4 other = paired(own[i]);
          if (r < run.count) {
            rotate<MODE>(x, p, own[i], other, nullptr, table + r * p.half, c);
            *reinterpret_cast<uint4*>(out + r * p.q_stride + 8 * c) = pack_bf16x8(x);
          }
        }
      }
    } else if (group < run.held) {
      uint8_t* cache = (is_k ? p.k_cache : p.v_cache) + run.page * p.page_stride + (((long long)group << p.page_shift) + run.in_page) * D;
      float* scale = p.scales + 2 * (((run.page * p.kv + group) << (p.page_shift - 4)) + (run.in_page >> 4)) + !is_k;
      const float old = run.first > 0 ? *scale : 0.f;
      uint8_t* to = cache + run.first * D;
      if (is_k) {
        float x[R::ITEMS][8];
        uint32_t top = 0;                             // of the magnitudes' bits, which order as the magnitudes do
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS, c = k % R::CHUNKS;
          const uint4 other = paired(own[i]);
          if (r < run.count) rotate<MODE>(x[i], p, own[i], other, rows + r * p.width + column(u), table + r * p.half, c);
          else spread(x[i], own[i]);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7fffffffu);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        const bool finite = top < kInfinity;
        if (!finite) {                                // once more without what is not
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < R::ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[i][e]) < INFINITY ? fabsf(x[i][e]) : 0.f);
          top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
        }
        const float inv = inverse_scale(rescale<D>(cache, scale, old, __uint_as_float(top), run.first, lane, 32));
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS;
          if (r < run.count) *reinterpret_cast<uint2*>(to + 8 * k) = finite ? numbers<true>(x[i], inv) : numbers<false>(x[i], inv);
        }
      } else {
        uint32_t both = 0;                            // two bf16 magnitudes
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          both = __vmaxu2(both, own[i].x & 0x7fff7fffu);
          both = __vmaxu2(both, own[i].y & 0x7fff7fffu);
          both = __vmaxu2(both, own[i].z & 0x7fff7fffu);
          both = __vmaxu2(both, own[i].w & 0x7fff7fffu);
        }
        uint32_t top = __reduce_max_sync(0xffffffffu, max(both << 16, both & 0xffff0000u));
        const bool finite = top < kInfinity;
        if (!finite) {
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < R::ITEMS; ++i) {
            float x[8];
            spread(x, own[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.f);
          }
          top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
        }
        const float inv = inverse_scale(rescale<D>(cache, scale, old, __uint_as_float(top), run.first, lane, 32));
#pragma unroll
        for (int i = 0; i < R::ITEMS; ++i) {
          const int k = 32 * i + lane, r = k / R::CHUNKS;
          float x[8];
          spread(x, own[i]);
          if (r < run.count) *reinterpret_cast<uint2*>(to + 8 * k) = finite ? numbers<true>(x, inv) : numbers<false>(x, inv);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < R::ITEMS; ++i) own[i] = next[i];
  }
}

// One token of every sequence: a CTA a token, D / 8 lanes a head, all heads at once.  Everything that does not hang on the page
// -- the row, the frequencies, the lengths -- is read in one round trip.
template <int D, int MODE>
__global__ void __launch_bounds__(kAppThreads) append_one_q8_kernel(const AppendParams p) {
  constexpr int LANES = D / 8, HEADS = 32 / LANES;    // of a head; of a warp
  __shared__ __align__(16) float2 table[D / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % LANES;
  const int seq = blockIdx.x, s = seq / p.n_seqs, warps = blockDim.x >> 5;
  griddep_launch_dependents();
  griddep_wait();
  const __nv_bfloat16* row = p.in + (long long)seq * p.width;
  const int units = 2 * p.kv + (p.q_out ? p.heads : 0);
  auto column = [&](int u) { return (u < 2 * p.kv ? p.heads + u : u - 2 * p.kv) * D; };
  int u = warp * HEADS + lane / LANES;
  uint4 own = make_uint4(0, 0, 0, 0);
  if (u < units) own = *reinterpret_cast<const uint4*>(row + column(u) + 8 * c);
  const int n = p.new_len ? p.new_len[seq] : 1, len = p.kv_len[seq], seen = p.seen ? p.seen[seq] : len;
  const int held = p.kv_count ? max(0, min(p.kv, p.kv_count[s])) : p.kv;
  bool bad = false;
  if (n < 0 || n > 1) bad = true;
  else if (blocks_of(p, n, len, seen, bad) == 0 && !bad) return;     // no new token
  if (bad) {
    report(p, threadIdx.x == 0);
    return;
  }
  const int slot = len - 1, first = slot & 15;
  const int page = p.page_table[(long long)seq * p.max_pages + (slot >> p.page_shift)];
  fill_table<MODE>(p, table, seen - 1, 1);
  __syncthreads();
  if ((unsigned)page >= (unsigned)p.n_pages) {
    report(p, threadIdx.x == 0);
    return;
  }
  const int in_page = slot & ((1 << p.page_shift) - 1) & ~15;
#pragma unroll 1
  for (; __any_sync(0xffffffffu, u < units); u += warps * HEADS) {
    const bool live = u < units, is_q = u >= 2 * p.kv, is_k = u < p.kv;
    const int group = is_k ? u : u - p.kv;
    const __nv_bfloat16* head = row + (live ? column(u) : 0);
    uint4 other = own;
    if constexpr (MODE == MODE_HALF) {
      const int hop = p.half / 8, from = 8 * c >= p.rot ? lane : (c < hop ? lane + hop : lane - hop);
      other = make_uint4(__shfl_sync(0xffffffffu, own.x, from), __shfl_sync(0xffffffffu, own.y, from), __shfl_sync(0xffffffffu, own.z, from),
                         __shfl_sync(0xffffffffu, own.w, from));
    }
    const bool stores = live && !is_q && group < held;
    float* scale = nullptr;
    uint8_t* cache = nullptr;
    float old = 0.f;
    if (stores) {
      cache = (is_k ? p.k_cache : p.v_cache) + page * p.page_stride + (((long long)group << p.page_shift) + in_page) * D;
      scale = p.scales + 2 * ((((long long)page * p.kv + group) << (p.page_shift - 4)) + (in_page >> 4)) + !is_k;
      if (first > 0) old = *scale;
    }
    float x[8];
    if (live && (is_q || is_k)) rotate<MODE>(x, p, own, other, head, table, c);
    else spread(x, own);
    __syncwarp();                                     // the head has been read: now it may be written
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.f);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (live && is_q) {
      *reinterpret_cast<uint4*>(p.q_out + (long long)seq * p.q_stride + (u - 2 * p.kv) * D + 8 * c) = pack_bf16x8(x);
    } else if (stores) {
      const float inv = inverse_scale(rescale<D>(cache, scale, old, top, first, c, LANES));
      *reinterpret_cast<uint2*>(cache + first * D + 8 * c) = numbers<false>(x, inv);
    }
    const int next = u + warps * HEADS;
    if (next < units) own = *reinterpret_cast<const uint4*>(row + column(next) + 8 * c);
  }
}

template <int D>
int launch(const AppendParams& p, int S, int layout, cudaStream_t st) {
  int mode;
  if (layout == TWIST_ROPE_HALF) mode = p.half % 8 == 0 ? MODE_HALF : MODE_SLOW_HALF;
  else mode = p.rot % 8 == 0 ? MODE_PAIRS : MODE_SLOW_PAIRS;
  if (p.rot == 0) mode = MODE_PAIRS;
  if (!p.new_begin && p.rows_per_seq == 1) {
    // as many warps as take all heads at once, if a CTA may have them
    const int units = 2 * p.kv + (p.q_out ? p.heads : 0), heads = 256 / D, warps = (units + heads - 1) / heads;
    void (*kernel)(AppendParams) = mode == MODE_HALF ? append_one_q8_kernel<D, MODE_HALF>
                                   : mode == MODE_PAIRS ? append_one_q8_kernel<D, MODE_PAIRS>
                                   : mode == MODE_SLOW_HALF ? append_one_q8_kernel<D, MODE_SLOW_HALF>
                                                            : append_one_q8_kernel<D, MODE_SLOW_PAIRS>;
    TWIST_CUDA_TRY(launch_overlapped(kernel, dim3((unsigned)(S * p.n_seqs)), dim3(32 * (warps < kAppWarps ? warps : kAppWarps)), 0, st, 1, p));
    return TWIST_OK;
  }
  const long long grid = (long long)S * p.per_subnet;
  if (grid > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  void (*kernel)(AppendParams) = mode == MODE_HALF ? append_q8_kernel<D, MODE_HALF>
                                 : mode == MODE_PAIRS ? append_q8_kernel<D, MODE_PAIRS>
                                 : mode == MODE_SLOW_HALF ? append_q8_kernel<D, MODE_SLOW_HALF>
                                                          : append_q8_kernel<D, MODE_SLOW_PAIRS>;
  TWIST_CUDA_TRY(launch_overlapped(kernel, dim3((unsigned)grid), dim3(kAppThreads), 16 * p.half * sizeof(float2), st, 1, p));
  return TWIST_OK;
}

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" int32_t twist_kv_append_q8(const twist_kv_append_q8_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->tokens <= 0 || a->head_keep <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 ||
      a->max_pages <= 0 || a->page_size <= 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if (dh != 16 && dh != 32 && dh != 64 && dh != 128) return TWIST_ERR_UNSUPPORTED;
  if (a->rot_dims < 0 || a->rot_dims > dh || a->rot_dims % 2 != 0) return TWIST_ERR_SHAPE;
  if (a->layout != TWIST_ROPE_HALF && a->layout != TWIST_ROPE_PAIRS) return TWIST_ERR_SHAPE;
  const long long width = ((long long)a->head_keep + 2ll * a->kv_max) * dh, a_sub = (long long)a->head_keep * dh;
  if (width > (1 << 24)) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll - 1024) return TWIST_ERR_UNSUPPORTED;      // positions are 32-bit
  if (a->page_stride % 16 != 0 || a->page_stride < (long long)a->kv_max * a->page_size * dh) return TWIST_ERR_SHAPE;
  if (!a->new_begin && a->tokens % a->n_seqs != 0) return TWIST_ERR_SHAPE;
  if (a->new_begin && a->new_len) return TWIST_ERR_SHAPE;
  if (a->q_out && (a->q_stride % 8 != 0 || a->q_stride < a_sub)) return TWIST_ERR_SHAPE;
  if (!a->qkv || !a->k_cache || !a->v_cache || !a->scales || !a->page_table || !a->kv_len || (a->rot_dims > 0 && !a->inv_freq)) return TWIST_ERR_NULL;
  if (!aligned16(a->qkv) || !aligned16(a->q_out) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->scales) ||
      (reinterpret_cast<uintptr_t>(a->inv_freq) & 7))
    return TWIST_ERR_SHAPE;
  AppendParams p;
  memset(&p, 0, sizeof(p));
  const long long rows = (long long)a->n_subnets * a->tokens;
  if (rows > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  if (a->q_out && !(a->q_out == a->qkv && (a->q_stride == width || rows == 1)) &&
      overlap(a->qkv, rows * width * 2, a->q_out, ((rows - 1) * a->q_stride + a_sub) * 2))
    return TWIST_ERR_SHAPE;
  p.in = static_cast<const __nv_bfloat16*>(a->qkv);
  p.q_out = static_cast<__nv_bfloat16*>(a->q_out);
  p.k_cache = static_cast<uint8_t*>(a->k_cache);
  p.v_cache = static_cast<uint8_t*>(a->v_cache);
  p.scales = a->scales;
  p.inv_freq = a->inv_freq;
  p.page_table = a->page_table; p.kv_len = a->kv_len; p.seen = a->seen;
  p.new_begin = a->new_begin; p.new_len = a->new_len; p.kv_count = a->kv_count;
  p.q_stride = a->q_stride; p.page_stride = a->page_stride;
  p.T = a->tokens; p.heads = a->head_keep; p.kv = a->kv_max; p.width = (int)width;
  p.rot = a->rot_dims; p.half = a->rot_dims / 2;
  p.n_seqs = a->n_seqs;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages;
  // Blocks that n tokens can span: (n + 14) / 16 + 1.  Packed rows: as many as all sequences together can.
  if (a->new_begin) {
    p.rows_per_seq = p.per_seq = 1;
    const long long n = (long long)a->tokens / 16 + 2ll * (a->n_seqs < a->tokens ? a->n_seqs : a->tokens) + 1;
    if (n > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
    p.per_subnet = (int)n;
  } else {
    p.rows_per_seq = a->tokens / a->n_seqs;
    p.per_seq = (p.rows_per_seq + 14) / 16 + 1;
    if ((long long)p.per_seq * a->n_seqs > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
    p.per_subnet = p.per_seq * a->n_seqs;
  }
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dh) {
    case 16: return launch<16>(p, a->n_subnets, a->layout, st);
    case 32: return launch<32>(p, a->n_subnets, a->layout, st);
    case 64: return launch<64>(p, a->n_subnets, a->layout, st);
    default: return launch<128>(p, a->n_subnets, a->layout, st);
  }
}
