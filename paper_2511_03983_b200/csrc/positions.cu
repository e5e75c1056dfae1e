// twist_rope_fwd / twist_rope_bwd: rotation of the Q and K columns of projected activations by the token's position, and
// twist_kv_append: the same rotation on the way of new K and V rows into a paged cache.
//
// Per pair of a head: (x, y) <- (x cos a - y sin a, x sin a + y cos a), a = position * inv_freq[j].  The work is moving
// bytes: 4 per element (2 read, 2 written) against 3 operations per element, so both are HBM-bound for long inputs and
// latency-bound for the rows of one decoding step.
//
// Angles.  A CTA takes a tile of token rows and first fills a table [row][pair] of (cos, sin) in shared memory, one
// evaluation per (token, pair) instead of one per (token, head, pair).  position * inv_freq is formed in 64 bits and
// reduced to a fraction of a turn there: at position 10^6 an fp32 product would be off by 0.06 rad.  The fraction, at
// most half a turn, is exact to 2^-25 in fp32, and sincospif takes it from there.
//
// Bytes in flight and instructions.  A thread takes a unit (below) in several rows at once: the index arithmetic of a unit
// is done once for them and their loads are in flight together.  Rotating, a thread holds 128 bytes and issues its first
// loads before the CTA finds positions and angles, on which they do not depend.  Appending, finding a row's place costs
// two dependent round trips, and rows of no sequence are not read: the places come first and more, lighter CTAs share an
// SM to cover them (44 000 packed rows of 4.6 KB: 134 us loads first, 4 CTAs an SM; 116 us places first, 6 CTAs; 5 CTAs
// and fewer spilled registers: 122).
//
// Rotation.  A thread's unit of work owns both elements of every pair it rotates, so rotating in place is safe without
// any ordering between threads: a unit is two 16-byte chunks half a rotation apart in the HALF layout, one chunk in the
// PAIRS layout and in what is not rotated (appending, two neighbours where they come in twos: 116 -> 113 us in the case
// above; rotating, twice the rows in flight are worth more: 190 us against 194); where chunks would straddle the halves
// (rot_dims/2 or rot_dims not a multiple of 8) a unit is a whole head, element by element.
#include "common.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kPosThreads = 256;
constexpr int kMaxRows = 8;            // token rows of a tile
constexpr int kMaxHead = 256;
constexpr double kInvTwoPi = 0.15915494309189533577;

__device__ inline float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ inline float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ inline uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&t);
}

// n / d by a multiplication where that is exact (n (d - 1) < 2^32 for every n that occurs).
struct Divisor {
  uint32_t d, m;
  __device__ uint32_t divide(uint32_t n) const { return m ? __umulhi(n, m) : n / d; }
};
Divisor divisor(uint32_t d, uint64_t max_n) {
  const bool exact = d > 1 && max_n * (d - 1) < (1ull << 32);
  return {d, exact ? (uint32_t)(((1ull << 32) + d - 1) / d) : 0u};
}

struct PosParams {
  const __nv_bfloat16* in;       // [rows][width]
  __nv_bfloat16* out;            // rope: [rows][width]; append: Q rows, q_stride apart (may be null)
  const double* inv_freq;
  const int32_t* pos;            // rope: [rows] or null
  long long rows;                // S * T
  long long q_stride;
  int T, seq_len, heads, kv, dh, width;
  int rot, half;                 // half = rot / 2
  int tile_rows;
  int units_per_head, first_unit, head_units, row_units;    // a row's units: those of its heads, then those of V
  int wide;                      // appending: units that are not half a rotation apart are two neighbouring chunks, not one
  Divisor by_units, by_head, by_half, by_chunks;
  float sign;
  int in_place;
  // append
  __nv_bfloat16* k_cache;
  __nv_bfloat16* v_cache;
  const int32_t *page_table, *kv_len, *new_begin, *new_len, *kv_count;
  int n_seqs, rows_per_seq, page_shift, n_pages, max_pages;
  long long page_stride;
  int* status;
};

struct RowInfo {
  long long cache;     // append: element offset of the row's slot in position 0 of its page
  int pos, valid, held;
};

// Append: which token of which sequence row (s, t) is, and where it goes.  One warp per row; two round trips: the
// sequences' first rows and lengths (every lane keeps the last sequence of its that begins at or before t), the page.
__device__ inline RowInfo find_row(const PosParams& p, long long r, int lane) {
  RowInfo ri;
  ri.valid = 0; ri.pos = 0; ri.cache = 0; ri.held = -1;
  const int s = (int)(r / p.T), t = (int)(r - (long long)s * p.T);
  const int32_t* lens = p.kv_len + (long long)s * p.n_seqs;
  const int held = p.kv_count ? p.kv_count[s] : p.kv;
  int b, i, n, len;
  if (p.new_begin) {
    const int32_t* nb = p.new_begin + (long long)s * (p.n_seqs + 1);
    int at = -1, begin = 0, end = 0, count = 0;
    len = 0;
    for (int k = lane; k < p.n_seqs; k += 32) {
      const int x = nb[k], y = nb[k + 1], l = lens[k];
      if (x <= t) { at = k; begin = x; end = y; len = l; ++count; }
    }
    b = __reduce_max_sync(0xffffffffu, at);
    count = __reduce_add_sync(0xffffffffu, count);
    if (b < 0) return ri;                             // a row before the first sequence
    begin = __shfl_sync(0xffffffffu, begin, b & 31);
    end = __shfl_sync(0xffffffffu, end, b & 31);
    len = __shfl_sync(0xffffffffu, len, b & 31);
    if (count != b + 1 || begin < 0 || end > p.T) {   // not ascending, or rows that the call does not have
      if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
      return ri;
    }
    if (t >= end) return ri;                          // a row behind the last sequence
    i = t - begin;
    n = end - begin;
  } else {
    b = t / p.rows_per_seq;
    i = t - b * p.rows_per_seq;
    len = lens[b];
    n = p.new_len ? p.new_len[(long long)s * p.n_seqs + b] : p.rows_per_seq;
    if (n < 0 || n > p.rows_per_seq) {
      if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
      return ri;
    }
    if (i >= n) return ri;
  }
  const long long pos = (long long)len - n + i, page_slot = pos >> p.page_shift;
  int page = -1;
  if (pos >= 0 && page_slot < p.max_pages) page = p.page_table[((long long)s * p.n_seqs + b) * p.max_pages + page_slot];
  if ((unsigned)page >= (unsigned)p.n_pages) {
    if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
    return ri;
  }
  ri.valid = 1;
  ri.pos = (int)pos;
  ri.cache = page * p.page_stride + (pos & ((1 << p.page_shift) - 1)) * p.dh;
  ri.held = max(0, min(p.kv, held));
  return ri;
}

__device__ inline void rotate8(uint4& lo, uint4& hi, const float2* cs) {
  uint32_t* a = reinterpret_cast<uint32_t*>(&lo);
  uint32_t* b = reinterpret_cast<uint32_t*>(&hi);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 c0 = cs[2 * w], c1 = cs[2 * w + 1];
    const float x0 = bf_lo(a[w]), x1 = bf_hi(a[w]), y0 = bf_lo(b[w]), y1 = bf_hi(b[w]);
    a[w] = pack2(x0 * c0.x - y0 * c0.y, x1 * c1.x - y1 * c1.y);
    b[w] = pack2(x0 * c0.y + y0 * c0.x, x1 * c1.y + y1 * c1.x);
  }
}
__device__ inline void rotate_pairs(uint4& v, const float2* cs) {
  uint32_t* a = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 c = cs[w];
    const float x = bf_lo(a[w]), y = bf_hi(a[w]);
    a[w] = pack2(x * c.x - y * c.y, x * c.y + y * c.x);
  }
}

enum { MODE_HALF = 0, MODE_PAIRS = 1, MODE_SLOW_HALF = 2, MODE_SLOW_PAIRS = 3 };

// Rows that a thread has in flight (see above).
__host__ __device__ constexpr int batch_rows(bool append, int mode) { return append ? 2 : (mode == MODE_PAIRS ? 8 : 4); }

// Positions (and, appending, destinations) of the tile's rows, then their (cos, sin) table.
template <bool APPEND>
__device__ inline void fill_table(const PosParams& p, float2* table, RowInfo* info, long long row0, int n_rows) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if constexpr (APPEND) {
    for (int r = warp; r < n_rows; r += kPosThreads / 32) {
      const RowInfo ri = find_row(p, row0 + r, lane);
      if (lane == 0) info[r] = ri;
    }
  } else if (threadIdx.x < n_rows) {
    const long long r = row0 + threadIdx.x;
    info[threadIdx.x].pos = p.pos ? p.pos[r] : (int)((r % p.T) % p.seq_len);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < n_rows * p.half; k += kPosThreads) {
    const int r = (int)p.by_half.divide(k), j = k - r * p.half;
    double turns = (double)info[r].pos * (p.inv_freq[j] * kInvTwoPi);
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    table[k] = make_float2(c, p.sign * s);
  }
  __syncthreads();
}

template <bool APPEND, int MODE>
__global__ void __launch_bounds__(kPosThreads, APPEND ? 6 : 4) rotate_rows_kernel(PosParams p) {
  extern __shared__ float2 table[];                 // [tile_rows][half]
  __shared__ RowInfo info[kMaxRows];
  constexpr bool SLOW = MODE == MODE_SLOW_HALF || MODE == MODE_SLOW_PAIRS;
  constexpr int kBatch = batch_rows(APPEND, MODE);
  const long long row0 = (long long)blockIdx.x * p.tile_rows;
  const int n_rows = (int)min((long long)p.tile_rows, p.rows - row0), n_heads = p.heads + p.kv, pair_units = p.half / 8;
  // work item: unit k % row_units of the rows kBatch * (k / row_units) ...
  const uint32_t items = (uint32_t)((n_rows + kBatch - 1) / kBatch) * p.row_units;
  griddep_launch_dependents();
  griddep_wait();
  if (APPEND) fill_table<APPEND>(p, table, info, row0, n_rows);
  for (uint32_t k = threadIdx.x; k < items || (!APPEND && k == threadIdx.x); k += kPosThreads) {
    const int batch = (int)p.by_units.divide(k), u = (int)k - batch * p.row_units + p.first_unit;
    const int r0 = batch * kBatch, n = k < items ? min(kBatch, n_rows - r0) : 0;
    // unit j of head h, or of V (h = n_heads): elements at .. at + 7 of it, and (two) those `hop` further
    const int h = u < p.head_units ? (int)p.by_head.divide(u) : n_heads, j = u - (u < p.head_units ? h * p.units_per_head : p.head_units);
    const bool pair = MODE == MODE_HALF && h < n_heads && j < pair_units, two = pair || (APPEND && p.wide);
    const int hop = pair ? p.half : 8, step = APPEND && p.wide ? 16 : 8;
    const int at = pair ? 8 * j : (MODE == MODE_HALF && h < n_heads ? p.rot + step * (j - pair_units) : step * j);
    const __nv_bfloat16* src = p.in + (row0 + r0) * p.width + h * p.dh + at;
    uint4 lo[kBatch], hi[kBatch];
    if (!SLOW || h == n_heads) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (i < n && (!APPEND || info[r0 + i].valid)) {
          lo[i] = *reinterpret_cast<const uint4*>(src + (long long)i * p.width);
          if (two) hi[i] = *reinterpret_cast<const uint4*>(src + (long long)i * p.width + hop);
        }
      }
    }
    if (!APPEND && k == threadIdx.x) fill_table<APPEND>(p, table, info, row0, n_rows);
    // where the unit's rows go: a row's own place (q_stride / width apart) or its slot in the cache
    __nv_bfloat16* dst;
    int group = -1;                                 // appending: KV position of the unit, -1: Q
    if constexpr (APPEND) {
      if (h < p.heads) {
        dst = p.out + (row0 + r0) * p.q_stride + h * p.dh + at;
      } else if (h < n_heads) {
        group = h - p.heads;
        dst = p.k_cache + (((long long)group * p.dh) << p.page_shift) + at;
      } else {
        group = (int)p.by_chunks.divide(j);
        dst = p.v_cache + (((long long)group * p.dh) << p.page_shift) + (at - group * p.dh);
      }
    } else {
      dst = p.out + (row0 + r0) * p.width + h * p.dh + at;
    }
    const long long down = APPEND ? p.q_stride : p.width;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (i >= n) continue;
      const int r = r0 + i;
      __nv_bfloat16* to = dst + i * down;
      if constexpr (APPEND) {
        const RowInfo ri = info[r];
        if (group >= ri.held) continue;             // not held, or a row of no sequence (held = -1)
        if (group >= 0) to = dst + ri.cache;
        else if (!ri.valid) continue;
      }
      const float2* cs = table + r * p.half;
      if constexpr (SLOW) {
        if (h < n_heads) {
          const __nv_bfloat16* x = p.in + (row0 + r) * p.width + h * p.dh;
          for (int q = 0; q < p.half; ++q) {
            const int ix = MODE == MODE_SLOW_HALF ? q : 2 * q, iy = MODE == MODE_SLOW_HALF ? q + p.half : 2 * q + 1;
            const float a = __bfloat162float(x[ix]), b = __bfloat162float(x[iy]);
            const float2 c = cs[q];
            to[ix] = __float2bfloat16(a * c.x - b * c.y);
            to[iy] = __float2bfloat16(a * c.y + b * c.x);
          }
          for (int e = p.rot; e < p.dh; ++e) to[e] = x[e];
          continue;
        }
      }
      if (MODE == MODE_HALF && pair) {
        rotate8(lo[i], hi[i], cs + at);
      } else if (MODE == MODE_PAIRS && h < n_heads && at < p.rot) {
        rotate_pairs(lo[i], cs + at / 2);
        if (two) rotate_pairs(hi[i], cs + at / 2 + 4);
      }
      *reinterpret_cast<uint4*>(to) = lo[i];
      if (two) *reinterpret_cast<uint4*>(to + hop) = hi[i];
    }
  }
}

template <bool APPEND>
int launch(PosParams& p, int layout, cudaStream_t st) {
  int mode;
  if (layout == TWIST_ROPE_HALF) mode = p.half % 8 == 0 ? MODE_HALF : MODE_SLOW_HALF;
  else mode = p.rot % 8 == 0 ? MODE_PAIRS : MODE_SLOW_PAIRS;
  if (p.rot == 0) mode = MODE_PAIRS;                                                    // plain 16-byte chunks
  p.wide = APPEND && p.dh % 16 == 0 && (mode == MODE_HALF ? (p.dh - p.rot) % 16 == 0 : mode == MODE_PAIRS ? p.rot % 16 == 0 : true);
  const int step = p.wide ? 16 : 8;
  p.units_per_head = mode == MODE_HALF ? p.half / 8 + (p.dh - p.rot) / step : mode == MODE_PAIRS ? p.dh / step : 1;
  p.first_unit = APPEND && !p.out ? p.heads * p.units_per_head : 0;                     // Q is not wanted
  p.head_units = (p.heads + p.kv) * p.units_per_head;
  p.row_units = p.head_units - p.first_unit + (APPEND || !p.in_place ? p.kv * p.dh / step : 0);
  // Rows of a tile: as many as still give every SM several tiles.
  const long long want = p.rows / ((long long)sm_count() * 4);
  p.tile_rows = (int)(want < 1 ? 1 : (want > kMaxRows ? kMaxRows : want));
  const long long tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
  if (tiles > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  p.by_units = divisor((uint32_t)p.row_units, (uint64_t)((p.tile_rows + batch_rows(APPEND, mode) - 1) / batch_rows(APPEND, mode)) * p.row_units + kPosThreads);
  p.by_head = divisor((uint32_t)p.units_per_head, (uint64_t)p.head_units);
  p.by_half = divisor((uint32_t)(p.half > 0 ? p.half : 1), (uint64_t)p.tile_rows * p.half);
  p.by_chunks = divisor((uint32_t)(p.dh / step), (uint64_t)p.kv * p.dh / step);
  const size_t smem = (size_t)p.tile_rows * p.half * sizeof(float2);                    // at most 8 KB
  void (*kernel)(PosParams) = mode == MODE_HALF ? rotate_rows_kernel<APPEND, MODE_HALF>
                              : mode == MODE_PAIRS ? rotate_rows_kernel<APPEND, MODE_PAIRS>
                              : mode == MODE_SLOW_HALF ? rotate_rows_kernel<APPEND, MODE_SLOW_HALF>
                                                       : rotate_rows_kernel<APPEND, MODE_SLOW_PAIRS>;
  TWIST_CUDA_TRY(launch_overlapped(kernel, dim3((unsigned)tiles), dim3(kPosThreads), smem, st, 1, p));
  return TWIST_OK;
}

bool overlap(const void* a, long long a_bytes, const void* b, long long b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

int check_heads(int dtype, int S, int T, int heads, int kv, int dh, int rot, int layout) {
  if (dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (S <= 0 || T <= 0 || heads <= 0 || kv <= 0 || dh <= 0 || dh % 8 != 0 || rot < 0 || rot > dh || rot % 2 != 0) return TWIST_ERR_SHAPE;
  if (layout != TWIST_ROPE_HALF && layout != TWIST_ROPE_PAIRS) return TWIST_ERR_SHAPE;
  if (dh > kMaxHead || ((long long)heads + 2ll * kv) * dh > (1 << 24)) return TWIST_ERR_UNSUPPORTED;
  return TWIST_OK;
}

int rope(const twist_rope_args* a, float sign, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  int rc = check_heads(a->dtype, a->n_subnets, a->tokens, a->head_keep, a->kv_max, a->d_head, a->rot_dims, a->layout);
  if (rc != TWIST_OK) return rc;
  if (a->rot_dims < 2 || (!a->pos && a->seq_len <= 0)) return TWIST_ERR_SHAPE;
  if (!a->in || !a->out || !a->inv_freq) return TWIST_ERR_NULL;
  if (!aligned16(a->in) || !aligned16(a->out) || (reinterpret_cast<uintptr_t>(a->inv_freq) & 7)) return TWIST_ERR_SHAPE;
  PosParams p;
  memset(&p, 0, sizeof(p));
  p.in = static_cast<const __nv_bfloat16*>(a->in);
  p.out = static_cast<__nv_bfloat16*>(a->out);
  p.inv_freq = a->inv_freq; p.pos = a->pos;
  p.rows = (long long)a->n_subnets * a->tokens;
  p.T = a->tokens; p.seq_len = a->seq_len > 0 ? a->seq_len : 1;
  p.heads = a->head_keep; p.kv = a->kv_max; p.dh = a->d_head;
  p.width = (a->head_keep + 2 * a->kv_max) * a->d_head;
  p.rot = a->rot_dims; p.half = a->rot_dims / 2; p.sign = sign;
  p.in_place = a->in == a->out;
  const long long bytes = p.rows * p.width * 2;
  if (!p.in_place && overlap(a->in, bytes, a->out, bytes)) return TWIST_ERR_SHAPE;
  return launch<false>(p, a->layout, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" int32_t twist_rope_fwd(const twist_rope_args* a, void* stream) { return rope(a, 1.0f, stream); }
extern "C" int32_t twist_rope_bwd(const twist_rope_args* a, void* stream) { return rope(a, -1.0f, stream); }

extern "C" int32_t twist_kv_append(const twist_kv_append_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  int rc = check_heads(a->dtype, a->n_subnets, a->tokens, a->head_keep, a->kv_max, a->d_head, a->rot_dims, a->layout);
  if (rc != TWIST_OK) return rc;
  if (a->n_seqs <= 0 || a->n_pages <= 0 || a->max_pages <= 0 || a->page_size <= 0) return TWIST_ERR_SHAPE;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;      // positions are 32-bit
  if (a->page_stride % 8 != 0 || a->page_stride < (long long)a->kv_max * a->page_size * a->d_head) return TWIST_ERR_SHAPE;
  if (!a->new_begin && a->tokens % a->n_seqs != 0) return TWIST_ERR_SHAPE;
  if (a->new_begin && a->new_len) return TWIST_ERR_SHAPE;
  const long long width = ((long long)a->head_keep + 2 * a->kv_max) * a->d_head, a_sub = (long long)a->head_keep * a->d_head;
  if (a->q_out && (a->q_stride % 8 != 0 || a->q_stride < a_sub)) return TWIST_ERR_SHAPE;
  if (!a->qkv || !a->k_cache || !a->v_cache || !a->page_table || !a->kv_len || (a->rot_dims > 0 && !a->inv_freq)) return TWIST_ERR_NULL;
  if (!aligned16(a->qkv) || !aligned16(a->q_out) || !aligned16(a->k_cache) || !aligned16(a->v_cache) ||
      (reinterpret_cast<uintptr_t>(a->inv_freq) & 7))
    return TWIST_ERR_SHAPE;
  PosParams p;
  memset(&p, 0, sizeof(p));
  p.rows = (long long)a->n_subnets * a->tokens;
  if (a->q_out && !(a->q_out == a->qkv && (a->q_stride == width || p.rows == 1)) &&
      overlap(a->qkv, p.rows * width * 2, a->q_out, ((p.rows - 1) * a->q_stride + a_sub) * 2))
    return TWIST_ERR_SHAPE;
  p.in = static_cast<const __nv_bfloat16*>(a->qkv);
  p.out = static_cast<__nv_bfloat16*>(a->q_out);
  p.inv_freq = a->inv_freq;
  p.q_stride = a->q_stride;
  p.T = a->tokens; p.seq_len = 1;
  p.heads = a->head_keep; p.kv = a->kv_max; p.dh = a->d_head;
  p.width = (int)width;
  p.rot = a->rot_dims; p.half = a->rot_dims / 2; p.sign = 1.0f;
  p.k_cache = static_cast<__nv_bfloat16*>(a->k_cache);
  p.v_cache = static_cast<__nv_bfloat16*>(a->v_cache);
  p.page_table = a->page_table; p.kv_len = a->kv_len;
  p.new_begin = a->new_begin; p.new_len = a->new_len; p.kv_count = a->kv_count;
  p.n_seqs = a->n_seqs; p.rows_per_seq = a->new_begin ? 1 : a->tokens / a->n_seqs;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages; p.page_stride = a->page_stride;
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  return launch<true>(p, a->layout, static_cast<cudaStream_t>(stream));
}
