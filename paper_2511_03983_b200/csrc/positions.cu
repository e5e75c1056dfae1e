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
// Rotation.  A thread's unit of work owns both elements of every pair it rotates, so rotating in place is safe without
// any ordering between threads: in the HALF layout a unit is two 16-byte chunks half a rotation apart, in the PAIRS
// layout one 16-byte chunk; where chunks would straddle the halves (rot_dims/2 or rot_dims not a multiple of 8) a unit
// is a whole head, element by element.
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
  int units_per_head, head_units, chunk_units, row_units;   // rotated heads' units, then 8-element chunks of V
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

// Append: which token of which sequence row (s, t) is, and where it goes.  One warp per row (lane-parallel count of the
// sequences that begin at or before t).
__device__ inline RowInfo find_row(const PosParams& p, long long r, int lane) {
  RowInfo ri;
  ri.valid = 0; ri.pos = 0; ri.cache = 0; ri.held = 0;
  const int s = (int)(r / p.T), t = (int)(r - (long long)s * p.T);
  int b, i, n;
  if (p.new_begin) {
    const int32_t* nb = p.new_begin + (long long)s * (p.n_seqs + 1);
    int c = 0;                                        // sequences 1 .. n_seqs (n_seqs: the end) that begin at or before t
    for (int k = 1 + lane; k <= p.n_seqs; k += 32) c += nb[k] <= t;
    for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    b = c;
    if (b >= p.n_seqs || t < nb[0]) return ri;        // a row behind the last sequence (or before the first)
    i = t - nb[b];
    n = nb[b + 1] - nb[b];
    if (i < 0 || i >= n) {                            // not ascending
      if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
      return ri;
    }
  } else {
    b = t / p.rows_per_seq;
    i = t - b * p.rows_per_seq;
    n = p.new_len ? p.new_len[(long long)s * p.n_seqs + b] : p.rows_per_seq;
    if (n < 0 || n > p.rows_per_seq) {
      if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
      return ri;
    }
    if (i >= n) return ri;
  }
  const long long seq = (long long)s * p.n_seqs + b;
  const long long pos = (long long)p.kv_len[seq] - n + i;
  const long long page_slot = pos >> p.page_shift;
  int page = -1;
  if (pos >= 0 && page_slot < p.max_pages) page = p.page_table[seq * p.max_pages + page_slot];
  if ((unsigned)page >= (unsigned)p.n_pages) {
    if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
    return ri;
  }
  ri.valid = 1;
  ri.pos = (int)pos;
  ri.cache = page * p.page_stride + (pos & ((1 << p.page_shift) - 1)) * p.dh;
  ri.held = p.kv_count ? min(p.kv, p.kv_count[s]) : p.kv;
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

template <bool APPEND, int MODE>
__global__ void __launch_bounds__(kPosThreads) rotate_rows_kernel(PosParams p) {
  extern __shared__ float2 table[];                 // [tile_rows][half]
  __shared__ RowInfo info[kMaxRows];
  const long long row0 = (long long)blockIdx.x * p.tile_rows;
  const int n_rows = (int)min((long long)p.tile_rows, p.rows - row0);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  griddep_launch_dependents();
  griddep_wait();
  if constexpr (APPEND) {
    if (warp < n_rows) {
      const RowInfo ri = find_row(p, row0 + warp, lane);
      if (lane == 0) info[warp] = ri;
    }
  } else if (threadIdx.x < n_rows) {
    const long long r = row0 + threadIdx.x;
    info[threadIdx.x].pos = p.pos ? p.pos[r] : (int)((r % p.T) % p.seq_len);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < n_rows * p.half; k += kPosThreads) {
    const int r = k / p.half, j = k - r * p.half;
    double turns = (double)info[r].pos * (p.inv_freq[j] * kInvTwoPi);
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    table[k] = make_float2(c, p.sign * s);
  }
  __syncthreads();
  const int total = n_rows * p.row_units;
  for (int k = threadIdx.x; k < total; k += kPosThreads) {
    const int r = k / p.row_units;
    int u = k - r * p.row_units;
    if (APPEND && !info[r].valid) continue;
    const __nv_bfloat16* src = p.in + (row0 + r) * p.width;
    if (APPEND && !p.out) u += p.heads * p.units_per_head;        // Q is not wanted
    const float2* cs = table + r * p.half;
    if (u < p.head_units) {
      const int h = u / p.units_per_head, j = u - h * p.units_per_head;
      src += h * p.dh;
      __nv_bfloat16* dst;
      if constexpr (APPEND) {
        if (h < p.heads) {
          dst = p.out + (row0 + r) * p.q_stride + h * p.dh;
        } else {
          if (h - p.heads >= info[r].held) continue;
          dst = p.k_cache + info[r].cache + (((long long)(h - p.heads) * p.dh) << p.page_shift);
        }
      } else {
        dst = p.out + (row0 + r) * p.width + h * p.dh;
      }
      if constexpr (MODE == MODE_HALF) {
        const int pair_units = p.half / 8;
        if (j < pair_units) {
          uint4 lo = *reinterpret_cast<const uint4*>(src + 8 * j);
          uint4 hi = *reinterpret_cast<const uint4*>(src + p.half + 8 * j);
          rotate8(lo, hi, cs + 8 * j);
          *reinterpret_cast<uint4*>(dst + 8 * j) = lo;
          *reinterpret_cast<uint4*>(dst + p.half + 8 * j) = hi;
        } else {
          const int at = p.rot + 8 * (j - pair_units);
          *reinterpret_cast<uint4*>(dst + at) = *reinterpret_cast<const uint4*>(src + at);
        }
      } else if constexpr (MODE == MODE_PAIRS) {
        uint4 v = *reinterpret_cast<const uint4*>(src + 8 * j);
        if (8 * j < p.rot) rotate_pairs(v, cs + 4 * j);
        *reinterpret_cast<uint4*>(dst + 8 * j) = v;
      } else {
        for (int q = 0; q < p.half; ++q) {
          const int ix = MODE == MODE_SLOW_HALF ? q : 2 * q, iy = MODE == MODE_SLOW_HALF ? q + p.half : 2 * q + 1;
          const float x = __bfloat162float(src[ix]), y = __bfloat162float(src[iy]);
          const float2 c = cs[q];
          dst[ix] = __float2bfloat16(x * c.x - y * c.y);
          dst[iy] = __float2bfloat16(x * c.y + y * c.x);
        }
        for (int e = p.rot; e < p.dh; ++e) dst[e] = src[e];
      }
    } else {
      const int c = u - p.head_units, at = (p.heads + p.kv) * p.dh + 8 * c;        // a chunk of V
      const uint4 v = *reinterpret_cast<const uint4*>(src + at);
      if constexpr (APPEND) {
        const int g = 8 * c / p.dh, e = 8 * c - g * p.dh;
        if (g >= info[r].held) continue;
        *reinterpret_cast<uint4*>(p.v_cache + info[r].cache + (((long long)g * p.dh) << p.page_shift) + e) = v;
      } else {
        *reinterpret_cast<uint4*>(p.out + (row0 + r) * p.width + at) = v;
      }
    }
  }
}

template <bool APPEND>
int launch(PosParams& p, int layout, cudaStream_t st) {
  int mode;
  if (layout == TWIST_ROPE_HALF) mode = p.half % 8 == 0 ? MODE_HALF : MODE_SLOW_HALF;
  else mode = p.rot % 8 == 0 ? MODE_PAIRS : MODE_SLOW_PAIRS;
  if (p.rot == 0) mode = MODE_PAIRS;                                                    // plain 16-byte chunks
  p.units_per_head = mode == MODE_HALF ? p.half / 8 + (p.dh - p.rot) / 8 : mode == MODE_PAIRS ? p.dh / 8 : 1;
  p.head_units = (p.heads + p.kv) * p.units_per_head;
  p.chunk_units = p.kv * p.dh / 8;
  p.row_units = p.head_units + (APPEND || !p.in_place ? p.chunk_units : 0);
  if (APPEND && !p.out) p.row_units -= p.heads * p.units_per_head;
  // Rows of a tile: as many as still give every SM several tiles.
  const long long want = p.rows / ((long long)sm_count() * 8);
  p.tile_rows = (int)(want < 1 ? 1 : (want > kMaxRows ? kMaxRows : want));
  const long long tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
  if (tiles > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  const size_t smem = (size_t)p.tile_rows * p.half * sizeof(float2);                    // at most 8 KB
  const unsigned grid = (unsigned)tiles;
  void (*kernel)(PosParams) = mode == MODE_HALF ? rotate_rows_kernel<APPEND, MODE_HALF>
                              : mode == MODE_PAIRS ? rotate_rows_kernel<APPEND, MODE_PAIRS>
                              : mode == MODE_SLOW_HALF ? rotate_rows_kernel<APPEND, MODE_SLOW_HALF>
                                                       : rotate_rows_kernel<APPEND, MODE_SLOW_PAIRS>;
  TWIST_CUDA_TRY(launch_overlapped(kernel, dim3(grid), dim3(kPosThreads), smem, st, p));
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
