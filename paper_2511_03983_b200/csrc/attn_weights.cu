// The attention weight that cached keys gather, summed over the queries that look at them:
//     twist_attn_weights:       w_j = prior_j + sum_h exp(q_h . k_j / sqrt(d) - lse_h)          one new token per sequence, paged cache
//     twist_attn_core_weights:  w_j = sum_h sum_{i >= j} exp(q_hi . k_j / sqrt(d) - lse_hi)     prompts, projected activations
// The log-sum-exp is known, so every key is on its own: no running maximum, nothing to join, one writer per result.
//
// One new token.  K is read once (two bytes or one per element) against 2 operations per head and element: bound by HBM.
// Up to eight heads ride on one pass over the keys, with the operands of the decode kernel (decode_tiles.cuh).  A warp takes runs
// of tiles of one KV position of one sequence, the first run of every item before any second one, and its copies run on ahead
// from one run to the next.
//
// Prompts.  A CTA holds 128 (small heads: 64) keys and walks over the queries behind them: 2 d operations and an exponential
// for each pair of a query and a key of each head, nothing to speak of from memory.
#include "attn_weights.cuh"
#include "decode_tiles.cuh"
#include "plan.cuh"

namespace twist {
namespace {

struct WeightParams {
  DecParams d;                 // q, k, scales, table, len, heads; out and the workspace are not used
  const float* lse;            // [S][heads][n_seqs]
  const int32_t* new_len;
  const int32_t* seen;
  const float* prior;
  float* weights;
  int32_t* slot_pos;
  int run_tiles, runs;         // tiles of a run; runs of the longest sequence that can be
  float scale;                 // 1 / sqrt(d)
};

constexpr int kLenCache = 512, kCountCache = 256, kMaxRun = 16;

// exp(score * scale - lse).  The difference is formed before it is multiplied: it is small where the weight is not.
__device__ inline float weight_of(float score, float scale, float lse) { return ex2(fmaf(score, scale, -lse) * kLog2e); }

// A warp's ring of two tiles of SUB * 16 keys, filled by bulk copies: the 16 rows of a step lie next to each other in their page,
// and so do their prior weights.  Tiles of up to 4 KB and 16 warps an SM.  Measured (eight subnets of 16 ragged sequences of up to
// 8192 keys, e4m3, d = 128, 630 MB: 133 us; 64 ragged sequences of up to 16000, 32 heads on 4 positions of d = 64, 152 MB: 55.5).
// When these took 132 and 53 (before pages outside the pool and scores beyond fp32 were looked at): three tiles 157 and 64, d = 128 by
// 4 steps 155; keys straight into registers 180 and 84 to 105, 16 keys (32 at d = 64) at a time through rings 181 and 75: what a tile
// costs beside its keys has to be spread over many of them.
constexpr int kRing = 2;
template <int D, int B>
struct KeyRing {
  static constexpr int SUB = D * B >= 64 ? 256 / (D * B) : 4, TILE = 16 * SUB;
  struct alignas(16) {
    uint8_t k[TILE * D * B];
    float prior[TILE];
  } tile[kRing];
  float2 scale[kRing][SUB];
  int page[kRing][SUB];                        // -1: outside the pool, nothing may be written
  alignas(16) uint64_t full[kRing];            // of every step: its bytes to expect and, 8 bits, its scale
};

// Tiles t0 .. t1 - 1 of a KV position of a sequence, heads 8 rt .. of those that read it.
struct Unit {
  uint32_t number;                             // of its run
  int seq, s, pos, rt, len, t0, t1;
};

template <int D, int B>
__global__ void __launch_bounds__(kDecThreads, 4) weights_kernel(const WeightParams w) {
  using Sh = Shape<D, B>;
  constexpr int SUB = KeyRing<D, B>::SUB, TILE = KeyRing<D, B>::TILE, AHEAD = 32 / SUB, ARRIVALS = B == 1 ? 2 : 1;
  const DecParams& p = w.d;
  __shared__ int cols[kDecWarps][2][kCols];
  __shared__ __align__(16) QueryBuf<D, B> qbuf[kDecWarps];
  __shared__ int counts[kCountCache];
  __shared__ int32_t lens[kLenCache], head_cache[kHeadCache], pos_cache[kPosCache];
  __shared__ volatile int abort_flag;
  extern __shared__ __align__(16) unsigned char rings[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int N = p.S * p.n_seqs;
  KeyRing<D, B>& ring = reinterpret_cast<KeyRing<D, B>*>(rings)[warp];
  if (threadIdx.x == 0) abort_flag = 0;
  for (int i = threadIdx.x; i < kCountCache; i += kDecThreads) counts[i] = 0;
  if (lane == 0) {
    for (int i = 0; i < kRing; ++i) mbar_init(smem_u32(&ring.full[i]), ARRIVALS * SUB);
    fence_async_smem();
  }
  griddep_launch_dependents();
  griddep_wait();
  copy_words(lens, p.len, min(N, kLenCache));
  const Heads hd = cache_heads(p, head_cache, pos_cache, 0, p.S);
  wait_copies();
  __syncthreads();
  // Heads of every position, where they can be counted: none is walked over for nothing.
  const bool counted = hd.idx != p.head_idx && p.S * p.kv_max <= kCountCache;
  if (counted) {
    for (int i = threadIdx.x; i < p.S * p.heads; i += kDecThreads) {
      const int s = i / p.heads;
      atomicAdd(&counts[s * p.kv_max + position_of(p, hd, s, i - s * p.heads)], 1);
    }
    __syncthreads();
  }
  auto row_tiles = [&](int s, int pos) { return counted ? min((counts[s * p.kv_max + pos] + kCols - 1) / kCols, p.row_tiles) : p.row_tiles; };
  const uint32_t items = (uint32_t)N * p.kv_max, total = items * (uint32_t)w.runs, stride = gridDim.x * kDecWarps;
  auto settle = [&](Unit x) {                        // the first unit from run x.number on that has keys and heads (or none: seq < 0)
    for (; x.number < total; x.number += stride) {
      const uint32_t run = x.number / items, item = x.number - run * items;
      x.seq = (int)(item / p.kv_max);
      x.pos = (int)(item - (uint32_t)x.seq * p.kv_max);
      x.s = x.seq / p.n_seqs;
      x.len = clamped_len(p, x.seq < kLenCache ? lens[x.seq] : p.len[x.seq]);
      x.t0 = (int)run * w.run_tiles;
      x.t1 = min((x.len + TILE - 1) / TILE, x.t0 + w.run_tiles);
      x.rt = 0;
      if (x.t0 < x.t1 && row_tiles(x.s, x.pos) > 0) return x;
    }
    x.seq = -1;
    return x;
  };
  auto following = [&](Unit x) {
    if (++x.rt < row_tiles(x.s, x.pos)) return x;
    x.number += stride;
    return settle(x);
  };
  Unit now;
  now.number = blockIdx.x * kDecWarps + warp;
  now = settle(now);
  if (now.seq < 0) return;
  // The filling side walks the units by itself, kRing tiles ahead.
  Unit at = now, behind = now;
  bool live = false, inside = false;
  int tile = now.t0, n = 0, head_ids = 0, to = 0, id = 0, in_page = 0;
  int next_ids = fetch_pages<SUB>(p, now.seq, now.t0, 1, lane);
  auto window = [&](int ids) {                       // the page ids of the AHEAD tiles from `tile` on have come
    id = check_pages<SUB>(p, ids, at.len - 1, tile, 1, lane);
    inside = id == ids;
    next_ids = fetch_pages<SUB>(p, at.seq, tile + AHEAD, 1, lane);
    const int key = (int)step_key<SUB>(tile, 1, lane);
    in_page = key & ((1 << p.page_shift) - 1);
    live = key < at.len;
    n = 0;
  };
  auto look = [&] {
    behind = following(at);
    if (behind.seq >= 0) head_ids = fetch_pages<SUB>(p, behind.seq, behind.t0, 1, lane);
  };
  auto fill = [&] {                                  // a group of copies, empty behind the last tile
    if (tile >= at.t1) {
      if (behind.seq < 0) { commit_copies(); return; }
      at = behind;
      tile = at.t0;
      window(head_ids);
      look();
    }
    if (n == AHEAD) window(next_ids);
    if (lane / SUB == n) {
      const int step = lane % SUB;
      const uint32_t bar = smem_u32(&ring.full[to]);
      ring.page[to][step] = inside ? id : -1;
      if (live) {
        const long long row = (((long long)id * p.kv_max + at.pos) << p.page_shift) + in_page;
        const bool prior = at.rt == 0 && w.prior;
        mbar_expect_tx(bar, 16 * D * B + (prior ? 64 : 0));
        bulk_load(smem_u32(ring.tile[to].k + 16 * D * B * step),
                  static_cast<const uint8_t*>(p.k) + B * (id * p.page_stride + (((long long)at.pos << p.page_shift) + in_page) * D), 16 * D * B, bar);
        if (prior) bulk_load(smem_u32(ring.tile[to].prior + 16 * step), w.prior + row, 64, bar);
        if constexpr (B == 1) {
          copy_async<8>(&ring.scale[to][step], p.scales + (row >> 4));
          asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
        }
      } else {                                       // a step behind the end
        for (int i = 0; i < ARRIVALS; ++i) mbar_arrive(bar);
      }
    }
    commit_copies();
    to = to + 1 == kRing ? 0 : to + 1;
    ++tile;
    ++n;
  };
  // What a unit needs beside its keys; the queries go to shared memory.
  struct Ask {
    float l0, l1;
    int fresh, seen;
  };
  auto ask = [&](const Unit& x, int* col) {
    Ask a;
    find_heads(p, hd, x.s, x.pos, x.rt, lane, col);
    prefetch_q<D, B>(qbuf[warp], p, x.seq, col[g], lane);
    const int h0 = col[2 * t], h1 = col[2 * t + 1];
    const float* lse = w.lse + (long long)x.s * p.heads * p.n_seqs + (x.seq - x.s * p.n_seqs);
    a.l0 = h0 >= 0 ? lse[(long long)h0 * p.n_seqs] : 0.f;
    a.l1 = h1 >= 0 ? lse[(long long)h1 * p.n_seqs] : 0.f;
    a.fresh = w.new_len ? w.new_len[x.seq] : min(1, x.len);
    a.seen = w.seen ? w.seen[x.seq] : x.len;
    return a;
  };
  Ask mine = ask(now, cols[warp][0]);
  commit_copies();
  window(next_ids);
  look();
#pragma unroll 1
  for (int i = 0; i < kRing; ++i) fill();
  int buf = 0, slot = 0, since = kRing;
  uint32_t parity = 0;
  bool ok = true;
  for (;;) {
    Query<D, B> q;
    if (since >= 2) wait_copies_but<2>();
    else wait_copies();
    take_q<D, B>(q, qbuf[warp], lane);
    // columns without a head have zeros for a query, which give NaN where a key is infinite
    const bool none = cols[warp][buf][0] < 0, has0 = cols[warp][buf][2 * t] >= 0, has1 = cols[warp][buf][2 * t + 1] >= 0;
    const Unit next = following(now);
    Ask then = mine;
    if (next.seq >= 0) then = ask(next, cols[warp][buf ^ 1]);
    commit_copies();
    since = now.t1 - now.t0;
    if (mine.fresh < 0 || mine.fresh > now.len) {
      if (lane == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
      mine.fresh = max(0, min(mine.fresh, now.len));
    }
    const int first_new = now.len - mine.fresh, ahead = mine.seen - now.len;
    for (int i = now.t0; i < now.t1; ++i) {
      ok = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&ring.full[slot]), parity, &abort_flag, p.status));
      if (!ok) break;
      if (!none) {
        float a[2 * SUB];                            // sums of the thread's two heads: keys g, g + 8 of every step
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
          uint32_t x[2][Sh::KCH][Sh::KW];
          float sc[4];
          take_keys<D, B>(x, ring.tile[slot].k + 16 * D * B * s, g, t);
          step_scores<D, B>(sc, x, q, B == 1 ? ring.scale[slot][s].x : 1.f);
          a[2 * s] = (has0 ? weight_of(sc[0], w.scale, mine.l0) : 0.f) + (has1 ? weight_of(sc[1], w.scale, mine.l1) : 0.f);
          a[2 * s + 1] = (has0 ? weight_of(sc[2], w.scale, mine.l0) : 0.f) + (has1 ? weight_of(sc[3], w.scale, mine.l1) : 0.f);
        }
        // over the four threads of a row, so that each ends with sums of its own: SUB = 4 both of step t, 2 one of step t / 2, 1 one
        // for two threads
#pragma unroll
        for (int e = 0; e < SUB; ++e) {
          const float send = t & 2 ? a[e] : a[SUB + e], keep = t & 2 ? a[SUB + e] : a[e];
          a[e] = keep + __shfl_xor_sync(0xffffffffu, send, 2);
        }
        if constexpr (SUB == 1) {
          a[0] += __shfl_xor_sync(0xffffffffu, a[0], 1);
        } else {
#pragma unroll
          for (int e = 0; e < SUB / 2; ++e) {
            const float send = t & 1 ? a[e] : a[SUB / 2 + e], keep = t & 1 ? a[SUB / 2 + e] : a[e];
            a[e] = keep + __shfl_xor_sync(0xffffffffu, send, 1);
          }
        }
        const int in_tile = g + (SUB == 4 ? 16 * t : SUB == 2 ? 8 * t : 8 * (t >> 1)), key = i * TILE + in_tile;
        const int page = ring.page[slot][in_tile >> 4];
        const long long to_ = (((long long)page * p.kv_max + now.pos) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
#pragma unroll
        for (int e = 0; e < (SUB == 4 ? 2 : 1); ++e) {
          if (key + 8 * e < now.len && page >= 0 && (SUB > 1 || (t & 1) == 0)) {
            if (now.rt > 0) {
              w.weights[to_ + 8 * e] += a[e];        // the same thread wrote it
            } else {
              const bool fresh = key + 8 * e >= first_new;
              w.weights[to_ + 8 * e] = (fresh || !w.prior ? 0.f : ring.tile[slot].prior[in_tile + 8 * e]) + a[e];
              if (fresh && w.slot_pos) w.slot_pos[to_ + 8 * e] = key + 8 * e + ahead;
            }
          }
        }
      }
      __syncwarp();                                  // the tile has been read
      if (++slot == kRing) { slot = 0; parity ^= 1; }
      fill();
    }
    if (!ok || next.seq < 0) break;
    now = next;
    mine = then;
    buf ^= 1;
  }
  if (!ok) drain_after_abort(&abort_flag);
}

template <int D, int B>
int run_weights(WeightParams& w, long long max_len, cudaStream_t st) {
  DecParams& p = w.d;
  const long long items = (long long)p.S * p.n_seqs * p.kv_max;
  const long long longest = (((long long)p.max_pages << p.page_shift) + KeyRing<D, B>::TILE - 1) / KeyRing<D, B>::TILE + 2;
  if (items * p.row_tiles > 0x7fffffffll / longest) return TWIST_ERR_UNSUPPORTED;
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  constexpr size_t smem = kDecWarps * sizeof(KeyRing<D, B>);
  static int resident[64] = {0};
  const int slot = device_slot();
  if (resident[slot] == 0) {
    int n = 0;
    TWIST_CUDA_TRY(cudaFuncSetAttribute(weights_kernel<D, B>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    TWIST_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, weights_kernel<D, B>, kDecThreads, smem));
    resident[slot] = n < 1 ? 1 : n;
  }
  const long long warps = (long long)sm_count() * resident[slot] * kDecWarps;
  const long long tiles = (max_len + KeyRing<D, B>::TILE - 1) / KeyRing<D, B>::TILE;
  // One run a warp, but not so long that ragged lengths leave warps idle (twice as many runs, 256 ragged items of up to 2048 keys:
  // 12.2 us against 10.7; runs of up to 64 tiles, the first of the cases above: 156).
  const long long run_tiles = (tiles * items + warps - 1) / warps;
  w.run_tiles = (int)(run_tiles < kMaxRun ? run_tiles : kMaxRun);
  // every slot that the table has is in a run: the bound only chooses how long they are
  const long long all = (((long long)p.max_pages << p.page_shift) + KeyRing<D, B>::TILE - 1) / KeyRing<D, B>::TILE;
  w.runs = (int)((all + w.run_tiles - 1) / w.run_tiles);
  const long long need = (items * ((tiles + w.run_tiles - 1) / w.run_tiles) + kDecWarps - 1) / kDecWarps, most = warps / kDecWarps;
  TWIST_CUDA_TRY(launch_overlapped(weights_kernel<D, B>, dim3((unsigned)(need < most ? need : most)), dim3(kDecThreads), smem, st, 1, w));
  return TWIST_OK;
}

// ------------------------------------------------------------------------------------------------ prompts

constexpr int kCoreWarps = 4, kCoreThreads = 32 * kCoreWarps, kCoreKeys = 16 * kCoreWarps;

// Heads of 8, and of 16 and 32 where a key has few queries (see below).  A CTA holds a tile of 64 keys of one KV position in registers
// (a warp 16 of them) and walks over the queries that may look at them, head after head, tiles of QT through shared memory, the
// next one on its way.  The sums stay in the registers of the threads that own the scores and are joined over the four threads
// of a row at the end.  Bound by the chains of dependent instructions: more keys a warp mean longer ones and fewer CTAs (4 subnets of
// 4 prompts of 2048, 16 heads on 4 positions of d = 32: 16, 32 and 64 keys a warp 326, 454 and 544 us).
template <int D, int QT>
__global__ void __launch_bounds__(kCoreThreads) core_weights_kernel(const CoreParams p) {
  using Sh = Shape<D, 2>;
  constexpr int KEYS = kCoreKeys, STRIDE = D + 8;
  __shared__ __align__(16) __nv_bfloat16 qs[2][QT * STRIDE];
  __shared__ float ls[2][QT];
  __shared__ short list[kMaxHeads];
  __shared__ int n_list;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  // the tiles with the most queries first
  const unsigned items = (unsigned)p.S * p.n_seqs * p.kv_max, item = blockIdx.x % items;
  const int key0 = (int)(blockIdx.x / items) * KEYS, pos = (int)(item % p.kv_max);
  const long long seq = item / p.kv_max;
  const int s = (int)(seq / p.n_seqs), b = (int)(seq - (long long)s * p.n_seqs);
  griddep_launch_dependents();
  griddep_wait();
  const int len = prompt_len(p, seq);
  if (key0 >= len) return;
  if (warp == 0) {
    const int n = heads_of(p, s, pos, lane, list);
    if (lane == 0) n_list = n;
  }
  const __nv_bfloat16* rows = p.qkv + ((long long)s * p.T + (long long)b * p.seq_len) * p.nq;
  const int mine = key0 + 16 * warp;
  uint32_t x[2][Sh::KCH][Sh::KW];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int key = mine + g + 8 * r;
#pragma unroll
    for (int c = 0; c < Sh::KCH; ++c) {
      if (key < len) {
        load_words<Sh::KW>(x[r][c], rows + (long long)key * p.nq + (p.heads + pos) * D + c * 8 * Sh::KW + t * 2 * Sh::KW);
      } else {
#pragma unroll
        for (int w = 0; w < Sh::KW; ++w) x[r][c][w] = 0;
      }
    }
  }
  float sum0 = 0.f, sum1 = 0.f;                                    // of keys g and g + 8
  __syncthreads();
  if (n_list == 0) return;                                         // no head reads this position
  const int first = max(key0, p.last ? len - p.last : 0);          // the first query that counts
  const int begin = first / QT * QT;
  auto fetch = [&](int buf, int h, int q0) {                       // rows behind the end become zeros
    for (int k = threadIdx.x; k < QT * D / 8; k += kCoreThreads) {
      const int r = k / (D / 8), c = k % (D / 8), there = q0 + r < len;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(qs[buf] + r * STRIDE + 8 * c)),
                   "l"(rows + (long long)(there ? q0 + r : 0) * p.nq + h * D + 8 * c), "r"(there ? 16 : 0) : "memory");
    }
    if (threadIdx.x < QT) {
      const int q = q0 + threadIdx.x, there = q < len;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(ls[buf] + threadIdx.x)),
                   "l"(p.lse + ((long long)s * p.heads + h) * p.T + (long long)b * p.seq_len + (there ? q : 0)), "r"(there ? 4 : 0) : "memory");
    }
    commit_copies();
  };
  fetch(0, list[0], begin);
  int head = 0, q0 = begin;
  for (int buf = 0; head < n_list; buf ^= 1) {
    const int at = q0;
    if ((q0 += QT) >= len) { q0 = begin; ++head; }
    if (head < n_list) fetch(buf ^ 1, list[head], q0);
    else commit_copies();
    wait_copies_but<1>();
    __syncthreads();
    const bool edge = at < max(first, key0 + KEYS) || at + QT > len;
#pragma unroll 2
    for (int n = 0; n < QT; n += 8) {
      Query<D, 2> q;
      const __nv_bfloat16* row = qs[buf] + (n + g) * STRIDE + t * 2 * Sh::KW;
#pragma unroll
      for (int c = 0; c < Sh::KCH; ++c) take_words<Sh::KW>(q.w[c], reinterpret_cast<const uint8_t*>(row + c * 8 * Sh::KW));
      const float l0 = ls[buf][n + 2 * t], l1 = ls[buf][n + 2 * t + 1];
      float sc[4];
      step_scores<D, 2>(sc, x, q, 1.f);
      float e0 = weight_of(sc[0], p.scale, l0), e1 = weight_of(sc[1], p.scale, l1);
      float e2 = weight_of(sc[2], p.scale, l0), e3 = weight_of(sc[3], p.scale, l1);
      if (edge) {                                                  // queries a .. len - 1 (c .. for the second key) count
        const int i0 = at + n + 2 * t, a = max(mine + g, first), c = max(mine + g + 8, first);
        e0 = (unsigned)(i0 - a) < (unsigned)(len - a) ? e0 : 0.f;
        e1 = (unsigned)(i0 + 1 - a) < (unsigned)(len - a) ? e1 : 0.f;
        e2 = (unsigned)(i0 - c) < (unsigned)(len - c) ? e2 : 0.f;
        e3 = (unsigned)(i0 + 1 - c) < (unsigned)(len - c) ? e3 : 0.f;
      }
      sum0 += e0 + e1;
      sum1 += e2 + e3;
    }
    __syncthreads();                                               // the tile has been read
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    sum0 += __shfl_xor_sync(0xffffffffu, sum0, o);
    sum1 += __shfl_xor_sync(0xffffffffu, sum1, o);
  }
  const int key = mine + g + 8 * t;
  if (t < 2 && key < len) store_weight(p, seq, pos, key, t ? sum1 : sum0);
}

template <int D>
int run_core(CoreParams& p, cudaStream_t st) {
  const long long grid = (long long)p.S * p.n_seqs * p.kv_max * ((p.seq_len + kCoreKeys - 1) / kCoreKeys);
  if (grid > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  // Tiles of few queries where there are few of them (6 prompts of 77, the last 32 queries, d = 32: 5.8 us against 8.4); long prompts
  // with d = 8, which have no other kernel, take twice as many (those above at d = 16 in this kernel: 393 us against 320).
  void (*kernel)(CoreParams) = core_weights_kernel<D, 32>;
  if constexpr (D == 8) {
    if (p.seq_len > 256) kernel = core_weights_kernel<D, 64>;
  }
  TWIST_CUDA_TRY(launch_overlapped(kernel, dim3((unsigned)grid), dim3(kCoreThreads), 0, st, 1, p));
  return TWIST_OK;
}

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" int32_t twist_attn_weights(const twist_attn_weights_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->cache != TWIST_CACHE_BF16 && a->cache != TWIST_CACHE_E4M3) return TWIST_ERR_SHAPE;
  const bool q8 = a->cache == TWIST_CACHE_E4M3;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->head_keep <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 ||
      a->max_pages <= 0 || a->page_size <= 0 || a->max_len < 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if ((dh != 8 || q8) && dh != 16 && dh != 32 && dh != 64 && dh != 128) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets > TWIST_MAX_SUBNETS || a->n_heads > kMaxHeads || a->head_keep > kMaxHeads) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->n_subnets * a->n_seqs > 65535) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll - 1024) return TWIST_ERR_UNSUPPORTED;   // positions are 32-bit
  if (a->page_stride % (q8 ? 16 : 8) != 0 || a->page_stride < (long long)a->kv_max * a->page_size * dh) return TWIST_ERR_SHAPE;
  if (a->q_stride % 8 != 0 || a->q_stride < (long long)a->head_keep * dh) return TWIST_ERR_SHAPE;
  if (a->head_idx) {
    if (!a->kv_pos || a->n_heads <= 0 || a->n_kv_heads <= 0 || a->n_heads % a->n_kv_heads != 0) return TWIST_ERR_SHAPE;
  } else if (a->kv_max != a->head_keep) {
    return TWIST_ERR_SHAPE;
  }
  if (q8 != (a->scales != nullptr)) return TWIST_ERR_SHAPE;
  if (!a->q || !a->lse || !a->k_cache || !a->page_table || !a->kv_len || !a->weights) return TWIST_ERR_NULL;
  if (!aligned16(a->q) || !aligned16(a->lse) || !aligned16(a->k_cache) || !aligned16(a->scales) || !aligned16(a->prior) || !aligned16(a->weights) ||
      !aligned16(a->slot_pos))
    return TWIST_ERR_SHAPE;
  const long long bytes = (long long)a->n_pages * a->kv_max * a->page_size * 4;
  if ((a->prior && a->prior != a->weights && overlap(a->prior, bytes, a->weights, bytes)) ||
      (a->slot_pos && (overlap(a->slot_pos, bytes, a->weights, bytes) || (a->prior && overlap(a->slot_pos, bytes, a->prior, bytes)))))
    return TWIST_ERR_SHAPE;
  WeightParams w;
  memset(&w, 0, sizeof(w));
  DecParams& p = w.d;
  p.q = static_cast<const __nv_bfloat16*>(a->q);
  p.k = a->k_cache;
  p.scales = reinterpret_cast<const float2*>(a->scales);
  p.table = a->page_table; p.len = a->kv_len; p.head_idx = a->head_idx; p.kv_pos = a->kv_pos;
  p.page_stride = a->page_stride; p.q_stride = a->q_stride;
  p.S = a->n_subnets; p.n_seqs = a->n_seqs; p.heads = a->head_keep; p.kv_max = a->kv_max;
  p.per_group = a->head_idx ? a->n_heads / a->n_kv_heads : 1;
  p.n_kv_heads = a->head_idx ? a->n_kv_heads : a->kv_max;
  p.row_tiles = (p.per_group + kCols - 1) / kCols;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages;
  w.lse = a->lse; w.new_len = a->new_len; w.seen = a->seen;
  w.prior = a->prior; w.weights = a->weights; w.slot_pos = a->slot_pos;
  w.scale = 1.0f / sqrtf((float)dh);
  const long long table_len = (long long)a->max_pages * a->page_size;
  const long long max_len = a->max_len > 0 && a->max_len < table_len ? a->max_len : table_len;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (q8) {
    switch (dh) {
      case 16: return run_weights<16, 1>(w, max_len, st);
      case 32: return run_weights<32, 1>(w, max_len, st);
      case 64: return run_weights<64, 1>(w, max_len, st);
      default: return run_weights<128, 1>(w, max_len, st);
    }
  }
  switch (dh) {
    case 8: return run_weights<8, 2>(w, max_len, st);
    case 16: return run_weights<16, 2>(w, max_len, st);
    case 32: return run_weights<32, 2>(w, max_len, st);
    case 64: return run_weights<64, 2>(w, max_len, st);
    default: return run_weights<128, 2>(w, max_len, st);
  }
}

extern "C" int32_t twist_attn_core_weights(const twist_attn_core_weights_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->seq_len <= 0 || a->head_keep <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 ||
      a->max_pages <= 0 || a->page_size <= 0 || a->last_queries < 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if (dh != 8 && dh != 16 && dh != 32 && dh != 64 && dh != 128) return TWIST_ERR_UNSUPPORTED;
  if (a->n_subnets > TWIST_MAX_SUBNETS || a->head_keep > kMaxHeads || a->n_heads > kMaxHeads) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->max_pages * a->page_size > 0x7fffffffll - 1024 || a->seq_len > 0x7fffffff - 1024) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->n_seqs * a->seq_len > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  if (((long long)a->head_keep + 2ll * a->kv_max) * dh > (1 << 24)) return TWIST_ERR_UNSUPPORTED;
  if ((long long)a->n_subnets * a->n_seqs * a->kv_max > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  if (a->head_idx) {
    if (!a->kv_pos || a->n_heads <= 0 || a->n_kv_heads <= 0 || a->n_heads % a->n_kv_heads != 0) return TWIST_ERR_SHAPE;
  } else if (a->kv_max != a->head_keep) {
    return TWIST_ERR_SHAPE;
  }
  if (!a->qkv || !a->lse || !a->page_table || !a->weights) return TWIST_ERR_NULL;
  if (!aligned16(a->qkv) || !aligned16(a->lse) || !aligned16(a->weights) || !aligned16(a->slot_pos)) return TWIST_ERR_SHAPE;
  const long long bytes = (long long)a->n_pages * a->kv_max * a->page_size * 4;
  if (a->slot_pos && overlap(a->slot_pos, bytes, a->weights, bytes)) return TWIST_ERR_SHAPE;
  CoreParams p;
  memset(&p, 0, sizeof(p));
  p.qkv = static_cast<const __nv_bfloat16*>(a->qkv);
  p.lse = a->lse;
  p.table = a->page_table; p.new_len = a->new_len; p.head_idx = a->head_idx; p.kv_pos = a->kv_pos;
  p.weights = a->weights; p.slot_pos = a->slot_pos;
  p.S = a->n_subnets; p.n_seqs = a->n_seqs; p.seq_len = a->seq_len; p.heads = a->head_keep; p.kv_max = a->kv_max;
  p.per_group = a->head_idx ? a->n_heads / a->n_kv_heads : 1;
  p.n_kv_heads = a->head_idx ? a->n_kv_heads : a->kv_max;
  p.nq = (a->head_keep + 2 * a->kv_max) * dh;
  p.T = a->n_seqs * a->seq_len;
  p.last = a->last_queries;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages;
  p.scale = 1.0f / sqrtf((float)dh);
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // Heads of 16 and 32 go to the tensor cores too, unless their keys have few queries over all heads: a CTA's set-up there costs 4 us.
  // Average over the keys; d = 32, tensor cores against the other kernel: 64 prompts of up to 600, last 32 queries of 4 heads a
  // position 28.2 us against 20.5; 128 of up to 500, one head a position 64 against 41; 64 of 700, one head 39.2 against 39.2; 64 of up
  // to 200, 4 heads 19.5 against 28.3; one of 600, 4 heads 21.5 against 41.5; 16 of 2048, 4 heads 159 against 370.
  const long long queries = a->last_queries > 0 && a->last_queries < a->seq_len ? a->last_queries : a->seq_len / 2;
  const bool few = queries * a->head_keep < 320ll * a->kv_max;
  switch (dh) {
    case 8: return run_core<8>(p, st);
    case 16: if (few) return run_core<16>(p, st); break;
    case 32: if (few) return run_core<32>(p, st); break;
    default: break;
  }
  PlanScope scope(a->plan);
  return core_weights_tc(p, dh, st);
}
