// twist_kv_evict: every KV position of every sequence keeps its `keep` best tokens, by the attention weight that they have gathered.
//
// In place, and with few moves: attention does not depend on the order of the keys, so the tokens that stay below slot
// `keep` are not touched, and those that stay above it fill the slots below that became free (the i-th of one the i-th of
// the other).  Sources (from keep on) and destinations (below) do not meet, so all moves run at once; a full compaction
// would move half of the cache to drop one token.  Bytes: a weight and a position of every slot, and the rows that move.
//
// One cluster of 1 to 8 CTAs per (sequence, KV position); its warps take contiguous runs of slots.
//  1. A 32-bit key for each slot that orders as the tokens rank (protected tokens highest), kept in shared memory where it fits.
//  2. The keep-th largest key by radix selection, 11 + 11 + 10 bits: histograms in shared memory, added over the cluster.  Once its
//     bin holds few keys they are compared with each other, with their slots behind them (equal keys rank by slot).
//  3. Many equal keys are admitted in the order of slots: a running count over the runs.  Then every warp knows who stays:
//     bits to the workspace, with the number of free slots before each 32 and the list of the tokens that move.
//  4. bf16: the rows that move, in turn.  8 bits: the blocks of 16 slots that take tokens in, whose rows share a scale, are coded anew,
//     a warp a block.  The block that `keep` cuts holds sources too: it is last, when they have been read.
//
// Bound by the latency of these phases where a cache is a page over its budget (256 items of 1040 slots, d = 64 in 8 bits: 12.6 us of
// 0.7 us of bytes; all three passes of the selection and a warp for every 64 slots in 4., moved or not: 19.3), by it and the
// scattered rows for long prompts (64 items of up to 16000, d = 128 in bf16: 52 us, of which the moves are 28).
#include <cooperative_groups.h>

#include "e4m3.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kEvThreads = 512, kEvWarps = kEvThreads / 32;
constexpr int kBins = 2048;
constexpr int kKeyCache = 20480;          // keys that a CTA keeps in shared memory
constexpr int kMaxEvictCluster = 8, kSlotsPerCta = 1024;
constexpr int kLocalLen = 4096;           // longest sequence whose lists a CTA keeps there
constexpr int kTableCache = 1024;         // page ids that a CTA keeps there
// Candidates for the threshold that are compared with each other.  The long prompts above: 512 63 us, 256 58, 128 58.
constexpr int kDirect = 256;

struct EvictParams {
  uint8_t* k;                  // pages page_bytes apart
  uint8_t* v;
  float2* scales;              // (K, V) [n_pages][kv][page / 16]
  const int32_t *table, *len, *keep, *seen, *kv_count;
  const float* weights;
  const int32_t* slot_pos;
  float* weights_out;
  int32_t* slot_pos_out;
  int32_t* ws;
  long long page_bytes, ws_item;
  int n_seqs, kv, row_bytes, page_shift, n_pages, max_pages, max_len, recent, key_cache;
  int local;                   // the workspace of an item fits into shared memory
  int* status;
};

// The workspace of an item: stay bits and free slots before, one of each for 32 slots, the list of the tokens that move and that
// of the slots that they move to (at most half of the slots each).
__host__ __device__ constexpr long long groups_of(long long max_len) { return (max_len + 31) / 32; }
__host__ __device__ constexpr long long list_of(long long max_len) { return max_len / 2 + 1; }
__host__ __device__ constexpr long long item_words(long long max_len) { return (2 * groups_of(max_len) + 2 * list_of(max_len) + 3) / 4 * 4; }

__device__ inline uint32_t rank_key(float w, bool guarded) {
  if (guarded) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);                    // -0 counts as 0
  return min(u & 0x80000000u ? ~u : u | 0x80000000u, 0xfffffffeu);
}

// The item's slots: page and offset of slot i.
struct Slots {
  const int32_t* table;        // of the sequence, in shared memory where it fits
  long long base;              // kv position
  int kv, page_shift;
  __device__ int page(int i) const { return table[i >> page_shift]; }
  __device__ int offset(int i) const { return i & ((1 << page_shift) - 1); }
  __device__ long long at(int i) const { return (((long long)page(i) * kv + base) << page_shift) + offset(i); }
};

// Byte offset of slot's row in the caches.
__device__ inline long long row_of(const EvictParams& p, const Slots& sl, int slot) {
  return sl.page(slot) * p.page_bytes + ((sl.base << p.page_shift) + sl.offset(slot)) * p.row_bytes;
}
__device__ inline float2* scale_at(const EvictParams& p, const Slots& sl, int slot) {
  return p.scales + ((((long long)sl.page(slot) * p.kv + sl.base) << (p.page_shift - 4)) + (sl.offset(slot) >> 4));
}

// The slot whose token goes to a slot below keep: itself, or one that moves.
__device__ inline int source_of(const int32_t* bits, const int32_t* before, const int32_t* movers, int slot, int keep) {
  const int grp = slot >> 5, bit = slot & 31;
  const uint32_t stay = (uint32_t)bits[grp];
  if (stay >> bit & 1) return slot;
  const uint32_t live = (2u << min(31, keep - 1 - 32 * grp)) - 1;      // slots of the 32 that are below keep
  return movers[before[grp] + __popc(~stay & live & ((1u << bit) - 1))];
}

// Rows of a bf16 cache: the tokens movers[i] to slots[i].  A warp takes 32 at a time: a lane finds the places of one, then all
// of them carry 16 bytes of K or V per turn, kTurns turns in flight.  CH: 16-byte pieces of a row, 1 to 16, a power of two.
constexpr int kTurns = 4;                 // the long prompts above, eight turns 73 us, four 54, two 59
template <int CH>
__device__ inline void carry_rows(const EvictParams& p, long long from, long long to, int n, int lane) {
  constexpr int PER = 32 / (2 * CH);                                  // tokens of a turn
  constexpr int TURNS = 2 * CH < kTurns ? 2 * CH : kTurns;            // in flight; 2 CH turns carry 32 tokens
  const int mine = lane / (2 * CH), piece = lane % (2 * CH);
  uint8_t* cache = (piece >= CH ? p.v : p.k) + 16 * (piece % CH);
#pragma unroll 1
  for (int k = 0; k < 32 && k < n; k += PER * TURNS) {
    uint4 x[TURNS];
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
      const int i = k + j * PER + mine;
      const long long at = __shfl_sync(0xffffffffu, from, i);
      if (i < n) x[j] = *reinterpret_cast<const uint4*>(cache + at);
    }
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
      const int i = k + j * PER + mine;
      const long long at = __shfl_sync(0xffffffffu, to, i);
      if (i < n) *reinterpret_cast<uint4*>(cache + at) = x[j];
    }
  }
}
// CH 0: rows of other sizes.
template <int CH>
__device__ inline void move_rows(const EvictParams& p, const Slots& sl, const int32_t* movers, const int32_t* slots, int n, int warp, int warps, int lane) {
  for (int base = 32 * warp; base < n; base += 32 * warps) {
    const int i = base + lane, m = min(32, n - base);
    long long from = 0, to = 0;
    if (i < n) {
      const int a = movers[i], b = slots[i];
      from = row_of(p, sl, a);
      to = row_of(p, sl, b);
      const float w = p.weights[sl.at(a)];
      const int32_t x = p.slot_pos[sl.at(a)];
      p.weights_out[sl.at(b)] = w;
      p.slot_pos_out[sl.at(b)] = x;
    }
    if constexpr (CH > 0) {
      carry_rows<CH>(p, from, to, m, lane);
    } else {                                                           // a lane its own token
      for (int c = 0; i < n && c < p.row_bytes; c += 16) {
        *reinterpret_cast<uint4*>(p.k + to + c) = *reinterpret_cast<const uint4*>(p.k + from + c);
        *reinterpret_cast<uint4*>(p.v + to + c) = *reinterpret_cast<const uint4*>(p.v + from + c);
      }
    }
  }
}

// The largest magnitude of 16 e4m3 numbers, a NaN counting for nothing: magnitudes order as their bits do.
__device__ inline float largest(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t most = 0;                                                   // two at a time
#pragma unroll
  for (int i = 0; i < 4; ++i) most = __vmaxu2(most, __vmaxu2(w[i] & 0x007f007fu, w[i] >> 8 & 0x007f007fu));
  most = max(most & 0xffffu, most >> 16);
  float a[4];
  if (most < 0x7f) {
    widen4(a, most);
    return a[0];
  }
  float m = 0.f;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    widen4(a, i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    m = fmaxf(fmaxf(m, fmaxf(fabsf(a[0]), fabsf(a[1]))), fmaxf(fabsf(a[2]), fabsf(a[3])));
  }
  return m;
}

// A block of an 8-bit cache that takes tokens in: all its rows coded anew with the scale that they need.
template <int D>
__device__ inline void move_block(const EvictParams& p, const Slots& sl, int slot0, int from, int lane) {
  constexpr int CH = D / 16, N = D >= 32 ? D / 32 : 1;               // pieces of 16 numbers of a row, of a lane
  uint4 x[2][N];
  float scale[2][N], top[2] = {0.f, 0.f};
  int src[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int k = 32 * j + lane, r = k / CH, c = k % CH;
    src[j] = __shfl_sync(0xffffffffu, from, r & 15);
    if (r >= 16) src[j] = -1;
    if (src[j] >= 0) {
      const long long at = row_of(p, sl, src[j]) + 16 * c;
      const float2 both = *scale_at(p, sl, src[j]);
      x[0][j] = *reinterpret_cast<const uint4*>(p.k + at);
      x[1][j] = *reinterpret_cast<const uint4*>(p.v + at);
      scale[0][j] = both.x;
      scale[1][j] = both.y;
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (src[j] < 0) continue;
      top[which] = fmaxf(top[which], largest(x[which][j]) * scale[which][j]);
    }
  float2 now;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    top[which] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top[which])));
    (which ? now.y : now.x) = scale_for(top[which]);
  }
  __syncwarp();                                                        // everything has been read
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float to = which ? now.y : now.x, inv = inverse_scale(to);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int k = 32 * j + lane, r = k / CH, c = k % CH;
      if (src[j] < 0 || (src[j] == slot0 + r && scale[which][j] == to)) continue;
      const uint32_t w[4] = {x[which][j].x, x[which][j].y, x[which][j].z, x[which][j].w};
      const float f = scale[which][j] * inv;
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a[4];
        widen4(a, w[i]);
        y[i] = narrow4_finite(a[0] * f, a[1] * f, a[2] * f, a[3] * f);     // (a NaN stays one)
      }
      *reinterpret_cast<uint4*>((which ? p.v : p.k) + row_of(p, sl, slot0 + r) + 16 * c) = make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
  if (lane == 0) *scale_at(p, sl, slot0) = now;
}

__device__ inline uint32_t inclusive(uint32_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// D: elements of a row of an 8-bit cache; of a bf16 cache minus the 16-byte pieces of a row, 0 for sizes that move_rows has no own
// form for.
template <int D>
__global__ void __launch_bounds__(kEvThreads, 2) evict_kernel(const EvictParams p) {
  constexpr int WARPS = kEvWarps, THREADS = kEvThreads;
  static_assert(WARPS == 16 && kBins == 2048, "shifts below");
  extern __shared__ uint32_t keys[];
  __shared__ int32_t table[kTableCache];
  __shared__ __align__(16) uint32_t hist[3][kBins];
  __shared__ int counts[3][WARPS];
  __shared__ uint32_t sums[WARPS];
  __shared__ int ranks[kDirect];
  __shared__ int guarded, bad, n_cand, thr_slot_s;
  __shared__ uint32_t thr_key_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const uint32_t item = blockIdx.x / (unsigned)ctas, seq_ = item / (unsigned)p.kv;
  const long long seq = seq_;
  const int pos = (int)(item - seq_ * p.kv), s = (int)(seq_ / (unsigned)p.n_seqs);
  auto sync = [&] {
    if (ctas == 1) __syncthreads();
    else cluster.sync();
  };
  griddep_launch_dependents();
  for (int b = threadIdx.x; b < 3 * kBins; b += THREADS) hist[0][b] = 0;
  if (threadIdx.x == 0) guarded = bad = n_cand = 0;
  griddep_wait();
  // one round trip: the lengths, and the table whatever the length is
  const int held = p.kv_count ? p.kv_count[s] : p.kv;
  int len = p.len[seq], keep = p.keep[seq];
  const int seen = p.seen ? p.seen[seq] : len;
  for (int i = threadIdx.x; i < min(p.max_pages, kTableCache); i += THREADS) table[i] = p.table[seq * p.max_pages + i];
  __syncthreads();
  if (pos >= held) return;
  if (len < 0 || len > p.max_len || keep < 0 || keep > p.max_len) {
    if (threadIdx.x == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
    len = max(0, min(len, p.max_len));
    keep = max(0, min(keep, p.max_len));
  }
  const int pages = (len + (1 << p.page_shift) - 1) >> p.page_shift;
  const Slots sl{pages <= kTableCache ? table : p.table + seq * p.max_pages, pos, p.kv, p.page_shift};
  const bool in_place = p.weights == p.weights_out;
  if (len <= keep) {                                                   // all stay
    if (in_place) return;
    for (int i = rank * THREADS + threadIdx.x; i < len; i += ctas * THREADS) {
      if ((unsigned)sl.page(i) >= (unsigned)p.n_pages) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); continue; }
      p.weights_out[sl.at(i)] = p.weights[sl.at(i)];
      p.slot_pos_out[sl.at(i)] = p.slot_pos[sl.at(i)];
    }
    return;
  }
  if (keep == 0) return;
  const long long guard = (long long)seen - min(p.recent, keep);
  // the warp's run of slots
  const int log_ctas = __ffs(ctas) - 1, warps = ctas * WARPS, me = rank * WARPS + warp;           // a power of two
  const int run = (((len + warps - 1) >> (4 + log_ctas)) + 31) & ~31;
  const int lo = (int)min((long long)len, (long long)me * run), hi = min(len, lo + run);
  const int key0 = warp * run;                                         // of the run in shared memory
  auto compute_key = [&](int i) {
    const long long at = sl.at(i);
    return rank_key(p.weights[at], p.slot_pos[at] >= guard);
  };
  auto key_at = [&](int i) { return key0 + (i - lo) < p.key_cache ? keys[key0 + (i - lo)] : compute_key(i); };

  // Lanes that agree add up first: the same weight everywhere would be counted one by one.  (Lanes that agree with any other, by a
  // match over the warp: 15.7 and 58 us against 15.3 and 54 in the two cases above.)
  auto count = [&](uint32_t* bins, uint32_t bin, bool mine) {
    const unsigned live = __ballot_sync(0xffffffffu, mine);
    if (live == 0) return;
    const int leader = __ffs(live) - 1;
    const bool alike = __shfl_sync(0xffffffffu, bin, leader) == bin;
    if (__all_sync(0xffffffffu, alike || !mine)) {
      if (lane == leader) atomicAdd(&bins[bin], (uint32_t)__popc(live));
    } else if (mine) {
      atomicAdd(&bins[bin], 1u);
    }
  };
  // 1. keys
  {
    int mine = 0;
    bool wrong = false;
    constexpr int BATCH = 4;                                            // groups whose loads are in flight
    for (int g0 = lo; g0 < hi; g0 += 32 * BATCH) {
      float w[BATCH];
      int32_t x[BATCH];
      bool fine[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int i = g0 + 32 * j + lane;
        const bool there = i < hi;
        fine[j] = there && (unsigned)sl.page(i) < (unsigned)p.n_pages;
        wrong |= there && !fine[j];
        if (fine[j]) {
          const long long at = sl.at(i);
          w[j] = p.weights[at];
          x[j] = p.slot_pos[at];
        }
      }
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int i = g0 + 32 * j + lane;
        if (g0 + 32 * j >= hi) break;
        uint32_t key = 0;
        if (fine[j]) {
          key = rank_key(w[j], x[j] >= guard);
          if (key0 + (i - lo) < p.key_cache) keys[key0 + (i - lo)] = key;
        }
        const bool guards = fine[j] && key == 0xffffffffu;
        mine += guards;
        count(hist[0], key >> 21, fine[j] && !guards);
      }
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0 && mine) atomicAdd(&guarded, mine);
    if (wrong) bad = 1;
  }
  sync();
  int total_guarded = guarded, any_bad = bad;
  if (ctas > 1) {
    total_guarded = __reduce_add_sync(0xffffffffu, lane < ctas ? *cluster.map_shared_rank(&guarded, lane) : 0);
    any_bad = __any_sync(0xffffffffu, lane < ctas && *cluster.map_shared_rank(&bad, lane));
  }
  if (any_bad) {
    if (threadIdx.x == 0 && rank == 0) atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX);
    sync();                                                            // the others have read the counters
    return;
  }
  // 2. the threshold: keys above it stay, and of those that are it the first `quota`, up to slot thr_slot
  uint32_t threshold = 0xffffffffu;
  int quota = keep, equals = total_guarded, thr_slot = 0x7fffffff;
  if (total_guarded < keep) {
    int need = keep - total_guarded;
    uint32_t prefix = 0;
    int last = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      if (pass > 0 && (equals <= kDirect || equals == need)) break;
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
      constexpr int kLast = 1024;
      const int bins = pass == 2 ? kLast : kBins;
      if (pass > 0) {
        const int above = pass == 1 ? 21 : 10;
        for (int g0 = lo; g0 < hi; g0 += 32) {
          const int i = g0 + lane;
          const uint32_t key = i < hi ? key_at(i) : 0xffffffffu;
          count(hist[pass], (key >> shift) & (bins - 1), key != 0xffffffffu && key >> above == prefix >> above);
        }
        sync();
      }
      // The bin from the top in which the need-th key is: every warp adds up a 16th of the bins, then every warp finds the 16th
      // and the bin in it.  In a cluster every CTA adds up its share of all CTAs' bins first (each adding up everything moves a
      // cluster's worth of histograms through every SM: 54 us against 52 for the long prompts above).
      const int group = bins / WARPS;                                  // 128, or 64: half of the lanes
      const bool reads = 4 * lane < group;
      const int share = bins >> log_ctas, groups = WARPS >> log_ctas;  // of a CTA
      if (ctas > 1) {
        for (int b = rank * share + threadIdx.x; b < (rank + 1) * share; b += THREADS) {
          uint32_t n = 0;
#pragma unroll
          for (int c = 0; c < kMaxEvictCluster; ++c)                   // all on their way at once
            if (c < ctas) n += cluster.map_shared_rank(hist[pass], c)[b];
          hist[pass][b] = n;
        }
        __syncthreads();
      }
      auto four = [&](int b) {                                         // bins b .. b + 3
        const uint32_t* from = ctas == 1 ? hist[pass] : cluster.map_shared_rank(hist[pass], b >> ((pass == 2 ? 10 : 11) - log_ctas));
        return *reinterpret_cast<const uint4*>(from + b);
      };
      if (warp < groups) {
        const int b = (rank * groups + warp) * group + 4 * lane;
        const uint4 v = reads ? *reinterpret_cast<const uint4*>(hist[pass] + b) : make_uint4(0, 0, 0, 0);
        const uint32_t all = __reduce_add_sync(0xffffffffu, v.x + v.y + v.z + v.w);
        if (lane == 0) sums[rank * groups + warp] = all;
      }
      sync();
      uint32_t part = 0;
      if (lane < WARPS) {
        const int of = WARPS - 1 - lane;
        part = ctas == 1 ? sums[of] : cluster.map_shared_rank(sums, of >> (4 - log_ctas))[of];
      }
      const uint32_t upto = inclusive(part, lane);
      const int at = __ffs(__ballot_sync(0xffffffffu, upto >= (uint32_t)need)) - 1;
      const int top = bins - at * group - 4 - 4 * lane;                // the lane's four bins of it, from the highest down
      const uint4 v = reads ? four(top) : make_uint4(0, 0, 0, 0);
      const uint32_t mine = v.x + v.y + v.z + v.w;
      const uint32_t before_mine = __shfl_sync(0xffffffffu, upto - part, at) + inclusive(mine, lane) - mine;
      const int here = __ffs(__ballot_sync(0xffffffffu, before_mine + mine >= (uint32_t)need)) - 1;
      uint32_t over = before_mine, n_bin = v.w;
      int bin = top + 3;
      if (over + n_bin < (uint32_t)need) { over += n_bin; n_bin = v.z; --bin; }
      if (over + n_bin < (uint32_t)need) { over += n_bin; n_bin = v.y; --bin; }
      if (over + n_bin < (uint32_t)need) { over += n_bin; n_bin = v.x; --bin; }
      const int found_bin = __shfl_sync(0xffffffffu, bin, here), found_above = (int)__shfl_sync(0xffffffffu, over, here);
      equals = (int)__shfl_sync(0xffffffffu, n_bin, here);
      prefix |= (uint32_t)found_bin << shift;
      need -= found_above;
      last = pass;
    }
    threshold = prefix;
    quota = need;
    if (equals == need) {                                              // the whole bin stays: its lowest key will do
      quota = 0x7fffffff;
    } else if (equals <= kDirect) {
      // The keys of the bin, with their slots, into every CTA; each is compared with the others.
      const int at_shift = last == 0 ? 21 : (last == 1 ? 10 : 0);
      // nobody reads these bins any more, or yet
      unsigned long long* own = reinterpret_cast<unsigned long long*>(hist[last == 2 ? 0 : last + 1]), *all = own;
      for (int g0 = lo; g0 < hi; g0 += 32) {
        const int i = g0 + lane;
        const uint32_t key = i < hi ? key_at(i) : 0xffffffffu;
        const bool in_bin = key != 0xffffffffu && key >> at_shift == prefix >> at_shift;
        const unsigned vote = __ballot_sync(0xffffffffu, in_bin);
        if (vote == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&n_cand, __popc(vote));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(vote & ((1u << lane) - 1));
        if (in_bin) own[at] = (unsigned long long)key << 32 | (uint32_t)~i;
      }
      for (int i = threadIdx.x; i < equals; i += THREADS) ranks[i] = 0;
      sync();
      if (ctas > 1) {
        all = own + kDirect;
        const int n = lane < ctas ? *cluster.map_shared_rank(&n_cand, lane) : 0;
        const int before_them = (int)inclusive((uint32_t)n, lane) - n;
        for (int c = 0; c < ctas; ++c) {
          const int at = __shfl_sync(0xffffffffu, before_them, c), i = threadIdx.x;
          if (i < __shfl_sync(0xffffffffu, n, c)) all[at + i] = cluster.map_shared_rank(own, c)[i];
        }
        __syncthreads();
      }
      // 32 candidates to a warp, against a share of the others
      const int log_groups = 32 - __clz((equals - 1) >> 5), parts = WARPS >> log_groups, part = warp >> log_groups;
      const int mine = (warp & ((1 << log_groups) - 1)) * 32 + lane;
      if (mine < equals) {
        const unsigned long long me_ = all[mine];
        int above = 0;
        for (int i = part; i < equals; i += parts) above += all[i] > me_;
        if (above) atomicAdd(&ranks[mine], above);
      }
      __syncthreads();
      if (threadIdx.x < equals && ranks[threadIdx.x] == need - 1) {
        thr_key_s = (uint32_t)(all[threadIdx.x] >> 32);
        thr_slot_s = (int)~(uint32_t)all[threadIdx.x];
      }
      __syncthreads();
      threshold = thr_key_s;
      thr_slot = thr_slot_s;
      quota = 0x7fffffff;
    }
  }
  // numbers of the runs before this warp's
  auto before_me = [&](const int* of) {
    int n = 0;
    for (int w = lane; w < me; w += 32) n += ctas == 1 ? of[w] : cluster.map_shared_rank(of, w / WARPS)[w % WARPS];
    return __reduce_add_sync(0xffffffffu, n);
  };
  // 3. equal keys in the order of slots, if not all of them stay
  int equal = 0;
  if (equals > quota) {
    int n = 0;
    for (int i = lo + lane; i < hi; i += 32) n += key_at(i) == threshold;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) counts[0][warp] = n;
    sync();
    equal = before_me(counts[0]);
  }
  int32_t* bits = p.local ? reinterpret_cast<int32_t*>(keys + p.key_cache) : p.ws + item * p.ws_item;
  int32_t* before = bits + groups_of(p.max_len);
  int32_t* movers = before + groups_of(p.max_len);
  int32_t* slots = movers + list_of(p.max_len);
  int free_n = 0, move_n = 0;
  for (int g0 = lo; g0 < hi; g0 += 32) {
    const int i = g0 + lane;
    const uint32_t key = i < hi ? key_at(i) : 0u;
    const unsigned same = __ballot_sync(0xffffffffu, i < hi && key == threshold);
    const bool stays = i < hi && (key > threshold || (key == threshold && i <= thr_slot && equal + __popc(same & ((1u << lane) - 1)) < quota));
    const unsigned stay = __ballot_sync(0xffffffffu, stays);
    const unsigned below = keep >= g0 + 32 ? 0xffffffffu : (keep <= g0 ? 0u : (1u << (keep - g0)) - 1);
    equal += __popc(same);
    free_n += __popc(~stay & below);
    move_n += __popc(stay & ~below);
    if (lane == 0) bits[g0 >> 5] = (int32_t)stay;
  }
  if (lane == 0) {
    counts[1][warp] = free_n;
    counts[2][warp] = move_n;
  }
  sync();
  int free_at = before_me(counts[1]), move_at = before_me(counts[2]), moves = 0;
  if (D <= 0) {
    for (int w = lane; w < warps; w += 32) moves += ctas == 1 ? counts[2][w] : cluster.map_shared_rank(counts[2], w / WARPS)[w % WARPS];
    moves = __reduce_add_sync(0xffffffffu, moves);
  }
  for (int g0 = lo; g0 < hi; g0 += 32) {
    const uint32_t stay = (uint32_t)bits[g0 >> 5];                     // the warp's own words
    const uint32_t below = keep >= g0 + 32 ? 0xffffffffu : (keep <= g0 ? 0u : (1u << (keep - g0)) - 1);
    const uint32_t open = ~stay & below, all = stay & ~below, under = (1u << lane) - 1;
    if (all >> lane & 1) movers[move_at + __popc(all & under)] = g0 + lane;
    if (D > 0) {
      if (lane == 0) before[g0 >> 5] = free_at;
    } else if (open >> lane & 1) {
      slots[free_at + __popc(open & under)] = g0 + lane;
    }
    move_at += __popc(all);
    free_at += __popc(open);
  }
  sync();
  // 4. the moves
  if constexpr (D <= 0) {
    move_rows<-D>(p, sl, movers, slots, moves, me, warps, lane);
    const int first = rank * THREADS + threadIdx.x, stride = ctas * THREADS;
    if (!in_place)
      for (int i = first; i < keep; i += stride)
        if ((uint32_t)bits[i >> 5] >> (i & 31) & 1) {
          p.weights_out[sl.at(i)] = p.weights[sl.at(i)];
          p.slot_pos_out[sl.at(i)] = p.slot_pos[sl.at(i)];
        }
    return;
  }
  // weights and positions
  {
    const int first = rank * THREADS + threadIdx.x, stride = ctas * THREADS;
#pragma unroll 2
    for (int slot = first; slot < keep; slot += stride) {
      const int from = source_of(bits, before, movers, slot, keep);
      if (from != slot || !in_place) {
        const long long to = sl.at(slot), at = sl.at(from);
        const float w = p.weights[at];
        const int32_t x = p.slot_pos[at];
        p.weights_out[to] = w;
        p.slot_pos_out[to] = x;
      }
    }
  }
  // rows: the blocks that take tokens in, the one that `keep` cuts last (it holds sources too)
  const int cut = keep & 15 ? keep >> 4 : -1;
  auto fill = [&](int block) {
    const int slot0 = block << 4, slot = slot0 + (lane & 15);
    const int from = slot >= len ? -1 : slot >= keep ? slot : source_of(bits, before, movers, slot, keep);
    if constexpr (D > 0) move_block<D>(p, sl, slot0, from, lane);
  };
  auto takes_in = [&](int block) { return (~(uint32_t)bits[block >> 1] >> (block & 1 ? 16 : 0) & 0xffffu & ((1u << min(16, keep - 16 * block)) - 1)) != 0; };
  const int blocks = (keep + 15) >> 4;
  for (int b0 = 0, number = 0; b0 < blocks; b0 += 32) {                // the warps take them in turn
    const bool mine = b0 + lane < blocks && b0 + lane != cut && takes_in(b0 + lane);
    const unsigned vote = __ballot_sync(0xffffffffu, mine);
    const int turn = number + __popc(vote & ((1u << lane) - 1));
    for (unsigned todo = __ballot_sync(0xffffffffu, mine && ((turn ^ me) & (warps - 1)) == 0); todo; todo &= todo - 1) fill(b0 + __ffs(todo) - 1);
    number += __popc(vote);
  }
  if (cut >= 0) {
    sync();
    if (me == 0 && takes_in(cut)) fill(cut);
  }
}

template <int D>
int run_evict(EvictParams& p, long long items, cudaStream_t st) {
  // CTAs of an item: as many as still have kSlotsPerCta slots each, two for an SM (four: 85 us against 54 for the long prompts above,
  // one 74; a page over in two CTAs an item 30 against 12.6).
  int ctas = 1;
  while (ctas < kMaxEvictCluster && p.max_len > ctas * kSlotsPerCta && items * ctas <= sm_count()) ctas *= 2;
  const long long warps = (long long)ctas * kEvWarps, run = ((p.max_len + warps - 1) / warps + 31) / 32 * 32;
  p.key_cache = (int)(run * kEvWarps < kKeyCache ? run * kEvWarps : kKeyCache);
  static bool ready[64] = {false};
  const int slot = device_slot();
  if (!ready[slot]) {
    TWIST_CUDA_TRY(cudaFuncSetAttribute(evict_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeyCache * 4));
    ready[slot] = true;
  }
  p.local = ctas == 1 && p.max_len <= kLocalLen;
  const size_t smem = ((size_t)p.key_cache + (p.local ? item_words(p.max_len) : 0)) * 4;
  TWIST_CUDA_TRY(launch_overlapped(evict_kernel<D>, dim3((unsigned)(items * ctas)), dim3(kEvThreads), smem, st, ctas, p));
  return TWIST_OK;
}

constexpr long long kMaxItems = 1 << 20, kMaxSlots = 1 << 26;

}  // namespace
}  // namespace twist

using namespace twist;

extern "C" size_t twist_kv_evict_workspace_bytes(int32_t n_subnets, int32_t n_seqs, int32_t kv_max, int64_t max_len) {
  if (n_subnets <= 0 || n_seqs <= 0 || kv_max <= 0 || max_len <= 0 || max_len > kMaxSlots) return 0;
  if ((long long)n_subnets * n_seqs > kMaxItems || (long long)n_subnets * n_seqs * kv_max > kMaxItems) return 0;
  return (size_t)n_subnets * n_seqs * kv_max * item_words(max_len) * 4;
}

extern "C" int32_t twist_kv_evict(const twist_kv_evict_args* a, void* stream) {
  if (!a) return TWIST_ERR_NULL;
  if (a->dtype != TWIST_BF16) return TWIST_ERR_UNSUPPORTED;
  if (a->cache != TWIST_CACHE_BF16 && a->cache != TWIST_CACHE_E4M3) return TWIST_ERR_SHAPE;
  const bool q8 = a->cache == TWIST_CACHE_E4M3;
  if (a->n_subnets <= 0 || a->n_seqs <= 0 || a->kv_max <= 0 || a->d_head <= 0 || a->n_pages <= 0 || a->max_pages <= 0 || a->page_size <= 0 ||
      a->max_len < 0 || a->recent < 0)
    return TWIST_ERR_SHAPE;
  const int dh = a->d_head;
  if (q8 ? dh != 16 && dh != 32 && dh != 64 && dh != 128 : dh % 8 != 0 || dh > 256) return TWIST_ERR_UNSUPPORTED;
  if (a->page_size < 16 || a->page_size > 1024 || (a->page_size & (a->page_size - 1))) return TWIST_ERR_UNSUPPORTED;
  const long long table_len = (long long)a->max_pages * a->page_size;
  const long long max_len = a->max_len > 0 && a->max_len < table_len ? a->max_len : table_len;
  if (max_len > kMaxSlots || (long long)a->n_subnets * a->n_seqs > kMaxItems || (long long)a->n_subnets * a->n_seqs * a->kv_max > kMaxItems)
    return TWIST_ERR_UNSUPPORTED;
  if (a->page_stride % (q8 ? 16 : 8) != 0 || a->page_stride < (long long)a->kv_max * a->page_size * dh) return TWIST_ERR_SHAPE;
  if (q8 != (a->scales != nullptr)) return TWIST_ERR_SHAPE;
  if (!a->k_cache || !a->v_cache || !a->page_table || !a->kv_len || !a->keep || !a->weights || !a->slot_pos || !a->weights_out || !a->slot_pos_out)
    return TWIST_ERR_NULL;
  if (!aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->scales) || !aligned16(a->weights) || !aligned16(a->slot_pos) ||
      !aligned16(a->weights_out) || !aligned16(a->slot_pos_out) || !aligned16(a->ws))
    return TWIST_ERR_SHAPE;
  const long long bytes = (long long)a->n_pages * a->kv_max * a->page_size * 4;
  const bool in_place = a->weights == a->weights_out;
  if (in_place != (a->slot_pos == a->slot_pos_out)) return TWIST_ERR_SHAPE;
  if (overlap(a->weights, bytes, a->slot_pos, bytes) || overlap(a->weights_out, bytes, a->slot_pos_out, bytes) ||
      (!in_place && (overlap(a->weights, bytes, a->weights_out, bytes) || overlap(a->weights, bytes, a->slot_pos_out, bytes) ||
                     overlap(a->slot_pos, bytes, a->weights_out, bytes) || overlap(a->slot_pos, bytes, a->slot_pos_out, bytes))))
    return TWIST_ERR_SHAPE;
  if (!a->ws || a->ws_bytes < twist_kv_evict_workspace_bytes(a->n_subnets, a->n_seqs, a->kv_max, max_len)) return TWIST_ERR_WORKSPACE;
  EvictParams p;
  memset(&p, 0, sizeof(p));
  p.k = static_cast<uint8_t*>(a->k_cache);
  p.v = static_cast<uint8_t*>(a->v_cache);
  p.scales = reinterpret_cast<float2*>(a->scales);
  p.table = a->page_table; p.len = a->kv_len; p.keep = a->keep; p.seen = a->seen; p.kv_count = a->kv_count;
  p.weights = a->weights; p.slot_pos = a->slot_pos; p.weights_out = a->weights_out; p.slot_pos_out = a->slot_pos_out;
  p.ws = static_cast<int32_t*>(a->ws);
  p.row_bytes = dh * (q8 ? 1 : 2);
  p.page_bytes = a->page_stride * (q8 ? 1 : 2);
  p.ws_item = item_words(max_len);
  p.n_seqs = a->n_seqs; p.kv = a->kv_max;
  p.page_shift = 31 - __builtin_clz((unsigned)a->page_size);
  p.n_pages = a->n_pages; p.max_pages = a->max_pages; p.max_len = (int)max_len; p.recent = a->recent;
  p.status = device_status_ptr();
  if (!p.status) return TWIST_ERR_CUDA;
  const long long items = (long long)a->n_subnets * a->n_seqs * a->kv_max;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!q8) {
    switch (dh) {
      case 8: return run_evict<-1>(p, items, st);
      case 16: return run_evict<-2>(p, items, st);
      case 32: return run_evict<-4>(p, items, st);
      case 64: return run_evict<-8>(p, items, st);
      case 128: return run_evict<-16>(p, items, st);
      default: return run_evict<0>(p, items, st);
    }
  }
  switch (dh) {
    case 16: return run_evict<16>(p, items, st);
    case 32: return run_evict<32>(p, items, st);
    case 64: return run_evict<64>(p, items, st);
    default: return run_evict<128>(p, items, st);
  }
}
