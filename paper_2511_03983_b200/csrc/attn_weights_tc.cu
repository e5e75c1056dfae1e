// Prompts of twist_attn_core_weights on the tensor cores, heads of 16 to 128:
//     w_j = sum_h sum_{i >= j} exp(q_hi . k_j / sqrt(d) - lse_hi).
//
// One CTA per (block of 128 keys, KV position, sequence), blocks with the most queries first.  For every kept head that reads the
// position and every block of 128 queries at or behind the keys, S^T = K Q^T (tcgen05, 128 x 128 x d, accumulators in tensor
// memory): the thread that owns lane r of tensor memory owns key r and adds up its row of exponentials in registers over all
// blocks and heads; nothing is written but the sums.  Two S^T buffers: the next block's product runs while this one's
// exponentials are taken.  Warps 0-7: exponentials (two per lane quarter, 64 queries each); warp 8, one lane: TMA and MMA issue.
// Two CTAs share an SM.
//
// Bound by the exponentials: an SM's special-function units give 16 a cycle, 1024 cycles a block, against 128 (d = 64) of MMA,
// and by the instructions beside them.  4 subnets of 4 prompts of 2048, 16 heads on 4 positions of d = 64 (130 us of special-function
// unit): 531 us with warp-level MMA from shared memory, 192 us first on tcgen05, 172 with the log-sum-exps staged for eight blocks
// at a time instead of for each, 162 with every fourth pair of exponentials by a polynomial (half of them: more instructions
// than the unit has to spare), 160 without the columns that count for no key of a warp (64 prompts of up to 1000, the last 32
// queries of 32 heads: 100 us before, 67).  Sixteen warps of 32 queries each: 182.  Statistics staged for eight blocks across heads:
// 172.  Smaller heads take as long: 159 at d = 32, 157 at 16.
// Every wait is bounded; on expiry the CTA records TWIST_ERR_DEVICE_TIMEOUT and leaves.
#include <type_traits>

#include "attn_weights.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kBlock = 128;
constexpr int kParts = 2, kCols = kBlock / kParts, kEw = 4 * kParts;      // warps to a lane quarter, columns of each
constexpr int kThreads = 32 * (kEw + 1);
constexpr int kChunk = 8;                // blocks of a head whose log-sum-exps are staged together
constexpr int kTmemCols = 256;           // two S^T buffers of 128 columns
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPolyPairs = 1;            // of four pairs of exponentials, how many are taken without the special-function unit

__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int D>
struct Tc {
  static constexpr int PANELS = D > 64 ? D / 64 : 1;          // boxes of 64 columns of a block (small heads: their neighbours come along)
  static constexpr int STEPS = (D > 64 ? 64 : D) / 16;        // of the product, in a panel
  static constexpr int BOX = kBlock * 64 * 2, BLOCK = PANELS * BOX;
  static constexpr int STAGES = D <= 64 ? 3 : 2;              // of queries
  static constexpr int SMEM = BLOCK * (1 + STAGES) + 1024 + 256;
};

// Two fp32 numbers at a time: half the issue slots.
using f32x2 = unsigned long long;
__device__ inline f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ inline void split(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ inline f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ inline f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Barrier of the exponential warps; whether any of their threads says so.
__device__ inline bool sync_any(bool mine) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"((uint32_t)mine), "n"(32 * kEw) : "memory");
  return r != 0;
}
// 2^t without the special-function unit, t a number and t <= 64 or so: t = n + f with n whole and |f| <= 1/2, 2^f by the polynomial
// of degree 5 of least relative error there (7.5e-8, by Remez exchange), n into the exponent.  What is below 2^-126 comes out as
// 2^-126.
__device__ inline f32x2 exp2_poly(f32x2 t) {
  float a, b;
  split(t, a, b);
  t = pair(fmaxf(a, -126.f), fmaxf(b, -126.f));
  const f32x2 magic = pair(12582912.f, 12582912.f), z = add2(t, magic);            // 1.5 * 2^23: the sum's low bits are n
  const f32x2 f = add2(t, mul2(add2(z, pair(-12582912.f, -12582912.f)), pair(-1.f, -1.f)));
  f32x2 y = fma2(pair(1.32764721678e-3f, 1.32764721678e-3f), f, pair(9.67554133102e-3f, 9.67554133102e-3f));
  y = fma2(y, f, pair(5.55071327288e-2f, 5.55071327288e-2f));
  y = fma2(y, f, pair(2.40221197240e-1f, 2.40221197240e-1f));
  y = fma2(y, f, pair(6.93146967065e-1f, 6.93146967065e-1f));
  y = fma2(y, f, pair(1.00000007165f, 1.00000007165f));
  float ya, yb, za, zb;
  split(y, ya, yb);
  split(z, za, zb);
  return pair(__int_as_float(__float_as_int(ya) + (__float_as_int(za) << 23)), __int_as_float(__float_as_int(yb) + (__float_as_int(zb) << 23)));
}

// Adds 16 columns of one row to the sums; `lse` holds their log-sum-exps, negated.  MASKED: columns lo <= c < hi count.
template <bool MASKED>
__device__ inline void add_row(f32x2 (&sum)[4], const uint32_t (&v)[16], const float* lse, float scale, int lo, int hi) {
  const f32x2 scale2 = pair(scale, scale), log2e2 = pair(kLog2e, kLog2e);
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    const float4 l = *reinterpret_cast<const float4*>(lse + i);
    const f32x2 w[2] = {pair(l.x, l.y), pair(l.z, l.w)};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = i + 2 * j;
      const f32x2 t = mul2(fma2(pair(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), scale2, w[j]), log2e2);
      f32x2 e;
      if (!MASKED && c / 2 % 4 < kPolyPairs) {
        e = exp2_poly(t);
      } else {
        float a, b;
        split(t, a, b);
        a = ex2(a);
        b = ex2(b);
        if (MASKED) {
          a = c >= lo && c < hi ? a : 0.f;
          b = c + 1 >= lo && c + 1 < hi ? b : 0.f;
        }
        e = pair(a, b);
      }
      sum[c / 2 % 4] = add2(sum[c / 2 % 4], e);
    }
  }
}

// qkv viewed as [S * n_seqs][seq_len][nq]: rows past the end of a sequence read as zeros.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) core_weights_tc_kernel(const __grid_constant__ CUtensorMap map, const CoreParams p) {
  using T = Tc<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ short list[kMaxHeads];
  __shared__ int n_list_s;
  __shared__ __align__(16) float lse_s[2][kChunk * kBlock];   // negated log-sum-exps of the queries of a chunk and the next
  __shared__ float sums[kParts][kBlock];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t k_s = base, q_s = base + T::BLOCK, bar0 = q_s + T::STAGES * T::BLOCK;
  volatile uint32_t* ctrl = reinterpret_cast<volatile uint32_t*>(gen + (1 + T::STAGES) * T::BLOCK);
  enum { K_FULL = 0, Q_FULL = 1, Q_FREE = 1 + T::STAGES, S_FULL = 1 + 2 * T::STAGES, S_FREE = S_FULL + 2, N_BARS = S_FREE + 2 };
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile uint32_t* tmem_slot = ctrl + 32;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 33);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned items = (unsigned)p.S * p.n_seqs * p.kv_max, item = blockIdx.x % items;
  const int kb = (int)(blockIdx.x / items), pos = (int)(item % p.kv_max), z = (int)(item / p.kv_max), s = z / p.n_seqs, b = z - s * p.n_seqs;
  if (threadIdx.x == 32 * kEw) {
    tma_prefetch_desc(&map);
    for (int i = 0; i < N_BARS; ++i) mbar_init(bar(i), i >= S_FREE ? kEw : 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  griddep_wait();
  if (warp == 0) {                         // beside the round trip of the length
    const int n = heads_of(p, s, pos, lane, list);
    if (lane == 0) n_list_s = n;
  }
  const int len = prompt_len(p, z);
  if (kb * kBlock >= len) return;
  auto load = [&](uint32_t to, uint32_t full, int col, int block) {
    mbar_expect_tx(full, T::BLOCK);
#pragma unroll
    for (int j = 0; j < T::PANELS; ++j) tma_load_3d_local(to + j * T::BOX, &map, full, col + 64 * j, block * kBlock, z);
  };
  if (threadIdx.x == 32 * kEw) load(k_s, bar(K_FULL), (p.heads + pos) * D, kb);
  if (warp == kEw) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"((uint32_t)kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch_dependents();             // not before the allocation: what is launched next may take tensor memory and wait for this grid
  const uint32_t tmem = *tmem_slot;
  const int first = max(kb * kBlock, p.last ? len - p.last : 0);       // the first query that counts
  const int i0 = first / kBlock, per_head = (len + kBlock - 1) / kBlock - i0, total = n_list_s * per_head;
  if (warp == kEw) {
    if (lane == 0) {                       // also without heads: the keys are on their way
      int head = 0, block = i0, filled = 0;                            // of the next unit to load
      auto load_q = [&] {
        load(q_s + filled % T::STAGES * T::BLOCK, bar(Q_FULL + filled % T::STAGES), list[head] * D, block);
        ++filled;
        if (++block == i0 + per_head) { block = i0; ++head; }
      };
      while (filled < T::STAGES && filled < total) load_q();
      constexpr uint32_t idesc = idesc_bf16(0, 0, kBlock, kBlock);     // S^T = K Q^T, both K-major
      bool ok = mbar_wait_cta(bar(K_FULL), 0, abort_flag, p.status);
      for (int n = 0; ok && n < total; ++n) {
        const int st = n % T::STAGES, buf = n & 1;
        if (!mbar_wait_cta(bar(Q_FULL + st), n / T::STAGES & 1, abort_flag, p.status)) break;
        if (n >= 2 && !mbar_wait_cta(bar(S_FREE + buf), (n >> 1) - 1 & 1, abort_flag, p.status)) break;
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < T::PANELS; ++j) {
          const uint64_t ak = smem_desc(k_s + j * T::BOX, 16u, 1024u), bq = smem_desc(q_s + st * T::BLOCK + j * T::BOX, 16u, 1024u);
#pragma unroll
          for (int k = 0; k < T::STEPS; ++k) mma1(tmem + 128u * buf, ak + 2u * k, bq + 2u * k, idesc, (j | k) != 0);
        }
        commit1(bar(S_FULL + buf));
        commit1(bar(Q_FREE + st));
        // the unit before this one is done with its queries
        if (n > 0 && filled < total) {
          const int old = (n - 1) % T::STAGES;
          if (!mbar_wait_cta(bar(Q_FREE + old), (n - 1) / T::STAGES & 1, abort_flag, p.status)) break;
          load_q();
        }
      }
    }
  } else {
    const int quarter = warp & 3, part = warp >> 2, r = quarter * 32 + lane, key = kb * kBlock + r;
    const uint32_t t_s = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(kCols * part);
    constexpr int STAGED = kChunk * kBlock / (32 * kEw);                 // of a chunk, by a thread
    float ahead[STAGED];
    auto fetch = [&](int head, int c0) {                                 // of the chunk that begins at block c0
      if (head >= n_list_s) return;
      const float* lse = p.lse + ((long long)s * p.heads + list[head]) * p.T + (long long)b * p.seq_len + c0 * kBlock;
#pragma unroll
      for (int j = 0; j < STAGED; ++j) {
        const int q = 32 * kEw * j + threadIdx.x;
        ahead[j] = c0 * kBlock + q < len ? -lse[q] : 0.f;
      }
    };
    bool odd;                                                            // a log-sum-exp that is not finite: the polynomial is not for those
    auto stage = [&](int to) {
      odd = false;
#pragma unroll
      for (int j = 0; j < STAGED; ++j) {
        lse_s[to][32 * kEw * j + threadIdx.x] = ahead[j];
        odd |= !(fabsf(ahead[j]) < INFINITY);
      }
    };
    fetch(0, i0);
    stage(0);
    float sum = 0.f;
    bool ok = true;
    const int end = i0 + per_head;
    int n = 0, chunk = 0;
    for (int head = 0, c0 = i0; head < n_list_s; ++chunk) {           // a warp that gave up still meets the others
      // the chunk's statistics are there, and nobody reads those of the one before
      const bool plain = !sync_any(odd);
      const int last = min(c0 + kChunk, end), next_c0 = last == end ? i0 : last, next_head = head + (last == end);
      fetch(next_head, next_c0);
      const float* lse = lse_s[chunk & 1] + kCols * part;
      for (int i = c0; ok && i < last; ++i, ++n, lse += kBlock) {
        const int buf = n & 1;
        if (!__all_sync(0xffffffffu, mbar_wait_cta(bar(S_FULL + buf), n >> 1 & 1, abort_flag, p.status))) { ok = false; break; }
        tc_fence_after();
        // 16 columns at a time, the next ones on their way out of tensor memory
        const uint32_t from = t_s + 128u * buf;
        f32x2 sum4[4] = {0, 0, 0, 0};
        auto unit = [&](auto masked) {
          constexpr bool MASKED = decltype(masked)::value;
          const int q0 = i * kBlock + kCols * part, lo = max(first, key) - q0, hi = len - q0, least = max(first, kb * kBlock + quarter * 32) - q0;
          auto live = [&](int c) { return !MASKED || (c + 16 > least && c < hi); };      // some of them count for a key of the warp
          uint32_t va[16], vb[16];
          tc_ld16(from, va);
          tc_wait_ld();
#pragma unroll
          for (int c = 0; c < kCols; c += 32) {
            tc_ld16(from + c + 16, vb);
            if (live(c)) add_row<MASKED>(sum4, va, lse + c, p.scale, lo - c, hi - c);
            tc_wait_ld();
            if (c + 32 < kCols) {
              tc_ld16(from + c + 32, va);
            } else {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(S_FREE + buf));
            }
            if (live(c + 16)) add_row<MASKED>(sum4, vb, lse + c + 16, p.scale, lo - c - 16, hi - c - 16);
            if (c + 32 < kCols) tc_wait_ld();
          }
        };
        if (!plain || i * kBlock < max(first, (kb + 1) * kBlock) || (i + 1) * kBlock > len) unit(std::true_type{});
        else unit(std::false_type{});
        float x, y;
        split(add2(add2(sum4[0], sum4[1]), add2(sum4[2], sum4[3])), x, y);
        sum += x + y;
      }
      stage(chunk + 1 & 1);
      head = next_head;
      c0 = next_c0;
    }
    sums[part][r] = sum;
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kEw) : "memory");
    if (part == 0 && ok && n_list_s > 0 && key < len) {
#pragma unroll
      for (int j = 1; j < kParts; ++j) sum += sums[j][r];
      store_weight(p, z, pos, key, sum);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    drain_after_abort(abort_flag);
    __syncthreads();
  }
  if (warp == kEw) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kTmemCols) : "memory");
  }
}

template <int D>
int run_tc(const CoreParams& p, cudaStream_t st) {
  const unsigned long long dims[3] = {(unsigned long long)p.nq, (unsigned long long)p.seq_len, (unsigned long long)p.S * p.n_seqs};
  const unsigned long long strides[2] = {(unsigned long long)p.nq * 2, (unsigned long long)p.seq_len * p.nq * 2};
  const unsigned box[3] = {64, kBlock, 1};
  CUtensorMap map;
  const int rc = encode_map_3d_bf16(&map, p.qkv, dims, strides, box, 128);
  if (rc != TWIST_OK) return rc;
  const long long grid = (long long)p.S * p.n_seqs * p.kv_max * ((p.seq_len + kBlock - 1) / kBlock);
  if (grid > 0x7fffffffll) return TWIST_ERR_UNSUPPORTED;
  static bool ready[64] = {false};
  const int slot = device_slot();
  if (!ready[slot]) {
    TWIST_CUDA_TRY(cudaFuncSetAttribute(core_weights_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tc<D>::SMEM));
    ready[slot] = true;
  }
  TWIST_CUDA_TRY(launch_overlapped(core_weights_tc_kernel<D>, dim3((unsigned)grid), dim3(kThreads), Tc<D>::SMEM, st, 1, map, p));
  return TWIST_OK;
}

}  // namespace

int core_weights_tc(const CoreParams& p, int d_head, cudaStream_t st) {
  switch (d_head) {
    case 16: return run_tc<16>(p, st);
    case 32: return run_tc<32>(p, st);
    case 64: return run_tc<64>(p, st);
    default: return run_tc<128>(p, st);
  }
}

}  // namespace twist
