// Prompts of twist_attn_core_weights on the tensor cores, heads of 64 and 128:
//     w_j = sum_h sum_{i >= j} exp(q_hi . k_j / sqrt(d) - lse_hi).
//
// One CTA per (block of 128 keys, KV position, sequence), blocks with the most queries first.  For every kept head that reads the
// position and every block of 128 queries at or behind the keys, S^T = K Q^T (tcgen05, 128 x 128 x d, accumulators in tensor
// memory): the thread that owns lane r of tensor memory owns key r and adds up its row of exponentials in registers over all
// blocks and heads; nothing is written but the sums.  Two S^T buffers: the next block's product runs while this one's
// exponentials are taken.  Warps 0-7: exponentials (two per lane quarter, 64 queries each); warp 8, one lane: TMA and MMA issue.
// Two CTAs share an SM.
//
// Bound by the exponentials: an SM's special-function units give 16 a cycle, 1024 cycles a block, against 128 (d = 64) of MMA.
// Every wait is bounded; on expiry the CTA records TWIST_ERR_DEVICE_TIMEOUT and leaves.
#include "attn_weights.cuh"
#include "ptx.cuh"

namespace twist {
namespace {

constexpr int kBlock = 128;
constexpr int kThreads = 288;
constexpr int kTmemCols = 256;           // two S^T buffers of 128 columns
constexpr float kLog2e = 1.4426950408889634f;

__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int D>
struct Tc {
  static constexpr int PANELS = D / 64;                       // boxes of 64 columns of a block
  static constexpr int BOX = kBlock * 64 * 2, BLOCK = PANELS * BOX;
  static constexpr int STAGES = D == 64 ? 3 : 2;              // of queries
  static constexpr int SMEM = BLOCK * (1 + STAGES) + 1024 + 256;
};

// Sum over 32 columns of one row.  MASKED: columns lo <= c < hi count.
template <bool MASKED>
__device__ inline float row_sum(const uint32_t (&v)[32], uint32_t lse, float scale, int lo, int hi) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const uint4 l = lds128(lse + 4 * i);
    const float w[4] = {__uint_as_float(l.x), __uint_as_float(l.y), __uint_as_float(l.z), __uint_as_float(l.w)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float e = ex2(fmaf(__uint_as_float(v[i + j]), scale, -w[j]) * kLog2e);
      if (MASKED) e = i + j >= lo && i + j < hi ? e : 0.f;
      sum[j] += e;
    }
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// qkv viewed as [S * n_seqs][seq_len][nq]: rows past the end of a sequence read as zeros.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) core_weights_tc_kernel(const __grid_constant__ CUtensorMap map, const CoreParams p) {
  using T = Tc<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ short list[kMaxHeads];
  __shared__ int n_list_s;
  __shared__ __align__(16) float lse_w[8][64];                // per warp: its 64 queries
  __shared__ float halves[kBlock];
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
  if (threadIdx.x == 256) {
    tma_prefetch_desc(&map);
    for (int i = 0; i < N_BARS; ++i) mbar_init(bar(i), i >= S_FREE ? 8 : 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  griddep_wait();
  const int len = prompt_len(p, z);
  if (kb * kBlock >= len) return;
  if (warp == 0) {
    const int n = heads_of(p, s, pos, lane, list);
    if (lane == 0) n_list_s = n;
  }
  if (warp == 8) {
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
  if (warp == 8) {
    if (lane == 0 && total > 0) {
      auto load = [&](uint32_t to, uint32_t full, int col, int block) {
        mbar_expect_tx(full, T::BLOCK);
#pragma unroll
        for (int j = 0; j < T::PANELS; ++j) tma_load_3d_local(to + j * T::BOX, &map, full, col + 64 * j, block * kBlock, z);
      };
      int head = 0, block = i0, filled = 0;                            // of the next unit to load
      auto load_q = [&] {
        load(q_s + filled % T::STAGES * T::BLOCK, bar(Q_FULL + filled % T::STAGES), list[head] * D, block);
        ++filled;
        if (++block == i0 + per_head) { block = i0; ++head; }
      };
      load(k_s, bar(K_FULL), (p.heads + pos) * D, kb);
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
          for (int k = 0; k < 4; ++k) mma1(tmem + 128u * buf, ak + 2u * k, bq + 2u * k, idesc, (j | k) != 0);
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
    const int quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane, key = kb * kBlock + r;
    const uint32_t t_s = tmem + ((uint32_t)(quarter * 32) << 16) + 64u * half, lse_s = smem_u32(lse_w[warp]);
    // the statistics of the warp's 64 queries, one unit ahead in registers (a lane: queries lane and lane + 32 of its half)
    int head = 0, block = i0;
    float l0 = INFINITY, l1 = INFINITY;
    auto next_lse = [&] {
      l0 = l1 = INFINITY;
      if (head == n_list_s) return;
      const float* lse = p.lse + ((long long)s * p.heads + list[head]) * p.T + (long long)b * p.seq_len;
      const int q = block * kBlock + 64 * half + lane;
      if (q < len) l0 = lse[q];
      if (q + 32 < len) l1 = lse[q + 32];
      if (++block == i0 + per_head) { block = i0; ++head; }
    };
    next_lse();
    float sum = 0.f;
    bool ok = true;
    for (int n = 0, i = i0; n < total; ++n) {
      __syncwarp();                                                    // the unit before has read the staging area
      lse_w[warp][lane] = l0;
      lse_w[warp][lane + 32] = l1;
      __syncwarp();
      next_lse();
      const int buf = n & 1;
      if (!__all_sync(0xffffffffu, mbar_wait_cta(bar(S_FULL + buf), n >> 1 & 1, abort_flag, p.status))) { ok = false; break; }
      tc_fence_after();
      uint32_t va[32], vb[32];
      tc_ld32(t_s + 128u * buf, va);
      tc_ld32(t_s + 128u * buf + 32, vb);
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(S_FREE + buf));
      const int q0 = i * kBlock + 64 * half;
      if (i * kBlock < max(first, (kb + 1) * kBlock) || (i + 1) * kBlock > len) {
        const int lo = max(first, key) - q0, hi = len - q0;
        sum += row_sum<true>(va, lse_s, p.scale, lo, hi) + row_sum<true>(vb, lse_s + 128, p.scale, lo - 32, hi - 32);
      } else {
        sum += row_sum<false>(va, lse_s, p.scale, 0, 0) + row_sum<false>(vb, lse_s + 128, p.scale, 0, 0);
      }
      if (++i == i0 + per_head) i = i0;
    }
    if (half == 1) halves[r] = sum;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (half == 0 && ok && n_list_s > 0 && key < len) store_weight(p, z, pos, key, sum + halves[r]);
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    drain_after_abort(abort_flag);
    __syncthreads();
  }
  if (warp == 8) {
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

int core_weights_tc(const CoreParams& p, int d_head, cudaStream_t st) { return d_head == 64 ? run_tc<64>(p, st) : run_tc<128>(p, st); }

}  // namespace twist
