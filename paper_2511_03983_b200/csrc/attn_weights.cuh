// Parameters and pieces that the kernels of twist_attn_core_weights share (attn_weights.cu, and on the tensor cores
// attn_weights_tc.cu).
#pragma once
#include "common.cuh"

namespace twist {

struct CoreParams {
  const __nv_bfloat16* qkv;    // [S][T][nq]
  const float* lse;            // [S][heads][T]
  const int32_t *table, *new_len, *head_idx, *kv_pos;
  float* weights;
  int32_t* slot_pos;
  int S, n_seqs, seq_len, heads, kv_max, per_group, n_kv_heads, nq, T, last;
  int page_shift, n_pages, max_pages;
  float scale;
  int* status;
};

constexpr int kMaxHeads = 1024;

// The kept heads that read KV position `pos`, in ascending order, into list; returns their number.  One warp; bad entries
// are replaced by position 0 and reported.
__device__ inline int heads_of(const CoreParams& p, int s, int pos, int lane, short* list) {
  if (!p.head_idx) {
    if (lane == 0) list[0] = (short)pos;
    return 1;
  }
  int seen = 0;
  for (int h0 = 0; h0 < p.heads; h0 += 32) {
    const int hq = h0 + lane;
    bool mine = false;
    if (hq < p.heads) {
      const int h = p.head_idx[(long long)s * p.heads + hq];
      int g = h < 0 ? -1 : h / p.per_group;
      if ((unsigned)g >= (unsigned)p.n_kv_heads) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); g = 0; }
      int at = p.kv_pos[(long long)s * p.n_kv_heads + g];
      if ((unsigned)at >= (unsigned)p.kv_max) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); at = 0; }
      mine = at == pos;
    }
    const unsigned vote = __ballot_sync(0xffffffffu, mine);
    if (mine) list[seen + __popc(vote & ((1u << lane) - 1))] = (short)hq;
    seen += __popc(vote);
  }
  return seen;
}

// Tokens of sequence (s, b), checked.
__device__ inline int prompt_len(const CoreParams& p, long long seq) {
  int n = p.new_len ? p.new_len[seq] : p.seq_len;
  if (n < 0 || n > p.seq_len) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); n = n < 0 ? 0 : p.seq_len; }
  return n;
}

// Token j's sum into its page.
__device__ inline void store_weight(const CoreParams& p, long long seq, int pos, int j, float sum) {
  const int page = j >> p.page_shift, id = page < p.max_pages ? p.table[seq * p.max_pages + page] : -1;
  if ((unsigned)id >= (unsigned)p.n_pages) { atomicMin(p.status, (int)TWIST_ERR_BAD_INDEX); return; }
  const long long at = (((long long)id * p.kv_max + pos) << p.page_shift) + (j & ((1 << p.page_shift) - 1));
  p.weights[at] = sum;
  if (p.slot_pos) p.slot_pos[at] = j;
}

int core_weights_tc(const CoreParams& p, int d_head, cudaStream_t st);

}  // namespace twist
