// Bookkeeping of a paged cache on the GPU (fier_block_table): which pool blocks every sequence gets or gives back when its
// length changes, where each of the new tokens goes, and the packed offsets of the new tokens.
//   held(x) = ceil(x / block_tokens).  Sequence b gives back give_b = max(0, held(old_b) - held(new_b)) blocks and takes
// take_b = max(0, held(new_b) - held(old_b)).  The free blocks are a stack S of n; the blocks given back, sequences and entries
// ascending, go on top of it (R in all), then the k-th block taken, in the same order, is S[n + R - 1 - k] (T in all).
// starts and the places in both orders are exclusive sums over the sequences.
#include "fier_dev.h"
#include "fier_kernels.h"

namespace fier {

constexpr int kTableEntries = 256;  // entries of a sequence per workgroup, one for each thread

// Grid (batch, ceil(entries / 256)), block 256, batch words of dynamic LDS.  Every workgroup forms the sums it needs from all
// lengths by itself (two coalesced words per sequence), so that one launch does it and nothing is handed over: a workgroup
// takes a block that another sequence gives back in this call from that sequence's old entries, which no workgroup changes.
// Entries of the table are written only past a growing sequence's old ones and places of the stack only from n on, while only
// those below n are read: the call can be repeated on its own results.
//   Too few blocks: the calls enqueued behind this one must not write through entries that nobody filled, so all offsets become
// starts[0], which only this case reads and no case but a successful one writes: then no sequence has new tokens.  A negative
// counter says the same of the call before: it is passed on, not taken for an empty stack.
__global__ __launch_bounds__(256) void block_table_kernel(int shift, int max_ctx, int batch, const int32_t* __restrict__ old_lens,
                                                          const int32_t* __restrict__ new_lens, int32_t* table,
                                                          int32_t* free_blocks, int n_blocks,
                                                          const int32_t* __restrict__ n_free, int32_t* __restrict__ n_free_out,
                                                          int32_t* __restrict__ starts, int32_t* __restrict__ slots, int n_slots) {
  extern __shared__ uint32_t give_at[];  // [batch] blocks given back by the sequences in front
  __shared__ uint32_t part[5][4], tmp[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, entries = max_ctx >> shift;
  const int round_up = (1 << shift) - 1;
  auto clamped = [&](int len) { return max(0, min(len, max_ctx)); };
  auto held = [&](int len) { return (len + round_up) >> shift; };
  // sums over the sequences in front of this one (take, give, tokens) and over all (take, give)
  uint32_t sum[5] = {0, 0, 0, 0, 0};
  for (int i = tid; i < batch; i += 256) {
    const int o = clamped(old_lens[i]), w = clamped(new_lens[i]), d = held(w) - held(o);
    const uint32_t take = (uint32_t)max(0, d), give = (uint32_t)max(0, -d);
    sum[3] += take, sum[4] += give;
    if (i < b) sum[0] += take, sum[1] += give, sum[2] += (uint32_t)max(0, w - o);
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    const uint32_t s = wave_sum_u32(sum[k]);
    if (lane == 0) part[k][wave] = s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 5; ++k) sum[k] = part[k][0] + part[k][1] + part[k][2] + part[k][3];
  const int take_before = (int)sum[0], give_before = (int)sum[1], tok_before = (int)sum[2];
  const int T = (int)sum[3], R = (int)sum[4], n = min(*n_free, n_blocks), left = n < 0 ? n : n + R - T;
  if (b == 0 && blockIdx.y == 0 && tid == 0) *n_free_out = left;
  if (left < 0) {
    if (starts && blockIdx.y == 0 && tid == 0) {
      const int none = starts[0];
      if (b > 0) starts[b] = none;
      if (b == batch - 1) starts[batch] = none;
    }
    return;
  }
  const int o = clamped(old_lens[b]), w = clamped(new_lens[b]);
  if (starts && blockIdx.y == 0 && tid == 0) {
    starts[b] = tok_before;
    if (b == batch - 1) starts[batch] = tok_before + max(0, w - o);
  }
  const int e0 = (int)blockIdx.y * kTableEntries, e = e0 + tid;
  const int have = held(o), want = held(w);
  if (e0 >= max(have, want)) return;
  int32_t* const row = table + (size_t)b * entries;
  if (want > have) {
    if (e0 + kTableEntries > have && take_before < R) {  // some of its blocks may be ones given back: where do they lie
      uint32_t before = 0;
      for (int i0 = 0; i0 < batch; i0 += 256) {
        const int i = i0 + tid;
        const uint32_t give = i < batch ? (uint32_t)max(0, held(clamped(old_lens[i])) - held(clamped(new_lens[i]))) : 0u;
        uint32_t total;
        const uint32_t at = block_excl_scan_u32<4>(give, tmp, total);
        if (i < batch) give_at[i] = before + at;
        before += total;
      }
      __syncthreads();
    }
    if (e >= have && e < want) {
      const int k = take_before + e - have;
      if (k >= R) {
        row[e] = free_blocks[n - 1 - (k - R)];
      } else {
        const uint32_t i = (uint32_t)(R - 1 - k);  // the last sequence whose first block is at or before place i gave it
        int lo = 0, hi = batch;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (give_at[mid] <= i) lo = mid;
          else hi = mid;
        }
        row[e] = table[(size_t)lo * entries + held(clamped(new_lens[lo])) + (int)(i - give_at[lo])];
      }
    }
  } else if (e >= want && e < have) {
    const int p = give_before + e - want;  // the first R - T given back stay on the stack
    if (p < R - T && n + p < n_blocks) free_blocks[n + p] = row[e];
  }
  if (!slots || w <= o) return;
  __syncthreads();  // the entries written above
  const int from = max(o, e0 << shift), to = min(w, (e0 + kTableEntries) << shift);
  for (int pos = from + tid; pos < to; pos += 256) {
    const int at = tok_before + pos - o;
    if (at < n_slots) slots[at] = (row[pos >> shift] << shift) + (pos & round_up);
  }
}

hipError_t launch_block_table(int block_shift, int max_ctx, int batch, const int32_t* old_lens, const int32_t* new_lens,
                              int32_t* table, int32_t* free_blocks, int n_blocks, const int32_t* n_free, int32_t* n_free_out,
                              int32_t* starts, int32_t* slots, int n_slots, hipStream_t st) {
  const int entries = max_ctx >> block_shift;
  const dim3 grid((unsigned)batch, (unsigned)((entries + kTableEntries - 1) / kTableEntries));
  block_table_kernel<<<grid, 256, (size_t)batch * sizeof(uint32_t), st>>>(block_shift, max_ctx, batch, old_lens, new_lens, table,
                                                                          free_blocks, n_blocks, n_free, n_free_out, starts,
                                                                          slots, n_slots);
  return hipGetLastError();
}

}  // namespace fier
