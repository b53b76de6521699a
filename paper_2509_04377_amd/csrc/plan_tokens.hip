// Pages, slots and positions of the new tokens of a batch (pe_plan_tokens).
//
// With n_s tokens that sequence s brings and p_s pages that each of its rows is to get, everything follows from two exclusive prefix sums
// over the sequences, of n_s and of rows * p_s: token t belongs to the sequence whose sum brackets t, and so does dealt page p.  The sums
// are short (a batch of sequences) and what hangs on them is long (a 64-bit slot for each token and row), so every workgroup makes all
// sums by itself, kThreads sequences at a time, and writes its own share of slots and pages in between: one launch, no workgroup waits
// for another, nothing is ordered by an atomic.  Shares are pieces of kThreads tokens or pages, cut out of the sequences that have just been
// summed.  The table is written where it has no entry yet and read where it has one, so that the order of workgroups does not matter.
//
// Bound: for a step of a batch by the chain of a launch (lengths, sums, the page, the slot; 32 sequences of eight rows 4.1 us, an empty fill
// 2.3), for a batch of prompts by its stores (19 MB of slots and table 8.9 us, a fill of as many bytes 6.5).  As the admission of a cache that is pruned asks,
// with a budget, spare pages, positions and all options but copies: 32 prompts of 17 to 16384 tokens, 2048 kept, 8.1 us, without options 7.8; eight of 4096
// 5.5, 5.0; a token each 4.9.
#include "pe_device.h"
#include "pe_tokens.h"

namespace pe {
namespace {

constexpr int kThreads = kPlanThreads;
constexpr int kWaves = kThreads / kWave;

struct Sums {
  int64_t tokens, pages;
};

// Inclusive sums over the lanes of a wave of numbers of up to 31 bits: in two parts, which 32 bits hold.
__device__ __forceinline__ int64_t wave_inclusive(uint32_t v) {
  return (int64_t)wave_prefix_sum_u32(v & 0xffffffu) + ((int64_t)wave_prefix_sum_u32(v >> 24) << 24);
}

// First i in [0, n) with end[i] > x (end ascending; the last one is).
__device__ __forceinline__ int bracket(const int64_t* end, int n, int64_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (end[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

struct Seqs {  // of the sequences that have just been summed
  int64_t token_end[kThreads], page_end[kThreads];
  int32_t have[kThreads], per_row[kThreads], len[kThreads], first[kThreads];
  int8_t served[kThreads];  // 0: left as it was; 1: pages are there, its slots are not known; 2: and they are
};
struct __attribute__((aligned(16))) Token {  // of a piece: where the pages of its rows stand, `step` entries apart
  int64_t at;
  int32_t step;
  int32_t slot;  // in its page; kInTable: the pages are in the table, not among the free ones; negative: no slot
};
constexpr int kInTable = 1 << 16;

// (The leading arguments are what a workgroup waits for first: they come in registers, the others with a load.  OPTIONS: there are some; as
// questions in one kernel they cost the plans without 0.2 us of 4.3, 0.4 of 10.0.)
template <bool OPTIONS>
__global__ __launch_bounds__(kThreads) void plan_tokens_kernel(const int32_t* free_used, const int32_t* seq_lens, const int32_t* new_lens,
                                                               const int32_t* first_positions, const int num_seqs, const int num_free,
                                                               const uint32_t token_pieces, const uint32_t pieces, const uint32_t inv_rows,
                                                               const PlanArgs a) {
  __shared__ Seqs q;
  __shared__ Token tok[kThreads];
  __shared__ Sums wave_sums[kWaves];
  __shared__ int64_t dealt_of[kWaves];

  const int me = (int)threadIdx.x, wave = me / kWave, lane = lane_id();
  const int B = a.block_size, log2_block = __builtin_ctz((unsigned)B), rows = a.rows_per_seq;
  const int64_t given = *free_used;
  const int64_t used = given < 0 ? 0 : given > num_free ? num_free : given;
  // (what the list holds; of several copies, what is one's share: the sums ascend, so that a share that holds a sum holds those before it)
  const int64_t left = OPTIONS && a.copies > 1 ? (int64_t)((uint32_t)(num_free - used) / (uint32_t)a.copies) : num_free - used;
  Sums before{0, 0};
  int64_t dealt = 0;

  for (int s0 = 0; s0 < num_seqs; s0 += kThreads) {
    const int s = s0 + me, count = num_seqs - s0 < kThreads ? num_seqs - s0 : kThreads;
    int n = 0, len = 0, have = 0, per_row = 0, first = 0;
    int64_t after = 0, kept = 0;
    bool fits = false;
    if (s < num_seqs) {
      len = seq_lens[s];
      n = new_lens[s];
      n = n < 0 ? 0 : n;
      const int64_t holds = len < 0 ? 0 : len;  // (below 0: no sequence, one can begin here)
      first = first_positions != nullptr ? first_positions[s] : (int)holds;
      have = (int)((holds + B - 1) >> log2_block);
      after = holds + n;
      kept = a.budget > 0 && after > a.budget ? (holds > a.budget ? holds : a.budget) : after;
      const int64_t pages = (kept + B - 1) >> log2_block;
      fits = (len >= 0 || n > 0) && pages <= a.max_blocks && kept <= 0x7fffffffLL;
      if (OPTIONS && a.only != nullptr) fits = fits && a.only[s] != 0;
      if (fits) per_row = (int)(pages - have) + (holds == 0 && n > 0 ? a.n_spare : 0);
    }
    const int need = per_row * rows;  // (the host keeps it under 2^31)
    const int64_t t_in = wave_inclusive((uint32_t)n), p_in = wave_inclusive((uint32_t)need);
    if (s0 > 0) __syncthreads();  // (what is written below may still be read)
    if (lane == kWave - 1) wave_sums[wave] = Sums{t_in, p_in};
    __syncthreads();
    Sums off = before;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
      if (w < wave) off.tokens += wave_sums[w].tokens, off.pages += wave_sums[w].pages;
    const int64_t t_end = off.tokens + t_in, p_end = off.pages + p_in;
    const bool served = fits && (need == 0 || p_end <= left);
    q.token_end[me] = t_end;
    q.page_end[me] = p_end;
    q.have[me] = have;
    q.per_row[me] = per_row;
    q.len[me] = len < 0 ? 0 : len;
    q.served[me] = served ? (kept == after ? 2 : 1) : 0;
    q.first[me] = first;
    if (blockIdx.x == 0) {
      // the sums ascend: the last that the list holds has the most
      int64_t mine = served && p_end <= left ? p_end : 0;
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int64_t o = __shfl_xor(mine, d);
        mine = o > mine ? o : mine;
      }
      if (lane == 0) dealt_of[wave] = mine;
      if (s < num_seqs) {
        a.seq_lens_out[s] = served ? (int32_t)kept : len;
        if (OPTIONS && a.admitted != nullptr) a.admitted[s] = !served || n == 0 ? 0 : len <= 0 ? 1 : 2;
        if (a.cu_out != nullptr) {
          if (s == 0) a.cu_out[0] = 0;
          a.cu_out[s + 1] = (int32_t)(t_end < 0x7fffffffLL ? t_end : 0x7fffffffLL);
        }
      }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) dealt = dealt_of[w] > dealt ? dealt_of[w] : dealt;
    }
    if (OPTIONS && (a.spare_used != nullptr || a.freed_phys != nullptr)) {  // rows of sequences that begin: what an earlier one left
      for (int idx = (int)blockIdx.x * kThreads + me; idx < count * rows; idx += (int)gridDim.x * kThreads) {
        const int i = idx / rows;
        if (q.served[i] == 0 || q.len[i] != 0 || q.token_end[i] == (i > 0 ? q.token_end[i - 1] : before.tokens)) continue;
        if (a.spare_used != nullptr) a.spare_used[(int64_t)s0 * rows + idx] = 0;
        if (a.freed_phys != nullptr) a.freed_phys[(int64_t)s0 * rows + idx] = -1;
      }
    }
    const int64_t t_last = q.token_end[count - 1] < a.total_tokens ? q.token_end[count - 1] : a.total_tokens;
    const int64_t p_last = q.page_end[count - 1] < left ? q.page_end[count - 1] : left;

    for (uint32_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
      if (piece < token_pieces) {
        const int64_t t0 = (int64_t)piece * kThreads;
        if (t0 >= t_last || t0 + kThreads <= before.tokens) continue;
        const int64_t t = t0 + me;
        Token mine{0, 0, -1};
        if (t >= before.tokens && t < t_last) {
          const int i = bracket(q.token_end, count, t);
          const int64_t nth = t - (i > 0 ? q.token_end[i - 1] : before.tokens);
          if (a.positions_out != nullptr) a.positions_out[t] = (int32_t)((uint32_t)q.first[i] + (uint32_t)nth);
          const int64_t at = q.len[i] + nth;
          if (q.served[i] == 2) {
            const int j = (int)(at >> log2_block), more = j - q.have[i], slot = (int)at & (B - 1);
            if (more < 0)
              mine = Token{(int64_t)(s0 + i) * rows * a.max_blocks + j, a.max_blocks, slot | kInTable};
            else
              mine = Token{used + (i > 0 ? q.page_end[i - 1] : before.pages) + more, q.per_row[i], slot};
          }
        }
        if (a.slots_out == nullptr) continue;
        tok[me] = mine;
        __syncthreads();
        // a thread for each (token, row), rows side by side as they are stored
        const int begin = (int)(before.tokens > t0 ? before.tokens - t0 : 0), end = (int)(t_last - t0 < kThreads ? t_last - t0 : kThreads);
#pragma unroll 8
        for (int idx = begin * rows + me; idx < end * rows; idx += kThreads) {
          const int k = inv_rows == ~0u ? idx / rows : inv_rows != 0u ? (int)((uint64_t)(uint32_t)idx * inv_rows >> 32) : idx, h = idx - k * rows;
          const Token of = tok[k];
          int64_t slot = -1;
          if (of.slot >= 0) {
            const int32_t page = ((of.slot & kInTable) ? a.block_table : a.free_pages)[of.at + (int64_t)h * of.step];
            if (page >= 0) slot = ((int64_t)page << log2_block) + (of.slot & (kInTable - 1));
          }
          a.slots_out[t0 * rows + idx] = slot;
        }
        __syncthreads();
      } else {
        const int64_t p = (int64_t)(piece - token_pieces) * kThreads + me;
        if (p < before.pages || p >= p_last) continue;
        const int i = bracket(q.page_end, count, p);
        if (!q.served[i]) continue;
        const int per = q.per_row[i];
        const uint32_t in = (uint32_t)(p - (i > 0 ? q.page_end[i - 1] : before.pages));
        const int32_t page = a.free_pages[used + p];
        const int h = (int)(in / (uint32_t)per), j = (int)(in - (uint32_t)h * (uint32_t)per);
        const bool begins = q.len[i] == 0 && a.n_spare > 0;  // (only one that brings tokens has pages here)
        const int of_table = begins ? per - a.n_spare : per;
        const int64_t row = (int64_t)(s0 + i) * rows + h;
        if (j < of_table)
          a.block_table[row * a.max_blocks + q.have[i] + j] = page;
        else
          a.spare[row * a.n_spare + (j - of_table)] = page;
      }
    }
    before = Sums{q.token_end[count - 1], q.page_end[count - 1]};
  }

  if (blockIdx.x == 0 && me == 0) *a.free_used_out = (int32_t)(used + dealt);
  // behind the last token
  for (int64_t t = before.tokens + (int64_t)blockIdx.x * kThreads + me; t < a.total_tokens; t += (int64_t)gridDim.x * kThreads) {
    if (a.positions_out != nullptr) a.positions_out[t] = 0;
    if (a.slots_out != nullptr)
      for (int h = 0; h < rows; ++h) a.slots_out[t * rows + h] = -1;
  }
}

}  // namespace

hipError_t launch_plan_tokens(const PlanArgs& a, int compute_units, hipStream_t stream) {
  const int64_t room = (int64_t)a.num_seqs * a.rows_per_seq * (a.max_blocks + (int64_t)a.n_spare);
  const int64_t pages = room < a.num_free ? room : a.num_free;
  const bool tokens = a.positions_out != nullptr || a.slots_out != nullptr;
  const uint32_t token_pieces = tokens ? (uint32_t)((a.total_tokens + kThreads - 1) / kThreads) : 0u;
  const uint32_t pieces = token_pieces + (uint32_t)((pages + kThreads - 1) / kThreads);
  // a workgroup a piece, as many as the compute units hold at once
  const uint32_t most = 8u * (uint32_t)compute_units, groups = pieces < most ? pieces : most;
  // idx / rows is the upper half of idx * inv_rows as long as idx * rows < 2^32 (idx < kThreads * rows); ~0: divided
  const uint32_t rows = (uint32_t)a.rows_per_seq, inv_rows = rows == 1 ? 0u : rows < 4096 ? (uint32_t)((1ull << 32) / rows + 1) : ~0u;
  const bool options = a.admitted != nullptr || a.spare_used != nullptr || a.freed_phys != nullptr || a.only != nullptr || a.copies > 1;
  const auto kernel = options ? plan_tokens_kernel<true> : plan_tokens_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(groups < 1 ? 1 : groups), dim3(kThreads), 0, stream, a.free_used, a.seq_lens,
                     a.new_lens, a.first_positions, a.num_seqs, a.num_free, token_pieces, pieces, inv_rows, a);
  return hipGetLastError();
}

}  // namespace pe
