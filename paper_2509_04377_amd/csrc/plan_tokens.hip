// Pages, slots and positions of the new tokens of a batch (pe_plan_tokens).
//
// With n_s tokens that sequence s brings and p_s pages that each of its rows is to get, everything follows from two exclusive prefix sums
// over the sequences, of n_s and of rows * p_s: token t belongs to the sequence whose sum brackets t, and so does dealt page p.  The sums
// are short (a batch of sequences) and what hangs on them is long (a 64-bit slot for each token and row), so every workgroup makes all
// sums by itself, kPlanThreads sequences at a time, and writes its own share of pages and slots in between: one launch, no workgroup waits
// for another, nothing is ordered by an atomic.  Shares are pieces of kPlanThreads tokens or pages, dealt round robin, that a workgroup cuts with
// the sequences it has just summed.  The table is written where it has no entry yet and read where it has one, so that the order
// of workgroups does not matter.
#include "pe_device.h"
#include "pe_tokens.h"

namespace pe {
namespace {

constexpr int kThreads = kPlanThreads;
constexpr int kWaves = kThreads / kWave;

struct Sums {
  int64_t tokens, pages;
};

// Inclusive sums over the lanes of a wave of numbers of up to 63 bits.
__device__ __forceinline__ int64_t wave_inclusive(int64_t v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t o = __shfl_up(v, d);
    if (lane_id() >= d) v += o;
  }
  return v;
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

// The first of this workgroup's pieces that reaches number x or lies behind it (what is dealt has fewer than 2^31 numbers; a sum
// may be larger, no piece is taken there).
__device__ __forceinline__ uint32_t first_piece(int64_t x) {
  const uint32_t p = (uint32_t)((x < 0x7fffffffLL ? x : 0x7fffffffLL) / kThreads), turn = p % gridDim.x;
  return p + (blockIdx.x >= turn ? blockIdx.x - turn : blockIdx.x + gridDim.x - turn);
}

__global__ __launch_bounds__(kThreads) void plan_tokens_kernel(const PlanArgs a) {
  __shared__ int64_t token_end[kThreads], page_end[kThreads];
  __shared__ int32_t have_of[kThreads], per_row_of[kThreads], len_of[kThreads], first_of[kThreads];
  __shared__ int8_t served_of[kThreads];  // 0: left as it was; 1: pages are there, its slots are not known; 2: and they are
  __shared__ Sums wave_sums[kWaves];
  __shared__ int64_t dealt_of[kWaves];

  const int me = (int)threadIdx.x, wave = me / kWave, lane = lane_id();
  const int B = a.block_size, log2_block = __builtin_ctz((unsigned)B), rows = a.rows_per_seq;
  const int64_t given = *a.free_used;
  const int64_t used = given < 0 ? 0 : given > a.num_free ? a.num_free : given;
  const int64_t left = a.num_free - used;
  Sums before{0, 0};
  int64_t dealt = 0;  // (thread 0's, in the end the launch's)

  for (int s0 = 0; s0 < a.num_seqs; s0 += kThreads) {
    const int s = s0 + me, count = a.num_seqs - s0 < kThreads ? a.num_seqs - s0 : kThreads;
    int64_t n = 0, need = 0;
    int len = 0, have = 0, per_row = 0;
    int64_t after = 0, kept = 0;
    bool fits = false;
    if (s < a.num_seqs) {
      len = a.seq_lens[s];
      n = a.new_lens[s];
      n = n < 0 ? 0 : n;
      const int64_t holds = len < 0 ? 0 : len;
      have = (int)((holds + B - 1) >> log2_block);
      after = holds + n;
      kept = a.budget > 0 && after > a.budget ? (holds > a.budget ? holds : a.budget) : after;
      const int64_t pages = (kept + B - 1) >> log2_block;
      fits = len >= 0 && pages <= a.max_blocks && kept <= 0x7fffffffLL;
      if (fits) per_row = (int)(pages - have) + (holds == 0 && n > 0 ? a.n_spare : 0);
      need = (int64_t)per_row * rows;
    }
    const int64_t t_in = wave_inclusive(n), p_in = wave_inclusive(need);
    __syncthreads();  // (those before may still be read)
    if (lane == kWave - 1) wave_sums[wave] = Sums{t_in, p_in};
    __syncthreads();
    Sums off = before;
    for (int w = 0; w < wave; ++w) off.tokens += wave_sums[w].tokens, off.pages += wave_sums[w].pages;
    const int64_t t_end = off.tokens + t_in, p_end = off.pages + p_in;
    const bool served = fits && (need == 0 || p_end <= left);
    token_end[me] = t_end;
    page_end[me] = p_end;
    have_of[me] = have;
    per_row_of[me] = per_row;
    len_of[me] = len;
    served_of[me] = served ? (kept == after ? 2 : 1) : 0;
    if (s < a.num_seqs) first_of[me] = a.first_positions != nullptr ? a.first_positions[s] : len;
    int64_t mine = served && p_end <= left ? p_end : 0;  // the sums ascend: the last that the list holds has the most
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int64_t o = __shfl_xor(mine, d);
      mine = o > mine ? o : mine;
    }
    if (lane == 0) dealt_of[wave] = mine;
    if (blockIdx.x == 0 && s < a.num_seqs) {
      a.seq_lens_out[s] = served ? (int32_t)kept : len;
      if (a.cu_out != nullptr) {
        if (s == 0) a.cu_out[0] = 0;
        a.cu_out[s + 1] = (int32_t)(t_end < 0x7fffffffLL ? t_end : 0x7fffffffLL);
      }
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) dealt = dealt_of[w] > dealt ? dealt_of[w] : dealt;

    // pages [before.pages, last) of the deal, those of this workgroup's pieces
    const int64_t p_last = page_end[count - 1] < left ? page_end[count - 1] : left;
    for (uint32_t piece = first_piece(before.pages); (int64_t)piece * kThreads < p_last; piece += gridDim.x) {
      const int64_t p = (int64_t)piece * kThreads + me;
      if (p < before.pages || p >= p_last) continue;
      const int i = bracket(page_end, count, p);
      if (!served_of[i]) continue;
      const int per = per_row_of[i];
      const uint32_t in = (uint32_t)(p - (i > 0 ? page_end[i - 1] : before.pages));  // (the host keeps a sequence's under 2^31)
      const int h = (int)(in / (uint32_t)per), j = (int)(in - (uint32_t)h * (uint32_t)per);
      const bool begins = len_of[i] == 0 && a.n_spare > 0;  // (only one that brings tokens has pages here)
      const int of_table = begins ? per - a.n_spare : per;
      const int64_t row = (int64_t)(s0 + i) * rows + h;
      const int32_t page = a.free_pages[used + p];
      if (j < of_table)
        a.block_table[row * a.max_blocks + have_of[i] + j] = page;
      else
        a.spare[row * a.n_spare + (j - of_table)] = page;
    }

    // tokens [before.tokens, last)
    if (a.positions_out != nullptr || a.slots_out != nullptr) {
      const int64_t t_last = token_end[count - 1] < a.total_tokens ? token_end[count - 1] : a.total_tokens;
      for (uint32_t piece = first_piece(before.tokens); (int64_t)piece * kThreads < t_last; piece += gridDim.x) {
        const int64_t t = (int64_t)piece * kThreads + me;
        if (t < before.tokens || t >= t_last) continue;
        const int i = bracket(token_end, count, t);
        const int64_t nth = t - (i > 0 ? token_end[i - 1] : before.tokens);
        if (a.positions_out != nullptr) a.positions_out[t] = (int32_t)((uint32_t)first_of[i] + (uint32_t)nth);
        if (a.slots_out == nullptr) continue;
        const int64_t at = len_of[i] + nth;
        const int j = (int)(at >> log2_block), slot = (int)at & (B - 1);
        const int64_t start = used + (i > 0 ? page_end[i - 1] : before.pages);
        for (int h = 0; h < rows; ++h) {
          int32_t page = -1;
          if (served_of[i] == 2)
            page = j < have_of[i] ? a.block_table[((int64_t)(s0 + i) * rows + h) * a.max_blocks + j]
                                  : a.free_pages[start + (int64_t)h * per_row_of[i] + (j - have_of[i])];
          a.slots_out[t * rows + h] = page < 0 ? -1 : (int64_t)page * B + slot;
        }
      }
    }
    __syncthreads();
    before = Sums{token_end[count - 1], page_end[count - 1]};
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
  // a workgroup for a piece of tokens or of pages (as many as a table could take), two a compute unit at most
  const int64_t pages = (int64_t)a.num_seqs * a.rows_per_seq * (a.max_blocks + (int64_t)a.n_spare);
  const int64_t most = pages < a.num_free ? pages : a.num_free, work = most > a.total_tokens ? most : a.total_tokens;
  int64_t groups = (work + kThreads - 1) / kThreads;
  if (groups > 2LL * compute_units) groups = 2LL * compute_units;
  if (groups < 1) groups = 1;
  hipLaunchKernelGGL(plan_tokens_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pe
