// The bookkeeping of a paged cache on the device: room for new tokens (block tables, slot map, cumulative
// lengths) and the way back of pages.
//
// Both are a prefix sum over the sequences (how many tokens, how many pages) and, behind it, one independent item
// per token or page: which sequence it belongs to is the first whose running sum exceeds its number, found by bisection in
// LDS.  Every block works the whole prefix sum out again (4 KB of input for 512 sequences) rather than wait for
// one that does: the calls are a few microseconds of latency, not of bytes, and a second launch costs more than
// the sum.  What a block reads of the state no other block writes, so that one launch does; only where the state
// is brought forward in place and more than one block is at work does a second, of one block, write the state.
#include <algorithm>

#include "tq_internal.h"

namespace tq {
namespace {

struct PagesParams {
  const int32_t* lens;        // [batch]
  const int32_t* ask;         // [batch]: new tokens (append), or tokens to keep (trim)
  int32_t* table;             // [batch][max_blocks]
  int32_t* stack;             // [n_pages]: free pages
  const int32_t* n_free;
  int32_t* lens_after;
  int32_t* n_free_after;
  int32_t* cu_seqlens;        // append only, as are the two below
  int32_t* slots;
  int32_t* served;
  int32_t batch, max_blocks, n_pages, page_tokens, bound;   // bound: max_new_tokens
  int32_t outputs, state;     // what this launch writes: everything but the two *_after arrays; those
  int32_t vector;             // slots is aligned to 16 bytes
};

constexpr int kThreads = 256, kManyThreads = 1024;

// a + b, or `most` where that is less (both at most `most` < 2^31: no wrap)
__device__ __forceinline__ uint32_t add_upto(uint32_t a, uint32_t b, uint32_t most) { return min(a + b, most); }

// Inclusive prefix sum of x over the block's threads on top of `carry` (sums stop at `most`), which becomes the sum of all.
// wave_sums: one word per wave, free again behind the caller's next barrier.
__device__ inline uint32_t block_scan(uint32_t x, uint32_t most, uint32_t* wave_sums, uint32_t& carry) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if (!__any(x > (1u << 24))) {                     // (64 of them cannot pass 2^31: plain sums)
    x = min((uint32_t)wave_scan((int)x), most);
  } else {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t y = __shfl_up(x, off);
      if (lane >= off) x = add_upto(x, y, most);
    }
  }
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  uint32_t before = carry, all = carry;
  for (int w = 0; w < waves; ++w) {
    const uint32_t y = wave_sums[w];
    if (w < wave) before = add_upto(before, y, most);
    all = add_upto(all, y, most);
  }
  carry = all;
  return add_upto(before, x, most);
}

// the first i with sums[i] > x, or n
__device__ __forceinline__ int first_above(const uint32_t* sums, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t page_tokens) { return (tokens + page_tokens - 1) / page_tokens; }

// RUN: neighbouring tokens (or pages) that a thread takes.  Many tokens: four, mostly of one sequence and page, with one search and one
// look-up; a decode step has one token to a sequence, and wants a thread for each.
template <int RUN>
__global__ __launch_bounds__(kManyThreads) void pages_append_kernel(PagesParams p) {
  extern __shared__ uint32_t lds[];
  uint32_t* const ends = lds;                       // tokens asked for up to and with sequence b, at most bound + 1
  uint32_t* const takes = lds + p.batch;            // pages likewise, at most n_pages + 1
  int32_t* const haves = reinterpret_cast<int32_t*>(lds + 2 * p.batch);   // tokens held; ~ of that where not served
  __shared__ uint32_t sums[2][kManyThreads / 64];
  __shared__ uint32_t taken_sh;
  const uint32_t P = p.page_tokens, bound = p.bound;
  const uint32_t nf = min(max(*p.n_free, 0), p.n_pages);
  const int64_t room = min((int64_t)p.max_blocks * P, (int64_t)INT32_MAX);   // (lengths are int32)
  if (threadIdx.x == 0) taken_sh = 0;
  uint32_t c0 = 0, c1 = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    uint32_t have = 0, want = 0;
    if (b < p.batch) {
      have = max(p.lens[b], 0);
      want = max(p.ask[b], 0);
    }
    const uint32_t end = block_scan(min(want, bound + 1), bound + 1, sums[0], c0);
    // (A sequence that passes the bound keeps its pages in the running sum here: all behind it that ask for a
    // token pass the bound as well, so that nobody is kept from being served by it.)
    const bool holds = (int64_t)have + want <= room;
    const uint32_t held = pages_of(have, P);
    const uint32_t need = holds ? pages_of(have + want, P) - held : 0;
    const uint32_t take = block_scan(min(need, (uint32_t)p.n_pages + 1), (uint32_t)p.n_pages + 1, sums[1], c1);
    if (b < p.batch) {
      const bool served = holds && (want == 0 || end <= bound) && (need == 0 || take <= nf);
      ends[b] = end;
      takes[b] = take;
      haves[b] = served ? (int32_t)have : ~(int32_t)have;
      if (served && need) atomicMax(&taken_sh, take);
    }
    __syncthreads();
  }
  const uint32_t taken = taken_sh;
  if (p.outputs) {
    const uint32_t stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
    if (blockIdx.x == 0) {
      for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
        p.cu_seqlens[b + 1] = (int32_t)min(ends[b], bound);
        p.served[b] = haves[b] >= 0;
      }
      if (threadIdx.x == 0) p.cu_seqlens[0] = 0;
    }
    for (uint32_t j = first; j < taken; j += stride) {           // page j from the stack's top
      const int b = first_above(takes, p.batch, j);
      const uint32_t held = pages_of((uint32_t)haves[b], P);      // (a page that is taken belongs to a sequence that is served)
      p.table[(int64_t)b * p.max_blocks + held + (j - (b ? takes[b - 1] : 0))] = p.stack[nf - 1 - j];
    }
    for (uint32_t t0 = first * RUN; t0 < bound; t0 += stride * RUN) {
      int b = first_above(ends, p.batch, t0), of = -1;
      uint32_t page_at = 0, taken_before = 0, shift = 0;        // of sequence `of`: its page in `page`; pages in front of its; position less token
      int32_t have = -1, page = -1, slot[RUN];
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        const uint32_t t = t0 + i;
        slot[i] = -1;
        if (RUN > 1) while (b < p.batch && ends[b] <= t) ++b;
        if (b >= p.batch) continue;
        bool other = b != of;
        if (other) {
          of = b;
          have = haves[b];
          shift = (uint32_t)have - (b ? ends[b - 1] : 0);
          taken_before = b ? takes[b - 1] : 0;
        }
        if (have < 0) continue;
        const uint32_t pos = shift + t, block = pos / P, held = pages_of(have, P);
        if (other || block != page_at) {
          page_at = block;
          page = block < held ? p.table[(int64_t)b * p.max_blocks + block] : p.stack[nf - 1 - (taken_before + block - held)];
        }
        if ((uint32_t)page < (uint32_t)p.n_pages) slot[i] = page * (int32_t)P + (int32_t)(pos - block * P);
      }
      if (RUN == 4 && p.vector && t0 + RUN <= bound) {
        *reinterpret_cast<int4*>(p.slots + t0) = make_int4(slot[0], slot[1 % RUN], slot[2 % RUN], slot[3 % RUN]);
      } else {
#pragma unroll
        for (int i = 0; i < RUN; ++i)
          if (t0 + i < bound) p.slots[t0 + i] = slot[i];
      }
    }
  }
  if (p.state && blockIdx.x == 0) {
    for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
      const int32_t have = haves[b];
      p.lens_after[b] = have >= 0 ? have + (int32_t)(ends[b] - (b ? ends[b - 1] : 0)) : ~have;
    }
    if (threadIdx.x == 0) *p.n_free_after = (int32_t)(nf - taken);
  }
}

template <int RUN>
__global__ __launch_bounds__(kManyThreads) void pages_trim_kernel(PagesParams p) {
  extern __shared__ uint32_t lds[];
  uint32_t* const backs = lds;                      // pages given back up to and with sequence b, at most n_pages + 1
  uint32_t* const lefts = lds + p.batch;            // pages sequence b keeps
  int32_t* const keeps = reinterpret_cast<int32_t*>(lds + 2 * p.batch);   // tokens it keeps
  __shared__ uint32_t sums[kManyThreads / 64];
  const uint32_t P = p.page_tokens;
  const uint32_t nf = min(max(*p.n_free, 0), p.n_pages), space = p.n_pages - nf;
  uint32_t carry = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    uint32_t have = 0, keep = 0, back = 0, left = 0;
    if (b < p.batch) {
      have = max(p.lens[b], 0);
      keep = min((uint32_t)max(p.ask[b], 0), have);
      const uint32_t held = min(pages_of(have, P), (uint32_t)p.max_blocks);
      left = min(pages_of(keep, P), held);
      back = held - left;
    }
    const uint32_t through = block_scan(min(back, (uint32_t)p.n_pages + 1), (uint32_t)p.n_pages + 1, sums, carry);
    if (b < p.batch) {
      backs[b] = through;
      lefts[b] = left;
      keeps[b] = keep;
    }
    __syncthreads();
  }
  const uint32_t returned = min(carry, space);
  if (p.outputs) {
    const uint32_t stride = gridDim.x * blockDim.x;
    for (uint32_t j0 = (blockIdx.x * blockDim.x + threadIdx.x) * RUN; j0 < returned; j0 += stride * RUN) {
      int b = first_above(backs, p.batch, j0);
      int32_t page[RUN];
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        const uint32_t j = min(j0 + i, returned - 1);
        if (RUN > 1) while (backs[b] <= j) ++b;       // (ends: the last sum is more than j)
        page[i] = p.table[(int64_t)b * p.max_blocks + lefts[b] + (j - (b ? backs[b - 1] : 0))];
      }
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (j0 + i < returned) p.stack[nf + j0 + i] = page[i];
    }
  }
  if (p.state && blockIdx.x == 0) {
    for (int b = threadIdx.x; b < p.batch; b += blockDim.x) p.lens_after[b] = keeps[b];
    if (threadIdx.x == 0) *p.n_free_after = (int32_t)(nf + returned);
  }
}

PagesParams params_of(const tq_page_state& st, const int32_t* ask, int32_t* lens_after, int32_t* n_free_after) {
  PagesParams p{};
  p.lens = st.seq_lens;
  p.ask = ask;
  p.table = st.block_table;
  p.stack = st.free_pages;
  p.n_free = st.n_free;
  p.lens_after = lens_after;
  p.n_free_after = n_free_after;
  p.batch = st.batch;
  p.max_blocks = st.max_blocks;
  p.n_pages = st.n_pages;
  p.page_tokens = st.page_tokens;
  return p;
}

// One launch; in place with more than `alone` items, which one block would take long over, two.  us of the kernel, one item to a thread /
// four: room for a decode step of 256 sequences 4.4 / 6.2, for 90 thousand tokens of prompts 7.8 / 6.2; pages back of 64 sequences that lose a
// few tokens 2.5 / 3.9, 45 thousand pages 6.6 / 4.8.
constexpr int64_t kMany = 4096;                     // items from which a thread takes four
hipError_t launch_pages(void (*kernel)(PagesParams), void (*kernel4)(PagesParams), PagesParams p, int64_t items, int64_t alone, hipStream_t s) {
  const bool in_place = p.lens_after == p.lens || p.n_free_after == p.n_free, many = items > kMany;
  const size_t lds = (size_t)3 * p.batch * sizeof(uint32_t);
  if (many) kernel = kernel4;
  p.outputs = 1;
  if (in_place && items <= alone) {
    p.state = 1;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(items <= kThreads ? kThreads : kManyThreads), lds, s, p);
    return hipGetLastError();
  }
  p.state = !in_place;
  const int64_t per_block = kThreads * (many ? 4 : 1);
  const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>(512, (items + per_block - 1) / per_block));
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), lds, s, p);
  if (in_place) {
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    p.outputs = 0;
    p.state = 1;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(kThreads), lds, s, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_append(const tq_page_state& st, const int32_t* new_lens, int32_t max_new_tokens, int32_t* lens_after,
                               int32_t* n_free_after, int32_t* cu_seqlens, int32_t* slots, int32_t* served, hipStream_t s) {
  PagesParams p = params_of(st, new_lens, lens_after, n_free_after);
  p.cu_seqlens = cu_seqlens;
  p.slots = slots;
  p.served = served;
  p.bound = max_new_tokens;
  p.vector = (reinterpret_cast<uintptr_t>(slots) & 15) == 0;
  return launch_pages(pages_append_kernel<1>, pages_append_kernel<4>, p, max_new_tokens, 4096, s);
}

hipError_t launch_pages_trim(const tq_page_state& st, const int32_t* keep_lens, int32_t* lens_after, int32_t* n_free_after,
                             hipStream_t s) {
  const PagesParams p = params_of(st, keep_lens, lens_after, n_free_after);
  return launch_pages(pages_trim_kernel<1>, pages_trim_kernel<4>, p, std::min<int64_t>((int64_t)st.batch * st.max_blocks, st.n_pages), 16384, s);
}

}  // namespace tq
