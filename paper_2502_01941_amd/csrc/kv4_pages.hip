// Pages of the 4-bit cache: block tables and slot maps from request lengths, and pages given back.
//
// A plan is prefix sums over the requests - new tokens before r (the start of its rows in the batch), pages needed before
// r (its place on the free stack) - and then one slot and one position per new token.  Every word is read or written once
// and the sums are over a few thousand words that lie in the caches, so the time is that of one launch and three dependent
// trips to memory: lengths, page, slot.  A workgroup per request adds up the lengths of all requests before its own itself
// rather than wait for a scan.  16 requests that grow by a token take 3.6 us; 512 prompts of 1 to 8192 tokens 6.6 us, with four
// tokens to a thread and their slots in one store (3.9 MB, 0.8 us at the rate of a copy), and 3.1 + 3.7 + 1.8 us to give back:
// rows, stack and lengths one after the other, because each goes by what the one before wrote for all requests.
#include "kv4.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;

__device__ __forceinline__ int pages_of(int tokens, int shift) {
  return static_cast<int>((static_cast<long long>(tokens) + (1 << shift) - 1) >> shift);
}

// Sum over the wave of numbers below 2^48 (exchanges between lanes are of 32 bits).
__device__ __forceinline__ long long wave_sum64(long long v) {
  const uint32_t low = wave_sum(static_cast<uint32_t>(v) & 0xffffffu), high = wave_sum(static_cast<uint32_t>(v >> 24));
  return (static_cast<long long>(high) << 24) + low;
}
// Two sums over the workgroup; every thread gets them.
__device__ __forceinline__ void block_sums(long long& a, long long& b, long long* scratch) {
  a = wave_sum64(a);
  b = wave_sum64(b);
  if (threadIdx.x % kWave == 0) {
    scratch[threadIdx.x / kWave] = a;
    scratch[kWaves + threadIdx.x / kWave] = b;
  }
  __syncthreads();
  a = b = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    a += scratch[w];
    b += scratch[kWaves + w];
  }
}
// Sum over the threads before this one, and over all.
__device__ __forceinline__ long long block_scan(long long v, long long* scratch, long long* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  long long sum = v;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const long long up = __shfl_up(sum, m);
    if (lane >= m) sum += up;
  }
  __syncthreads();
  if (lane == kWave - 1) scratch[wave] = sum;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    all += scratch[w];
  }
  *total = all;
  return before + sum - v;
}

// Whether a request's lengths make sense by themselves, and the pages that it needs then.
__device__ __forceinline__ bool lengths_ok(int cached, int fresh, int shift, int max_pages, int request_tokens) {
  return cached >= 0 && fresh >= 0 && (request_tokens == 0 || fresh <= request_tokens) &&
         static_cast<long long>(cached) + fresh <= static_cast<long long>(max_pages) << shift;
}

// Workgroup r < R: request r.  Workgroup R: what is left of the stack.
__global__ __launch_bounds__(kThreads) void pages_plan_kernel(
    int R, int shift, int max_pages, const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ new_lens,
    const int32_t* __restrict__ pos_start, const int32_t* __restrict__ free_pages, int stack_size,
    const int32_t* __restrict__ free_count, int32_t* block_table, int32_t* __restrict__ free_left, int32_t* __restrict__ seq_lens,
    int32_t* __restrict__ query_start, int T, int request_tokens, int32_t* __restrict__ slot_map,
    int32_t* __restrict__ token_pos, int32_t* __restrict__ status) {
  __shared__ long long scratch[2 * kWaves];
  const int r = blockIdx.x;
  const long long stack = min(max(*free_count, 0), stack_size);
  if (r == R) {
    // The requests that get their pages are those whose last one is on the stack: the most pages up to any of them.
    long long tokens = 0, pages = 0, given = 0;
    for (int base = 0; base < R; base += kThreads) {
      const int i = base + threadIdx.x;
      const int cached = i < R ? cached_lens[i] : 0, fresh = i < R ? new_lens[i] : 0;
      long long all;
      const long long rows = max(fresh, 0);
      const long long first = tokens + block_scan(rows, scratch, &all);
      tokens += all;
      bool ok = lengths_ok(cached, fresh, shift, max_pages, request_tokens);
      if (request_tokens == 0) ok = ok && (fresh == 0 || first + fresh <= T);
      else ok = ok && (fresh == 0 || static_cast<long long>(i) * request_tokens + fresh <= T);
      const int need = ok ? pages_of(cached + fresh, shift) - pages_of(cached, shift) : 0;
      const long long until = pages + block_scan(need, scratch, &all) + need;
      pages += all;
      if (need > 0 && until <= stack) given = max(given, until);
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) given = max(given, __shfl_xor(given, m));
    __syncthreads();
    if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = given;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kWaves; ++w) given = max(given, scratch[w]);
      *free_left = static_cast<int32_t>(stack - given);
      query_start[R] = static_cast<int32_t>(min(tokens, 0x7fffffffLL));
    }
    // rows of the batch that belong to no request
    const long long used = request_tokens ? static_cast<long long>(R) * request_tokens : tokens;
    for (long long t = used + threadIdx.x; t < T; t += kThreads) slot_map[t] = token_pos[t] = -1;
    return;
  }
  // Tokens and pages of the requests before this one.  Those before it whose rows end past the batch need no pages, but
  // if there are any its own rows lie past the batch too, and then it takes none either.
  long long tokens = 0, pages = 0;
  for (int i = threadIdx.x; i < r; i += kThreads) {
    const int cached = cached_lens[i], fresh = new_lens[i];
    tokens += max(fresh, 0);
    const bool ok = lengths_ok(cached, fresh, shift, max_pages, request_tokens) &&
                    (request_tokens == 0 || fresh == 0 || static_cast<long long>(i) * request_tokens + fresh <= T);
    if (ok) pages += pages_of(cached + fresh, shift) - pages_of(cached, shift);
  }
  const int cached = cached_lens[r], fresh = new_lens[r];
  block_sums(tokens, pages, scratch);
  const long long row0 = request_tokens ? static_cast<long long>(r) * request_tokens : tokens;
  const bool ok = lengths_ok(cached, fresh, shift, max_pages, request_tokens) && (fresh == 0 || row0 + fresh <= T);
  const int held = ok ? pages_of(cached, shift) : 0;
  const int need = ok ? pages_of(cached + fresh, shift) - held : 0;
  const bool fits = need == 0 || pages + need <= stack;
  const bool granted = ok && fits;
  int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
  // top of the stack for this request; page j of its new ones is top[-j]
  const int32_t* top = free_pages + (stack - 1 - pages);
  if (granted)
    for (int j = threadIdx.x; j < need; j += kThreads) row[held + j] = top[-j];
  if (threadIdx.x == 0) {
    seq_lens[r] = granted ? cached + fresh : cached;
    query_start[r] = static_cast<int32_t>(min(tokens, 0x7fffffffLL));
    status[r] = !ok ? SHOTKV_ST_BAD_LENGTH : fits ? SHOTKV_ST_OK : SHOTKV_ST_NO_FREE_PAGE;
  }
  const int pos0 = pos_start ? pos_start[r] : cached;
  const int page_mask = (1 << shift) - 1;
  const bool aligned = ((reinterpret_cast<uintptr_t>(slot_map) | reinterpret_cast<uintptr_t>(token_pos)) & 15u) == 0;
  const long long rows = request_tokens ? request_tokens : max(fresh, 0);
  const long long end = min(row0 + rows, static_cast<long long>(T));
  // Four tokens to a thread, at a multiple of four of the batch: they lie in one page or in two.
  for (long long t = (row0 & ~3ll) + 4 * threadIdx.x; t < end; t += 4 * kThreads) {
    const int first = static_cast<int>(max(t, row0) - row0), last = static_cast<int>(min(t + 3, end - 1) - row0);
    int page[2] = {-1, -1};
    const int p0 = granted ? (cached + first) >> shift : 0;
    if (granted && first < fresh) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int p = j == 0 ? p0 : (cached + min(last, fresh - 1)) >> shift;
        page[j] = p < held ? row[p] : top[-(p - held)];
      }
    }
    int32_t slot[4], pos[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = static_cast<int>(t + e - row0);
      slot[e] = pos[e] = -1;
      if (granted && i >= 0 && i < fresh) {
        const int at = cached + i, of = (at >> shift) == p0 ? page[0] : page[1];
        const long long s = (static_cast<long long>(of) << shift) + (at & page_mask);
        if (of >= 0 && s <= 0x7fffffffLL) slot[e] = static_cast<int>(s);
        pos[e] = pos0 + i;
      }
    }
    if (t >= row0 && t + 4 <= end && aligned) {
      *reinterpret_cast<int4*>(slot_map + t) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      *reinterpret_cast<int4*>(token_pos + t) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e >= row0 && t + e < end) {
          slot_map[t + e] = slot[e];
          token_pos[t + e] = pos[e];
        }
    }
  }
}

// Pages of a request that is given back: no more than its row lists.
__device__ __forceinline__ int held_pages(int tokens, int shift, int max_pages) {
  return min(pages_of(max(tokens, 0), shift), max_pages);
}

// Entries that are no pages leave the rows of the finished requests, the others close up, and the lengths become those of as many
// full pages: what a request gives back depends on its row, and the launch below goes by the lengths of all.
__global__ __launch_bounds__(kThreads) void pages_close_up_kernel(int shift, int max_pages, const uint8_t* __restrict__ finished,
                                                                  int32_t* __restrict__ seq_lens, int32_t* __restrict__ block_table) {
  __shared__ long long scratch[2 * kWaves];
  const int r = blockIdx.x;
  if (!finished[r]) return;
  const int n = held_pages(seq_lens[r], shift, max_pages);
  int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
  int kept = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int j = base + threadIdx.x;
    const int32_t page = j < n ? row[j] : -1;
    long long all = min(n - base, kThreads), before = threadIdx.x;
    if (__syncthreads_or(j < n && page < 0)) before = block_scan(page >= 0 ? 1 : 0, scratch, &all);
    if (page >= 0 && kept + before < j) row[kept + before] = page;
    kept += static_cast<int>(all);
  }
  if (threadIdx.x == 0) seq_lens[r] = kept << shift;
}

__global__ __launch_bounds__(kThreads) void pages_release_kernel(int R, int shift, int max_pages,
                                                                 const uint8_t* __restrict__ finished,
                                                                 const int32_t* __restrict__ seq_lens,
                                                                 int32_t* __restrict__ block_table,
                                                                 int32_t* __restrict__ free_pages, int stack_size,
                                                                 const int32_t* __restrict__ free_count) {
  __shared__ long long scratch[2 * kWaves];
  const int r = blockIdx.x;
  if (!finished[r]) return;
  long long before = 0, all = 0;
  for (int i = threadIdx.x; i < R; i += kThreads) {
    const int n = finished[i] ? held_pages(seq_lens[i], shift, max_pages) : 0;
    all += n;
    if (i < r) before += n;
  }
  block_sums(before, all, scratch);
  const int n = held_pages(seq_lens[r], shift, max_pages);
  int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
  const long long top = max(*free_count, 0) + all - 1 - before;
  for (int j = threadIdx.x; j < max_pages; j += kThreads) {
    const int32_t page = row[j];
    if (j < n && top - j < stack_size) free_pages[top - j] = page;
    row[j] = -1;
  }
}
// A launch of its own: every workgroup of the one above reads all lengths.
__global__ __launch_bounds__(kThreads) void pages_release_lens_kernel(int R, int shift, int max_pages,
                                                                      const uint8_t* __restrict__ finished,
                                                                      int32_t* __restrict__ seq_lens, int stack_size,
                                                                      int32_t* __restrict__ free_count) {
  __shared__ long long scratch[2 * kWaves];
  long long all = 0;
  for (int i = threadIdx.x; i < R; i += kThreads)
    if (finished[i]) {
      all += held_pages(seq_lens[i], shift, max_pages);
      seq_lens[i] = 0;
    }
  long long unused = 0;
  block_sums(all, unused, scratch);
  if (threadIdx.x == 0)
    *free_count = static_cast<int32_t>(min(max(*free_count, 0) + all, static_cast<long long>(max(stack_size, 0))));
}

// The entries of a request's row that a trim takes out: those of its pages between sinks and window, and those behind its end.
struct Trimmed {
  int from, between, end;  // entries [from, from + between), and `behind` ones from `end` on
  int behind;
  __device__ __forceinline__ Trimmed(int held_tokens, int tokens, int shift, int max_pages, int window, int n_sinks) {
    const int held = held_pages(held_tokens, shift, max_pages);
    tokens = static_cast<int>(min(static_cast<long long>(max(tokens, 0)), static_cast<long long>(max_pages) << shift));
    from = pages_of(n_sinks, shift);
    between = max(min((tokens - window + 1) >> shift, held) - from, 0);
    end = pages_of(tokens, shift);
    behind = max(held - end, 0);
  }
  __device__ __forceinline__ int count() const { return between + behind; }
  __device__ __forceinline__ int entry(int i) const { return i < between ? from + i : end + i - between; }
};
// Few requests that have few pages to look at: one workgroup, a wave to a request, in one launch.  With a plan before it and the calls
// from Python, 16 requests with drafts take 20.4 us so and 23.3 in the two launches below, 64 20.2 and 23.1; with a window, which
// all pages in front of it are looked at for, 64 requests of 513 pages 15.8 and 14.5, 32 of 1876 33 and 14.7.
constexpr int kTrimFewRequests = 64, kTrimThreads = 1024;
constexpr long long kTrimFewPages = 65536, kTrimFewWindowPages = 4096;  // rows of all requests
__global__ __launch_bounds__(kTrimThreads) void pages_trim_few_kernel(int R, int shift, int max_pages, const int32_t* __restrict__ held_lens,
                                                                      const int32_t* __restrict__ seq_lens, int window, int n_sinks,
                                                                      int32_t* __restrict__ block_table, int32_t* __restrict__ free_pages,
                                                                      int stack_size, const int32_t* __restrict__ free_count,
                                                                      int32_t* __restrict__ free_left, int32_t* __restrict__ given_back) {
  __shared__ int counts[kTrimFewRequests];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = kTrimThreads / kWave;
  for (int r = wave; r < R; r += waves) {
    const Trimmed t(held_lens[r], seq_lens[r], shift, max_pages, window, n_sinks);
    const int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
    int pages = 0;
    for (int i = lane; i < t.count(); i += kWave) pages += row[t.entry(i)] >= 0;
    pages = wave_sum(pages);
    if (lane == 0) counts[r] = given_back[r] = pages;
  }
  __syncthreads();
  int until = lane < R ? counts[lane] : 0;  // pages of the requests up to and with number `lane`
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int up = __shfl_up(until, m);
    if (lane >= m) until += up;
  }
  const long long count = min(max(*free_count, 0), stack_size);
  const int all = __shfl(until, kWave - 1);
  if (threadIdx.x == 0) *free_left = static_cast<int32_t>(min(count + all, static_cast<long long>(stack_size)));
  for (int r = wave; r < R; r += waves) {
    if (counts[r] == 0) continue;
    const Trimmed t(held_lens[r], seq_lens[r], shift, max_pages, window, n_sinks);
    int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
    long long top = count + all - 1 - (__shfl(until, r) - counts[r]);
    for (int base = 0; base < t.count(); base += kWave) {
      const int i = base + lane;
      const int32_t page = i < t.count() ? row[t.entry(i)] : -1;
      const unsigned long long there = __ballot(page >= 0);
      const long long to = top - __popcll(there & ((1ull << lane) - 1ull));
      top -= __popcll(there);
      if (page < 0) continue;
      if (to < stack_size) free_pages[to] = page;
      row[t.entry(i)] = -1;
    }
  }
}
__global__ __launch_bounds__(kThreads) void pages_trim_count_kernel(int shift, int max_pages, const int32_t* __restrict__ held_lens,
                                                                    const int32_t* __restrict__ seq_lens, int window, int n_sinks,
                                                                    const int32_t* __restrict__ block_table,
                                                                    int32_t* __restrict__ given_back) {
  __shared__ long long scratch[2 * kWaves];
  const int r = blockIdx.x;
  const Trimmed t(held_lens[r], seq_lens[r], shift, max_pages, window, n_sinks);
  const int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
  long long pages = 0, unused = 0;
  for (int i = threadIdx.x; i < t.count(); i += kThreads) pages += row[t.entry(i)] >= 0;
  block_sums(pages, unused, scratch);
  if (threadIdx.x == 0) given_back[r] = static_cast<int32_t>(pages);
}
// A launch of its own: where a request's pages go depends on how many all others give back.
__global__ __launch_bounds__(kThreads) void pages_trim_kernel(int R, int shift, int max_pages, const int32_t* __restrict__ held_lens,
                                                              const int32_t* __restrict__ seq_lens, int window, int n_sinks,
                                                              int32_t* __restrict__ block_table, int32_t* __restrict__ free_pages,
                                                              int stack_size, const int32_t* __restrict__ free_count,
                                                              int32_t* __restrict__ free_left, const int32_t* __restrict__ given_back) {
  __shared__ long long scratch[2 * kWaves];
  const int r = blockIdx.x;
  long long before = 0, all = 0;
  for (int i = threadIdx.x; i < R; i += kThreads) {
    const int n = given_back[i];
    all += n;
    if (i < r) before += n;
  }
  block_sums(before, all, scratch);
  const long long count = min(max(*free_count, 0), stack_size);
  if (r == 0 && threadIdx.x == 0) *free_left = static_cast<int32_t>(min(count + all, static_cast<long long>(stack_size)));
  if (given_back[r] == 0) return;
  const Trimmed t(held_lens[r], seq_lens[r], shift, max_pages, window, n_sinks);
  int32_t* row = block_table + static_cast<size_t>(r) * max_pages;
  long long top = count + all - 1 - before;
  for (int base = 0; base < t.count(); base += kThreads) {
    const int i = base + threadIdx.x;
    const int32_t page = i < t.count() ? row[t.entry(i)] : -1;
    long long given;
    const long long to = top - block_scan(page >= 0 ? 1 : 0, scratch, &given);
    top -= given;
    if (page < 0) continue;
    if (to < stack_size) free_pages[to] = page;
    row[t.entry(i)] = -1;
  }
}

}  // namespace

hipError_t launch_pages_trim(int R, int page_shift, int max_pages, const int32_t* held_lens, const int32_t* seq_lens, int window,
                             int n_sinks, int32_t* block_table, int32_t* free_pages, int stack_size, const int32_t* free_count,
                             int32_t* free_left, int32_t* given_back, hipStream_t s) {
  const bool windowed = window < max_pages << page_shift;
  if (R <= kTrimFewRequests && static_cast<long long>(R) * max_pages <= (windowed ? kTrimFewWindowPages : kTrimFewPages)) {
    pages_trim_few_kernel<<<1, kTrimThreads, 0, s>>>(R, page_shift, max_pages, held_lens, seq_lens, window, n_sinks, block_table, free_pages,
                                                     stack_size, free_count, free_left, given_back);
    return hipGetLastError();
  }
  pages_trim_count_kernel<<<R, kThreads, 0, s>>>(page_shift, max_pages, held_lens, seq_lens, window, n_sinks, block_table, given_back);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_trim_kernel<<<R, kThreads, 0, s>>>(R, page_shift, max_pages, held_lens, seq_lens, window, n_sinks, block_table, free_pages, stack_size,
                                           free_count, free_left, given_back);
  return hipGetLastError();
}

hipError_t launch_pages_plan(int R, int page_shift, int max_pages, const int32_t* cached_lens, const int32_t* new_lens,
                             const int32_t* pos_start, const int32_t* free_pages, int stack_size,
                             const int32_t* free_count, int32_t* block_table, int32_t* free_left, int32_t* seq_lens,
                             int32_t* query_start, int T, int request_tokens, int32_t* slot_map, int32_t* token_pos,
                             int32_t* status, hipStream_t s) {
  pages_plan_kernel<<<R + 1, kThreads, 0, s>>>(R, page_shift, max_pages, cached_lens, new_lens, pos_start, free_pages,
                                               stack_size, free_count, block_table, free_left, seq_lens, query_start, T,
                                               request_tokens, slot_map, token_pos, status);
  return hipGetLastError();
}

hipError_t launch_pages_release(int R, int page_shift, int max_pages, const uint8_t* finished, int32_t* seq_lens,
                                int32_t* block_table, int32_t* free_pages, int stack_size, int32_t* free_count,
                                hipStream_t s) {
  pages_close_up_kernel<<<R, kThreads, 0, s>>>(page_shift, max_pages, finished, seq_lens, block_table);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_release_kernel<<<R, kThreads, 0, s>>>(R, page_shift, max_pages, finished, seq_lens, block_table, free_pages,
                                              stack_size, free_count);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_release_lens_kernel<<<1, kThreads, 0, s>>>(R, page_shift, max_pages, finished, seq_lens, stack_size, free_count);
  return hipGetLastError();
}

}  // namespace shotkv
