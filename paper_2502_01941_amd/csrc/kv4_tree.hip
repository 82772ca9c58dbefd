// Trees of drafted tokens over the paged 4-bit cache: what each draft sees, and which of them stay.
//
// Both kernels are a launch and two to four dependent trips to memory (starts, drafts, slots, rows); there is next to nothing
// to compute or to move, so that is what bounds them.
#include "kv4.hpp"

namespace shotkv {

namespace {

struct Drafts {
  int first, n;  // of the batch
  __device__ __forceinline__ Drafts(const int32_t* __restrict__ query_start, int r, int T) {
    first = min(max(query_start[r], 0), T);
    n = max(min(max(query_start[r + 1], 0), T) - first, 0);
  }
};

// A workgroup per request, and one for the rows that no request has.  Ancestors are found in groups of 64 drafts, a wave each, in six
// steps that double how far a draft sees: its ancestors in the group are the bits of two words, and the first one outside is where
// it goes on.  Then every draft writes its row from group to group, the last first.  So a chain of 1024 drafts takes 16 trips
// through LDS and not 1023 (20 us with the call; following parents one by one it took 238).  16 trees of 16 to 64 drafts take
// 3.1 us on the GPU, 512 of up to 256 4.8; a call from Python is 7.
constexpr int kPlanThreads = 256;
__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(int R, int T, const int32_t* __restrict__ query_start,
                                                                 const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ pos_start, int words,
                                                                 uint32_t* __restrict__ tree_mask, int32_t* __restrict__ token_pos,
                                                                 int32_t* __restrict__ status) {
  constexpr int kMost = 32 * kTreeWords;
  __shared__ uint32_t low[kMost], high[kMost];  // bits of a draft's group
  __shared__ int outside[kMost];                // its first ancestor in a group before, below 0 if there is none
  const int r = blockIdx.x, lane = threadIdx.x % kWave;
  auto nothing = [&](long long from, long long to) {
    for (long long t = from + threadIdx.x; t < to; t += kPlanThreads) token_pos[t] = -1;
    for (long long w = from * words + threadIdx.x; w < to * words; w += kPlanThreads) tree_mask[w] = 0u;
  };
  if (r == R) {
    nothing(0, min(max(query_start[0], 0), T));
    nothing(min(max(query_start[R], 0), T), T);
    return;
  }
  const Drafts d(query_start, r, T);
  const long long pos0 = pos_start[r];
  const bool fits = d.n <= 32 * words;
  bool sound = true;
  if (fits) {
    for (int i = threadIdx.x; i - lane < d.n; i += kPlanThreads) {  // (whole waves)
      const int parent = i < d.n ? parents[d.first + i] : -1;
      sound = sound && parent < i;
      const int group = i - lane;
      int up = parent >= group && parent < i ? parent - group : -1, out = parent < group ? parent : -1;
      uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
      for (int step = 0; step < 6; ++step) {
        const int from = max(up, 0);
        const uint32_t more_lo = __shfl(lo, from), more_hi = __shfl(hi, from);
        const int further = __shfl(up, from), its = __shfl(out, from);
        if (up >= 0) {
          lo |= more_lo;
          hi |= more_hi;
          out = its;
          up = further;
        }
      }
      if (i < d.n) {
        low[i] = lo;
        high[i] = hi;
        outside[i] = out;
      }
    }
  }
  sound = !__syncthreads_or(!sound);
  if (threadIdx.x == 0) status[r] = !fits ? SHOTKV_ST_BAD_LENGTH : sound ? SHOTKV_ST_OK : SHOTKV_ST_BAD_TREE;
  if (!fits || !sound) {
    nothing(d.first, static_cast<long long>(d.first) + d.n);
    return;
  }
  for (int i = threadIdx.x; i < d.n; i += kPlanThreads) {
    uint32_t* row = tree_mask + static_cast<size_t>(d.first + i) * words;
    int end = words, depth = -1;  // words from `end` on are written
    for (int a = i; a >= 0; a = outside[a]) {
      const int w = a >> 6 << 1;
      for (int e = w + 2; e < end; ++e) row[e] = 0u;
      const uint32_t lo = low[a], hi = high[a];
      row[w] = lo;
      if (w + 1 < words) row[w + 1] = hi;
      depth += __builtin_popcount(lo) + __builtin_popcount(hi);
      end = w;
    }
    for (int e = 0; e < end; ++e) row[e] = 0u;
    const long long at = pos0 + depth;
    token_pos[d.first + i] = at <= 0x7fffffffLL ? static_cast<int>(at) : -1;
  }
}

// Four waves of a workgroup: a request, and four of its (layer, KV head) pairs.  Which child of a draft the model chose is found for all
// drafts at once, in LDS (the least number of those that fit, so the order does not matter), and then followed from draft 0 on by
// every wave.  Rows move in the order of the path: row path[j] >= j goes to place j, so nothing is read that an earlier one of
// them wrote, as long as those on their way together are all read before the first is written.  16 requests of 16 to 64 drafts take 4.8
// us on the GPU with 8 pairs of layer and head, 6.7 with 256; a chain of 64 that is kept takes 9 with the call (18 where every wave looked its
// children up in registers).
constexpr int kKeepThreads = 256, kKeepWaves = kKeepThreads / kWave;
constexpr int kHeld = 32 * kTreeWords;  // drafts in LDS; a request of more is looked through anew at every step
template <int D>
__global__ __launch_bounds__(kKeepThreads) void tree_keep_kernel(TreeKeepArgs p) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, r = blockIdx.x;
  Drafts d(p.query_start, r, p.T);
  if (p.status && p.status[r] != SHOTKV_ST_OK) d.n = 0;
  __shared__ int chosen[kHeld], child[kHeld];
  const bool stores = p.cache.base != nullptr;
  auto slot_of = [&](int i) {  // of the first layer
    const int slot = p.slot_map[d.first + i];
    return static_cast<uint32_t>(slot) < p.layer_slots ? slot : -1;
  };
  const int pair = blockIdx.y * kKeepWaves + wave;
  const bool writes = pair == 0;
  const bool held = d.n <= kHeld;
  if (held) {
    for (int i = threadIdx.x; i < d.n; i += kKeepThreads) {
      chosen[i] = p.chosen[d.first + i];
      child[i] = d.n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < d.n; i += kKeepThreads) {
      const int parent = p.parents[d.first + i], token = p.tokens[d.first + i];
      if (parent >= 0 && parent < i && token >= 0 && token == chosen[parent]) atomicMin(&child[parent], i);
    }
    __syncthreads();
  }
  if (!writes && (!stores || pair >= p.layers * p.cache.H_kv)) return;
  // The draft after draft `here`, d.n if there is none.
  auto after = [&](int here) {
    if (held) return __builtin_amdgcn_readfirstlane(child[here]);
    const int next = p.chosen[d.first + here];
    for (int base = here & ~(kWave - 1); next >= 0 && base < d.n; base += kWave) {
      const int i = base + lane;
      const unsigned long long fits = __ballot(i < d.n && i > here && p.parents[d.first + i] == here && p.tokens[d.first + i] == next);
      if (fits) return base + __builtin_ctzll(fits);
    }
    return d.n;
  };

  int here = d.n > 0 && (!stores || slot_of(0) >= 0) ? 0 : d.n;
  int last = -1;
  int accepted = 0;
  int32_t* path = p.path + static_cast<size_t>(r) * p.max_path;
  while (here < d.n && accepted < p.max_path) {
    // 64 of the path at a time: lane j holds the one that goes to place at + j
    const int at = accepted;
    int mine = -1;
    int count = 0;
    for (; here < d.n && count < kWave && at + count < p.max_path; ++count) {
      if (lane == count) mine = here;
      last = here;
      here = after(here);
    }
    accepted += count;
    if (writes && lane < count) path[at + lane] = mine;
    if (!stores || pair >= p.layers * p.cache.H_kv) continue;

    // ---- rows: sixteen (eight) lanes to a row, a word of keys and one of values each
    const int layer = pair / p.cache.H_kv, head = pair - layer * p.cache.H_kv;
    constexpr int kLanes = D / 8, kRows = kWave / kLanes, kGroups = D / 32, kDeep = 2;
    typedef Kv4Block<D> B;
    const int from = lane < count && mine != at + lane ? slot_of(mine) : -1;
    const int to = from >= 0 ? slot_of(at + lane) : -1;
    if (!__any(to >= 0)) continue;
    const int c = lane % kLanes;
    for (int j0 = 0; j0 < count; j0 += kRows * kDeep) {
      uint32_t k[kDeep], v[kDeep];
      uint8_t ks[kDeep], vs[kDeep];
      char* dst[kDeep];
      int token_to[kDeep];
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const int j = min(j0 + u * kRows + lane / kLanes, kWave - 1);
        const int source = __shfl(from, j), target = __shfl(to, j);
        dst[u] = nullptr;
        if (j0 + u * kRows + lane / kLanes < count && target >= 0) {
          const char* src = kv4_block_of_slot<D>(p.cache, static_cast<uint32_t>(source) + layer * p.layer_slots, head);
          const int t = source & 31;
          dst[u] = kv4_block_of_slot<D>(p.cache, static_cast<uint32_t>(target) + layer * p.layer_slots, head);
          token_to[u] = target & 31;
          k[u] = *reinterpret_cast<const uint32_t*>(src + B::key_word(t, c));
          v[u] = *reinterpret_cast<const uint32_t*>(src + B::value_word(t, c));
          if (c < kGroups) {
            ks[u] = *reinterpret_cast<const uint8_t*>(src + B::key_scale(t, c));
            vs[u] = *reinterpret_cast<const uint8_t*>(src + B::value_scale(t, c));
          }
        }
      }
      // all have arrived before the first is written: another lane may write what one of these loads reads
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
      for (int u = 0; u < kDeep; ++u)
        if (dst[u]) {
          *reinterpret_cast<uint32_t*>(dst[u] + B::key_word(token_to[u], c)) = k[u];
          *reinterpret_cast<uint32_t*>(dst[u] + B::value_word(token_to[u], c)) = v[u];
          if (c < kGroups) {
            *reinterpret_cast<uint8_t*>(dst[u] + B::key_scale(token_to[u], c)) = ks[u];
            *reinterpret_cast<uint8_t*>(dst[u] + B::value_scale(token_to[u], c)) = vs[u];
          }
        }
      asm volatile("" : : : "memory");
    }
  }
  if (!writes) return;
  for (int j = accepted + lane; j < p.max_path; j += kWave) path[j] = -1;
  if (lane == 0) {
    p.accepted[r] = accepted;
    p.next_token[r] = last < 0 ? -1 : max(p.chosen[d.first + last], -1);
    p.kept_lens[r] = p.cached_lens[r] + accepted;
  }
}

}  // namespace

hipError_t launch_tree_plan(int R, int T, const int32_t* query_start, const int32_t* parents, const int32_t* pos_start, int words,
                            uint32_t* tree_mask, int32_t* token_pos, int32_t* status, hipStream_t s) {
  tree_plan_kernel<<<R + 1, kPlanThreads, 0, s>>>(R, T, query_start, parents, pos_start, words, tree_mask, token_pos, status);
  return hipGetLastError();
}

hipError_t launch_tree_keep(const TreeKeepArgs& a, int R, int D, hipStream_t s) {
  const int pairs = a.cache.base ? a.layers * a.cache.H_kv : 1;
  const dim3 grid(R, (pairs + kKeepWaves - 1) / kKeepWaves);
  if (D == 128) tree_keep_kernel<128><<<grid, kKeepThreads, 0, s>>>(a);
  else tree_keep_kernel<64><<<grid, kKeepThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace shotkv
