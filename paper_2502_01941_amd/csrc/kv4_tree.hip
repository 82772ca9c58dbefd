// Trees of drafted tokens over the paged 4-bit cache: what each draft sees, and which of them stay.
//
// Both kernels are a launch and two to four dependent trips to memory (starts, drafts, slots, rows); there is next to nothing
// to compute or to move.
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

// A workgroup per request, and one for the rows that no request has.  Every thread follows the parents of a draft of its own,
// from LDS; they come in falling order, so the words of its row are done one after the other.
constexpr int kPlanThreads = 256;
__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(int R, int T, const int32_t* __restrict__ query_start,
                                                                 const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ pos_start, int words,
                                                                 uint32_t* __restrict__ tree_mask, int32_t* __restrict__ token_pos,
                                                                 int32_t* __restrict__ status) {
  __shared__ int up[32 * kTreeWords];
  const int r = blockIdx.x;
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
  bool fits = d.n <= 32 * words, sound = true;
  if (fits) {
    for (int i = threadIdx.x; i < d.n; i += kPlanThreads) {
      const int parent = parents[d.first + i];
      up[i] = parent;
      sound = sound && parent < i;
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
    int w = i >> 5, depth = 0;
    for (int e = w + 1; e < words; ++e) row[e] = 0u;
    uint32_t bits = 1u << (i & 31);
    for (int a = up[i]; a >= 0; a = up[a]) {
      while (w > a >> 5) {
        row[w--] = bits;
        bits = 0u;
      }
      bits |= 1u << (a & 31);
      ++depth;
    }
    for (; w >= 0; --w) {
      row[w] = bits;
      bits = 0u;
    }
    const long long at = pos0 + depth;
    token_pos[d.first + i] = at <= 0x7fffffffLL ? static_cast<int>(at) : -1;
  }
}

// Four waves of a workgroup: a request, and four of its (layer, KV head) pairs.  Every wave follows the drafts by itself, from
// registers, 64 of them to a chunk.  Rows move in the order of the path: row path[j] >= j goes to place j, so nothing is read
// that an earlier one of them wrote, as long as those on their way together are all read before the first is written.
constexpr int kKeepThreads = 256, kKeepWaves = kKeepThreads / kWave;
constexpr int kHeld = 4;  // chunks in registers; drafts behind them are read again at every step
template <int D>
__global__ __launch_bounds__(kKeepThreads) void tree_keep_kernel(TreeKeepArgs p) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, r = blockIdx.x;
  const Drafts d(p.query_start, r, p.T);
  const bool stores = p.cache.base != nullptr;
  auto slot_of = [&](int i) {  // of the first layer
    const int slot = p.slot_map[d.first + i];
    return static_cast<uint32_t>(slot) < p.layer_slots ? slot : -1;
  };
  const int pair = blockIdx.y * kKeepWaves + wave;
  const bool writes = pair == 0;
  if (!writes && (!stores || pair >= p.layers * p.cache.H_kv)) return;

  int parent[kHeld], token[kHeld], chosen[kHeld];
#pragma unroll
  for (int c = 0; c < kHeld; ++c) {
    const int i = c * kWave + lane;
    parent[c] = i < d.n ? p.parents[d.first + i] : -1;
    token[c] = i < d.n ? p.tokens[d.first + i] : -1;
    chosen[c] = i < d.n ? p.chosen[d.first + i] : -1;
  }
  int here = d.n > 0 && p.max_path > 0 && (!stores || slot_of(0) >= 0) ? 0 : -1;
  int next = -1;          // the token that the model chose after the last of the path
  int accepted = 0;
  int32_t* path = p.path + static_cast<size_t>(r) * p.max_path;
  while (here >= 0) {
    // 64 of the path at a time: lane j holds the one that goes to place at + j
    const int at = accepted;
    int mine = -1;
    int count = 0;
    for (; here >= 0 && count < kWave; ++count) {
      if (lane == count) mine = here;
      next = -1;
#pragma unroll
      for (int c = 0; c < kHeld; ++c)
        if (here / kWave == c) next = __builtin_amdgcn_readlane(chosen[c], here % kWave);
      if (here >= kHeld * kWave) next = p.chosen[d.first + here];
      next = __builtin_amdgcn_readfirstlane(next);
      int child = -1;
      if (next >= 0 && at + count + 1 < p.max_path) {
#pragma unroll
        for (int c = 0; c < kHeld; ++c) {
          if (child >= 0 || c * kWave + kWave <= here) continue;
          const unsigned long long fits = __ballot(parent[c] == here && token[c] == next && c * kWave + lane > here);
          if (fits) child = c * kWave + __builtin_ctzll(fits);
        }
        for (int base = max(kHeld * kWave, here & ~(kWave - 1)); child < 0 && base < d.n; base += kWave) {
          const int i = base + lane;
          const unsigned long long fits = __ballot(i < d.n && i > here && p.parents[d.first + i] == here && p.tokens[d.first + i] == next);
          if (fits) child = base + __builtin_ctzll(fits);
        }
      }
      here = child;
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
    p.next_token[r] = max(next, -1);
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
