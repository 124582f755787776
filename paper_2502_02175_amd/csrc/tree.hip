// Trees of drafted tokens: the path on which the drafts are what was chosen, and that path kept in the pages.  Whole numbers, and
// values that are copied bit for bit.
#include <algorithm>
#include <type_traits>

#include "pages.h"
#include "trees.h"

namespace {

// A workgroup takes an entry.  Every node that was drafted as its parent's choice offers itself to the parent, which keeps the
// first (a minimum: no order decides); then a wave follows the offers from node 0 on.  A path ascends (a node's offers come after it), so
// that a node's place in it is the number of those before it.
constexpr int kAccept = 256;
__global__ __launch_bounds__(kAccept) void tree_accept_kernel(const int* __restrict__ parents, const int* __restrict__ drafted,
                                                            const int* __restrict__ chosen, int tokens, int* __restrict__ out_path,
                                                            int* __restrict__ out_count, int* __restrict__ out_token) {
  __shared__ int pick[VLAC_TREE_MAX_NODES], next[VLAC_TREE_MAX_NODES];
  const int tid = threadIdx.x;
  const size_t at = (size_t)blockIdx.x * tokens;
  const bool begins = parents[at] == -1;
  for (int t = tid; t < tokens; t += kAccept) {
    pick[t] = chosen[at + t];
    next[t] = tokens;
  }
  __syncthreads();
  for (int t = tid; t < tokens; t += kAccept) {
    const int up = parents[at + t];
    if (t > 0 && up >= 0 && up < t && pick[up] >= 0 && drafted[at + t] == pick[up]) atomicMin(&next[up], t);
  }
  __syncthreads();
  if (tid >= 64) return;
  uint64_t way = 0;
  if (begins) follow<false>(0, [&](int t) { return t < tokens && next[t] < tokens ? next[t] : -1; }, way);
  int n = 0, last = -1;
  for (int k = 0; 64 * k < tokens; ++k) {
    const uint64_t part = part_of(way, k);
    if (part >> tid & 1) out_path[at + n + __popcll(part & ((1ull << tid) - 1))] = 64 * k + tid;
    n += __popcll(part);
    if (part) last = 64 * k + 63 - __clzll((long long)part);
  }
  for (int t = n + tid; t < tokens; t += 64) out_path[at + t] = -1;
  if (tid == 0) {
    out_count[blockIdx.x] = n;
    out_token[blockIdx.x] = n > 0 ? pick[last] : -1;
  }
}

struct KeepArgs {
  PoolView p;
  const int *seqs, *pos, *path, *count;
  int n, tokens;
};

// Whether entry i can be done, worked out by every workgroup that has to do with it: -> how many rows are kept, or -1; *stay: the first of
// them that stay where they are (a path ascends, so all others move).  from, to: where row k comes from and goes to, page * 32 +
// position in it.  A chain of reads (lists and path, length and table, counts of the pages), about 0.7 us each.
constexpr int kKeep = 256;
struct Rows { int from[VLAC_TREE_MAX_NODES], to[VLAC_TREE_MAX_NODES], bad, wrong, stay; };
__device__ int keep_entry(const KeepArgs& a, int i, Rows& rows, int* stay) {
  constexpr int PER = VLAC_TREE_MAX_NODES / kKeep;
  const PoolView& p = a.p;
  const int tid = threadIdx.x, s = a.seqs[i], p0 = a.pos[i], m = a.count[i];
  int node[PER], before[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int k = u * kKeep + tid;
    node[u] = k < a.tokens ? a.path[(size_t)i * a.tokens + k] : -1;
    before[u] = k > 0 && k < a.tokens ? a.path[(size_t)i * a.tokens + k - 1] : -1;
  }
  if (p0 < 0) return -1;
  const int l = checked_len(p, s);
  if (tid == 0) {
    rows.bad = l < 0 || m < 0 || m > a.tokens || (long long)p0 + a.tokens != l;
    rows.wrong = rows.stay = 0;
  }
  bool wrong = false;
  for (int k = tid; k < i; k += kKeep) wrong |= a.seqs[k] == s && a.pos[k] >= 0;
  __syncthreads();
  if (rows.bad) return -1;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int k = u * kKeep + tid, t = node[u];
    if (k >= m) break;
    if (t <= before[u] || t < k || t >= a.tokens) {
      wrong = true;
    } else if (t == k) {
      atomicAdd(&rows.stay, 1);
    } else {
      const int* row = p.table + (size_t)s * p.max_pages;
      const int fp = row[(p0 + t) / kPage], gp = row[(p0 + k) / kPage];
      rows.from[k] = fp * kPage + (p0 + t) % kPage;
      rows.to[k] = gp * kPage + (p0 + k) % kPage;
      wrong |= (unsigned)fp >= (unsigned)p.n_pages || (unsigned)gp >= (unsigned)p.n_pages || p.refs[min((unsigned)gp, p.n_pages - 1u)] != 1;
    }
  }
  if (wrong) rows.wrong = 1;  // (not `bad`, which another wave may still have to look at before it comes to the next barrier)
  __syncthreads();
  *stay = rows.stay;
  return rows.wrong ? -1 : m;
}

// The rows of the path, one behind the other.  A workgroup takes an entry, a layer and some kv heads; a thread takes 16 bytes of K of
// every row (8 features), and a feature of V.  A row only moves down and rows are taken in ascending order, a thread's own
// words: what is read was not written before.  Eight rows are asked for at a time.  Bound by the lines that the layout touches: a position's K
// lies in 16 lines of a head of 128, of which it has an eighth, its V in as many more.
// Tables, counts and lengths stay as they are until the next launch; that this entry can be done is left for it in the pool's
// scratch (is_dst of the sequence, zero between calls: the entry's number + 1).
constexpr int kHeads = 4;  // of a work item
__global__ __launch_bounds__(kKeep) void pages_keep_kernel(KeepArgs a, int head_groups, int items) {
  __shared__ Rows rows;
  const PoolView& p = a.p;
  const int hd = p.head_dim;
  const int *from = rows.from, *to = rows.to;
  const size_t page = p.page(), tile = p.tile();
  for (int it = blockIdx.x; it < items; it += gridDim.x) {
    const int hg = it % head_groups, rest = it / head_groups, layer = rest % p.n_layers, i = rest / p.n_layers;
    int stay = 0;
    const int m = keep_entry(a, i, rows, &stay);
    if (m >= 0 && threadIdx.x == 0 && hg == 0 && layer == 0) p.is_dst()[a.seqs[i]] = i + 1;
    const int h0 = hg * kHeads, heads = min(kHeads, p.n_kv_heads - h0);
    bf16_t* const k0 = p.data + ((size_t)layer * 2 * p.n_kv_heads + h0) * tile;
    bf16_t* const v0 = k0 + p.n_kv_heads * tile;
    auto move = [&](auto* base, auto at) {  // the rows' words that lie at(position) behind base, in their page
      for (int r0 = stay; r0 < m; r0 += 8) {
        std::decay_t<decltype(*base)> y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int f = from[min(r0 + e, m - 1)];
          y[e] = base[(f >> 5) * (page * sizeof(bf16_t) / sizeof(*base)) + at(f & 31)];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int k = min(r0 + e, m - 1), t = to[k];
          if (r0 + e < m) base[(t >> 5) * (page * sizeof(bf16_t) / sizeof(*base)) + at(t & 31)] = y[e];
        }
      }
    };
    for (int u = threadIdx.x; u < heads * hd / 8; u += kKeep) {  // 16 bytes of K
      const int h = u / (hd / 8), c = u - h * (hd / 8);
      move((u32x4*)(k0 + h * tile + (c >> 1) * 512 + (c & 1) * 256), [](int r) { return r; });
    }
    for (int u = threadIdx.x; u < heads * hd; u += kKeep) {  // a feature of V
      const int h = u / hd, f = u - h * hd;
      move(v0 + h * tile + (f >> 5) * 1024 + (f & 31) * 8, [](int r) { return (r >> 4) * 512 + (r >> 2 & 1) * 256 + (r >> 3 & 1) * 4 + (r & 3); });
    }
    __syncthreads();  // (from and to are written again)
  }
}

// Lengths, and what lies behind them is released.  A workgroup per entry, behind the launch that moves the rows.
__global__ __launch_bounds__(64) void pages_keep_end_kernel(KeepArgs a) {
  const PoolView& p = a.p;
  const int i = blockIdx.x, s = a.seqs[i], p0 = a.pos[i];
  if (p0 < 0) return;
  if ((unsigned)s >= (unsigned)p.max_seqs || p.is_dst()[s] != i + 1) {
    if (threadIdx.x == 0) report(p, PAGES_BAD_ENTRY);
    return;
  }
  const int m = a.count[i], kept = pages_of(p0 + m), held = pages_of(p0 + a.tokens);
  for (int j = kept + threadIdx.x; j < held; j += 64) {
    int* at = p.table + (size_t)s * p.max_pages + j;
    const int pg = *at;
    *at = -1;
    if ((unsigned)pg < (unsigned)p.n_pages) atomicAdd(p.refs + pg, -1);
    else report(p, PAGES_BAD_ENTRY);
  }
  if (threadIdx.x == 0) {
    p.len[s] = p0 + m;
    p.is_dst()[s] = 0;  // (another entry of the sequence finds this or i + 1, neither of which is its own)
  }
}

}  // namespace

extern "C" {

int vlac_tree_accept(const int32_t* parents, const int32_t* drafted, const int32_t* chosen, int n, int tokens, int32_t* out_path,
                     int32_t* out_count, int32_t* out_token, void* stream) {
  if (n < 0 || n > VLAC_PAGES_MAX_LIST || tokens < 1 || tokens > VLAC_TREE_MAX_NODES) return VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!parents || !drafted || !chosen || !out_path || !out_count || !out_token) return VLAC_E_NULL;
  hipLaunchKernelGGL(tree_accept_kernel, dim3(n), dim3(kAccept), 0, (hipStream_t)stream, parents, drafted, chosen, tokens, out_path,
                     out_count, out_token);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

int vlac_pages_keep(const vlac_pages* pages, const int32_t* seqs, const int32_t* pos, int n, int tokens, const int32_t* path,
                    const int32_t* count, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  if (n < 0 || n > VLAC_PAGES_MAX_LIST || tokens < 1 || tokens > VLAC_TREE_MAX_NODES) return VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!seqs || !pos || !path || !count) return VLAC_E_NULL;
  const KeepArgs a = {pool_view(pages), seqs, pos, path, count, n, tokens};
  hipStream_t st = (hipStream_t)stream;
  const int groups = (pages->n_kv_heads + kHeads - 1) / kHeads, items = n * pages->n_layers * groups;  // (less than 2^30)
  hipLaunchKernelGGL(pages_keep_kernel, dim3((unsigned)std::min(items, 1 << 16)), dim3(kKeep), 0, st, a, groups, items);
  hipLaunchKernelGGL(pages_keep_end_kernel, dim3(n), dim3(64), 0, st, a);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
