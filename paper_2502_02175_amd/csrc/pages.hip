// Pages of the cache: forking, growing, releasing and compacting sequences, writing new tokens, and taking
// over a prefill.  No arithmetic: integers of the tables, and values that are copied bit for bit.
//
// The state of the allocator is refs alone (0 = free), so which pages a call takes is a function of the state and
// the list: the free pages in ascending order, entry by entry.  One workgroup works that out (ranks by
// prefix sums, no order of atomics decides anything); the pages themselves are copied by a second
// launch over the whole chip, from a list in the pool's scratch.
#include <algorithm>

#include "pages.h"

namespace {

constexpr int kPlan = 1024;  // threads of a planning workgroup

// refs change by atomics, which go to the L2: read them there (this CU's L1 may hold what was before)
__device__ inline int ld_agent(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Everything before it is done for every thread of the workgroup
__device__ inline void meet() {
  stores_done();
  __syncthreads();
}

// Sum over the workgroup's threads before this one; *total: over all of them.  sums: [kPlan / 64] words of LDS
__device__ inline int scan_before(int x, int* sums, int* total) {
  static_assert(kPlan / 64 == 16, "the waves' sums are a row of lanes");
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, run = wave_sums(x);
  if (lane == 63) sums[w] = run;
  __syncthreads();
  const int s = row_sums(sums[lane & 15]);  // (every wave adds them for itself: no second meeting)
  *total = __builtin_amdgcn_readlane(s, 15);
  const int before = w > 0 ? __builtin_amdgcn_readlane(s, __builtin_amdgcn_readfirstlane(max(w - 1, 0))) : 0;
  __syncthreads();  // (sums are written again)
  return before + run - x;
}

// The free pages of lowest index, ascending, to out[0 .. most): -> how many there are (at most `most` are looked for)
__device__ int lowest_free(const PoolView& p, int most, int* out, int* sums) {
  int found = 0;
  for (int base = 0; base < p.n_pages && found < most; base += 4 * kPlan) {
    const int at = base + 4 * (int)threadIdx.x;
    int mine = 0, bits = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (at + e < p.n_pages && ld_agent(p.refs + at + e) == 0) {
        bits |= 1 << e;
        ++mine;
      }
    int total;
    int rank = found + scan_before(mine, sums, &total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (bits >> e & 1) {
        if (rank < most) out[rank] = at + e;
        ++rank;
      }
    found += total;
  }
  return min(found, most);
}

enum { FORK, EXTEND, IMPORT };

struct PlanArgs {
  PoolView p;
  const int *src, *dst;  // dst: the sequences that change
  int n, tokens, deep, want_len;
  int* out_pos;
};

// What an entry asks for: the sequence that changes (-1: the entry is ignored) and its source, pages it holds before (and
// loses, but for EXTEND), pages after, fresh ones, length of the source, first fresh page (in copy_dst)
constexpr int kMost = VLAC_PAGES_MAX_LIST;
struct Entries { int dst[kMost], src[kMost], held[kMost], pages[kMost], len[kMost], first[kMost + 1]; };

// One workgroup, which looks every entry up once and keeps it in LDS.  Everything or nothing: the destinations' pages are
// released, the fresh pages looked for, and if they do not suffice the release is taken back.  A chain of reads (list, lengths,
// tables of what is released, refs, tables of the sources), about 1 us each: fork of 16 entries 5.5 to 6.8 us, extend 2.8 (4
// entries) to 4.8 (16).
template <int MODE>
__global__ __launch_bounds__(kPlan) void pages_plan_kernel(PlanArgs a) {
  __shared__ int sums[kPlan / 64];
  __shared__ Entries es;
  __shared__ int s_flags;  // 1: an entry is ignored, 2: pages are released
  const PoolView& p = a.p;
  read_args(a.src, a.dst, a.n, a.tokens, a.deep, a.want_len, a.out_pos, p.refs, p.table, p.len, p.scratch, p.n_pages, p.max_seqs,
            p.max_pages);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int* const fresh_pages = p.copy_dst();
  if (tid == 0) s_flags = 0;

  // Only the first entry of a sequence counts, and none whose sequence is a source.  Short lists are compared in LDS, 32 lanes
  // per entry, long ones by marks in the scratch (a round trip more, but no square of the length).
  const bool marks = a.n > 256;
  for (int i = tid; i < a.n; i += kPlan) {
    const int d = a.dst[i], s = MODE == FORK ? a.src[i] : 0;
    es.dst[i] = d;
    es.src[i] = s;
    es.first[i] = 0;  // (until then: 1 if the entry does not count)
    if (marks) {
      if ((unsigned)d < (unsigned)p.max_seqs) atomicMax(p.is_dst() + d, a.n - i);
      if (MODE == FORK && (unsigned)s < (unsigned)p.max_seqs) atomicOr(p.is_src() + s, 1);
    }
  }
  if (marks) {
    meet();
  } else {
    __syncthreads();
    for (int i = tid >> 5; i < a.n; i += kPlan / 32) {
      const int d = es.dst[i];
      bool out = false;
      for (int k = lane & 31; k < a.n; k += 32) out |= (k < i && es.dst[k] == d) || (MODE == FORK && es.src[k] == d);
      if (out) es.first[i] = 1;
    }
    __syncthreads();
  }
  int need = 0;
  for (int base = 0; base < a.n; base += kPlan) {
    const int i = base + tid;
    int fresh = 0, d = -1;
    if (i < a.n) {
      d = es.dst[i];
      const int s = es.src[i];
      const int ld = checked_len(p, d), ls = MODE == FORK ? checked_len(p, s) : 0;
      bool ok = ld >= 0 && ls >= 0;
      if (marks) {
        ok = ok && ld_agent(p.is_dst() + d) == a.n - i && (MODE != FORK || ld_agent(p.is_src() + d) == 0);
      } else {
        ok = ok && es.first[i] == 0;
      }
      if (MODE == EXTEND)
        ok = ok && (long long)ld + a.tokens <= (long long)p.max_pages * kPage && (a.want_len < 0 || ld == a.want_len);
      const int len = MODE == FORK ? ls : MODE == EXTEND ? ld : a.tokens;
      const int held = ok ? pages_of(ld) : 0, pages = ok ? pages_of(MODE == EXTEND ? ld + a.tokens : len) : 0;
      if (ok) fresh = MODE == EXTEND ? pages - held : MODE == IMPORT || a.deep ? pages : (len % kPage != 0);
      es.held[i] = held;
      es.pages[i] = pages;
      es.len[i] = len;
      if (!ok) atomicOr(&s_flags, 1);
      else if (MODE != EXTEND && held > 0) atomicOr(&s_flags, 2);
      d = ok ? d : -1;
    }
    int total;
    const int before = scan_before(fresh, sums, &total);
    if (i < a.n) {
      es.first[i] = need + before;
      es.dst[i] = d;
    }
    need += total;
  }
  __syncthreads();
  if (marks)  // (before out_pos is written, which may lie over the list)
    for (int i = tid; i < a.n; i += kPlan) {
      const int d = a.dst[i], s = MODE == FORK ? a.src[i] : -1;
      if ((unsigned)d < (unsigned)p.max_seqs) p.is_dst()[d] = 0;
      if ((unsigned)s < (unsigned)p.max_seqs) p.is_src()[s] = 0;
    }
  if (tid == 0 && (s_flags & 1)) report(p, PAGES_BAD_ENTRY);
  const bool releases = (s_flags & 2) != 0;
  // (by `by` = -1 released, by +1 taken back)
  auto release = [&](int by) {
    for (int i = w; i < a.n; i += kPlan / 64) {
      const int d = es.dst[i];
      if (d < 0) continue;
      for (int j = lane; j < es.held[i]; j += 64) {
        const int pg = p.table[(size_t)d * p.max_pages + j];
        if ((unsigned)pg < (unsigned)p.n_pages) atomicAdd(p.refs + pg, by);
        else report(p, PAGES_BAD_ENTRY);
      }
    }
  };
  if (releases) {
    release(-1);
    meet();
  }
  const int found = need > 0 ? lowest_free(p, min(need, p.n_pages), fresh_pages, sums) : 0;
  meet();
  const bool room = found >= need;
  if (!room) {
    if (releases) release(1);
    if (tid == 0) report(p, PAGES_NO_ROOM);
  }
  if (tid == 0) p.scratch[PG_COPIES] = room && MODE != EXTEND ? need : 0;
  if (MODE == EXTEND)
    for (int i = tid; i < a.n; i += kPlan) a.out_pos[i] = room && es.dst[i] >= 0 ? es.len[i] : -1;
  if (room) {
    for (int i = w; i < a.n; i += kPlan / 64) {
      const int d = es.dst[i];
      if (d < 0) continue;
      const int held = es.held[i], pages = es.pages[i], len = es.len[i], first = es.first[i];
      int* const row = p.table + (size_t)d * p.max_pages;
      const int* const from = p.table + (size_t)es.src[i] * p.max_pages;
      const int kept = MODE == EXTEND ? held : MODE == FORK && !a.deep ? len / kPage : 0;  // pages that are not fresh
      for (int j = (MODE == EXTEND ? held : 0) + lane; j < max(held, pages); j += 64) {
        int pg = -1;
        if (j < pages) {
          if (j < kept) {
            pg = from[j];
          } else {
            const int f = first + j - kept;
            pg = fresh_pages[f];
            if (MODE == FORK) {
              const int of = from[j];
              p.copy_src()[f] = of;
              if ((unsigned)of >= (unsigned)p.n_pages) report(p, PAGES_BAD_ENTRY);  // (not copied)
            }
            if (MODE == IMPORT) p.copy_src()[f] = i << 16 | j;
          }
          if ((unsigned)pg < (unsigned)p.n_pages) atomicAdd(p.refs + pg, 1);
          else report(p, PAGES_BAD_ENTRY);
        }
        row[j] = pg;
      }
      if (lane == 0) p.len[d] = MODE == EXTEND ? len + a.tokens : len;
    }
  }
}

// copy_src -> copy_dst, whole pages; how many of them only the device knows.  A workgroup takes 16 KiB at a time, four
// loads in flight per thread.  REMAP: also lets the tables follow (compact).  Bound by memory: 13 last pages of 16 MiB from two
// sources in 40 us (33 MB read, 218 written), 92 MB of whole pages in 27.  The stores are non-temporal: with plain ones 49 and 28 us,
// 605 MB of a pool's moves 101 us, now 82 (loads marked so as well: 92).
__device__ inline void st_stream(uint4* p, const uint4& x) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4*)p); }
constexpr int kChunk = 1024;  // 16-byte words of a work item
template <bool REMAP>
__global__ __launch_bounds__(256) void pages_copy_kernel(PoolView p, long long page16) {
  const int n = ld_scalar(p.scratch + PG_COPIES);
  const int chunks = (int)((page16 + kChunk - 1) / kChunk);
  const long long items = (long long)n * chunks;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int k = (int)(it / chunks), c = (int)(it - (long long)k * chunks);
    const int from = ld_scalar(p.copy_src() + k), to = ld_scalar(p.copy_dst() + k);
    if ((unsigned)from >= (unsigned)p.n_pages) continue;
    const uint4* s = (const uint4*)p.data + (long long)from * page16;
    uint4* d = (uint4*)p.data + (long long)to * page16;
    const long long at = (long long)c * kChunk + threadIdx.x;
    // (a page is a multiple of 512 words: the last item holds two or four of a thread's words)
    const uint4 x0 = s[at], x1 = s[at + 256];
    if ((long long)(c + 1) * kChunk <= page16) {
      const uint4 x2 = s[at + 512], x3 = s[at + 768];
      st_stream(d + at + 512, x2);
      st_stream(d + at + 768, x3);
    }
    st_stream(d + at, x0);
    st_stream(d + at + 256, x1);
  }
  if (REMAP && n > 0) {
    const int live = ld_scalar(p.scratch + PG_COPIES + 1);
    for (int s = blockIdx.x; s < p.max_seqs; s += gridDim.x) {
      const int l = checked_len(p, s);
      if (l < 0 && threadIdx.x == 0) report(p, PAGES_BAD_ENTRY);
      for (int j = threadIdx.x; j < (l > 0 ? pages_of(l) : 0); j += 256) {
        int* at = p.table + (size_t)s * p.max_pages + j;
        const int pg = *at;
        if ((unsigned)pg >= (unsigned)p.n_pages) report(p, PAGES_BAD_ENTRY);
        else if (pg >= live) *at = p.moved_to()[pg];
      }
    }
  }
}

// Tiles of the streams' cache into fresh pages: work item = (page, layer, K or V, kv head); a tile of 4 or 8 KiB is the
// longest piece that lies together on both sides.  Bound by memory: 34 pages of 4 MiB (285 MB read and written) in 46 us, 9 in 13.
__global__ __launch_bounds__(256) void pages_import_kernel(PoolView p, const uint4* cache, long long stream16, int max_seq) {
  const int n = ld_scalar(p.scratch + PG_COPIES);
  const int tile16 = (int)(p.tile() / 8), heads = p.n_layers * 2 * p.n_kv_heads;
  const long long items = (long long)n * heads, head16 = (long long)max_seq * p.head_dim / 8, page16 = (long long)heads * tile16;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int k = (int)(it / heads), h = (int)(it - (long long)k * heads);
    const int from = ld_scalar(p.copy_src() + k), to = ld_scalar(p.copy_dst() + k);
    const uint4* s = cache + (from >> 16) * stream16 + h * head16 + (long long)(from & 0xffff) * tile16;
    uint4* d = (uint4*)p.data + to * page16 + (long long)h * tile16;
    for (int i = threadIdx.x; i < tile16; i += 256) d[i] = s[i];
  }
}

__global__ __launch_bounds__(256) void pages_reset_kernel(PoolView p, int scratch_words) {
  const long long rows = (long long)p.max_seqs * p.max_pages, step = (long long)gridDim.x * 256;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  for (long long i = at; i < rows; i += step) p.table[i] = -1;
  for (long long i = at; i < p.n_pages; i += step) p.refs[i] = 0;
  for (long long i = at; i < p.max_seqs; i += step) p.len[i] = 0;
  for (long long i = at; i < scratch_words; i += step) p.scratch[i] = 0;
}

// One workgroup per entry; whoever takes the length of a sequence first releases its pages.  (2.5 us: the exchange of the
// length, the row, the counts, one behind the other.)
__global__ __launch_bounds__(256) void pages_free_kernel(PoolView p, const int* __restrict__ seqs) {
  __shared__ int s_len;
  const int s = seqs[blockIdx.x];
  if ((unsigned)s >= (unsigned)p.max_seqs) {
    if (threadIdx.x == 0) report(p, PAGES_BAD_ENTRY);
    return;
  }
  if (threadIdx.x == 0) s_len = atomicExch(p.len + s, 0);
  __syncthreads();
  int l = s_len;
  if (l < 0 || l > p.max_pages * kPage) {
    if (threadIdx.x == 0) {
      atomicExch(p.len + s, l);  // (left as it was; another entry of the same sequence finds this or 0)
      report(p, PAGES_BAD_ENTRY);
    }
    return;
  }
  for (int j = threadIdx.x; j < pages_of(l); j += 256) {
    int* at = p.table + (size_t)s * p.max_pages + j;
    const int pg = *at;
    *at = -1;
    if ((unsigned)pg < (unsigned)p.n_pages) atomicAdd(p.refs + pg, -1);
    else report(p, PAGES_BAD_ENTRY);
  }
}

// One workgroup: counts the pages in use, then pairs those at or beyond the count with the free ones below it.  A thread
// takes 8 pages side by side, all of them asked for at once (301 pages 4.6 us, 5003 pages 5.5).
__global__ __launch_bounds__(kPlan) void pages_compact_kernel(PoolView p, int* out_live) {
  __shared__ int sums[kPlan / 64];
  constexpr int PER = 8, ROUND = PER * kPlan;
  read_args(p.refs, p.scratch, p.n_pages, out_live);
  const int tid = threadIdx.x;
  int used = 0;  // bits of this thread's pages (of the last round)
  auto look = [&](int base) {
    int r[PER];
    const int at = base + PER * tid;
#pragma unroll
    for (int e = 0; e < PER; ++e) r[e] = at + e < p.n_pages ? p.refs[at + e] : 0;
    used = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) used |= (r[e] > 0) << e;
  };
  int mine = 0;
  for (int base = 0; base < p.n_pages; base += ROUND) {
    look(base);
    mine += __popc(used);
  }
  int live;
  (void)scan_before(mine, sums, &live);
  int holes = 0, moves = 0;  // (equal in the end)
  for (int base = 0; base < p.n_pages; base += ROUND) {
    if (p.n_pages > ROUND) look(base);
    const int at = base + PER * tid;
    const int below = live <= at ? 0 : live >= at + PER ? (1 << PER) - 1 : (1 << (live - at)) - 1;
    const int in = p.n_pages >= at + PER ? (1 << PER) - 1 : p.n_pages <= at ? 0 : (1 << (p.n_pages - at)) - 1;
    const int hole = ~used & below & in, move = used & ~below;
    int total;
    const int before = scan_before(__popc(hole) << 16 | __popc(move), sums, &total);
    int to = holes + (before >> 16), from = moves + (before & 0xffff);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (hole >> e & 1) p.copy_dst()[to++] = at + e;
      if (move >> e & 1) p.copy_src()[from++] = at + e;
    }
    holes += total >> 16;
    moves += total & 0xffff;
  }
  meet();
  for (int k = tid; k < moves; k += kPlan) {
    const int from = p.copy_src()[k], to = p.copy_dst()[k];
    p.moved_to()[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (tid == 0) {
    p.scratch[PG_COPIES] = moves;
    p.scratch[PG_COPIES + 1] = live;
    *out_live = live;
  }
}

// K and V of new tokens.  A wave takes 64 features of a head at 8 positions that lie side by side in a page (so that what is
// asked of the tables is one page, by scalar loads, and a K store of 8 lanes is a line): 16 bytes of a row per lane for
// K, and for V, whose 4 neighbouring positions lie side by side, turned round in LDS, a feature per lane.  Bound by the latency
// of the table (list and position, then length, table and count of the page, then the stores): 8 tokens of 32 heads of 128 in 3.3 us,
// 32 entries x 56 tokens of 2 heads (3.7 MB) in 3.7.
// TILES: the rows come from tiles (one token per entry), else from rows.
struct AppendArgs {
  PoolView p;
  int layer, n, tokens, add, blocks;  // blocks: of 8 positions that an entry's tokens may touch
  const int *seqs, *pos;
  const bf16_t *k, *v;
  long long row_stride;
  int first;  // wave of the call that this launch begins with
};
template <bool TILES>
__global__ __launch_bounds__(256) void pages_append_kernel(AppendArgs a) {
  __shared__ uint4 turn[4][64];
  const PoolView& p = a.p;
  read_args(a.layer, a.n, a.tokens, a.add, a.blocks, a.seqs, a.pos, a.k, a.v, a.row_stride, a.first, p.data, p.refs, p.table, p.len, p.n_pages,
            p.max_seqs, p.max_pages, p.n_layers, p.n_kv_heads, p.head_dim);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 7, r8 = lane >> 3;
  const int per_block = p.n_kv_heads * (p.head_dim >> 6);  // waves for a block of positions
  const int u = a.first + blockIdx.x * 4 + w, ib = u / per_block, hf = u - ib * per_block, i = ib / a.blocks, blk = ib - i * a.blocks;
  if (i >= a.n) return;
  const int h = hf / (p.head_dim >> 6), f0 = (hf - h * (p.head_dim >> 6)) * 64;
  const int p0 = ld_scalar(a.pos + i), s = ld_scalar(a.seqs + i);
  if (p0 < 0) return;
  const long long first = (long long)p0 + a.add, at8 = (first / 8 + blk) * 8;  // the block's first position
  if (at8 >= first + a.tokens) return;
  const int t = (int)(at8 + r8 - first);  // this lane's token
  const bool mine = t >= 0 && t < a.tokens;
  // (the values are asked for before it is known whether they have a place)
  uint4 k8 = make_uint4(0, 0, 0, 0), v8 = k8;
  if (!TILES && mine) {
    const size_t src = ((size_t)i * a.tokens + t) * a.row_stride + (size_t)h * p.head_dim + f0 + 8 * c;
    k8 = *(const uint4*)(a.k + src);
    v8 = *(const uint4*)(a.v + src);
  }
  const bool known = (unsigned)s < (unsigned)p.max_seqs;
  const int l = known ? ld_scalar(p.len + s) : -1;
  const long long j = at8 / kPage;
  int pg = known && j < p.max_pages ? ld_scalar(p.table + (size_t)s * p.max_pages + j) : -1;
  const bool whole = l >= 0 && l <= p.max_pages * kPage && min(at8 + 8, first + a.tokens) <= l;  // (all of the block's tokens lie inside)
  if ((unsigned)pg >= (unsigned)p.n_pages || ld_scalar(p.refs + pg) != 1) pg = -1;
  if (lane == 0 && (pg < 0 || !whole)) report(p, PAGES_BAD_ENTRY);
  if (pg < 0 || l < 0 || l > p.max_pages * kPage) return;
  const bool store = mine && at8 + r8 < l;
  const int r = ((int)at8 & 31) + r8;
  const size_t tile = p.tile();
  bf16_t* kd = p.data + (size_t)pg * p.page() + ((size_t)a.layer * 2 * p.n_kv_heads + h) * tile + (size_t)f0 * 32;
  bf16_t* vd = kd + p.n_kv_heads * tile;
  const size_t k_at = (size_t)(c >> 1) * 512 + (c & 1) * 256 + r * 8;  // (f0: 64 features are 2048 values of either tile)
  // feature f0 + lane at position (at8 & 31) + 4 g of the V tile
  auto v_at = [&](int g) {
    return (size_t)(lane >> 5) * 1024 + (((int)at8 & 31) >> 4) * 512 + g * 256 + (lane & 31) * 8 + (((int)at8 >> 3) & 1) * 4;
  };
  if (TILES) {
    const bf16_t* ks = a.k + ((size_t)i * 2 * p.n_kv_heads + h) * tile + (size_t)f0 * 32;
    const bf16_t* vs = ks + p.n_kv_heads * tile;
    if (store) *(uint4*)(kd + k_at) = *(const uint4*)(ks + k_at);
    const int one = (int)(first - at8);  // the token's place among the 8 positions (inside: checked above)
    const size_t x = v_at(one >> 2) + (one & 3);
    if (first < l) vd[x] = vs[x];
    return;
  }
  if (store) *(uint4*)(kd + k_at) = k8;
  turn[w][lane] = v8;  // [position][64 features]
  asm volatile("" ::: "memory");  // (read as another type below: the order is the wave's own, if the compiler keeps it)
  const bf16_t* rows = (const bf16_t*)turn[w] + lane;
  const unsigned long long places = __ballot(store);  // (8 lanes each)
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = rows[(4 * g + e) * 64];
    bf16_t* d = vd + v_at(g);
    const uint32_t four = (uint32_t)(places >> (32 * g));
    if (four == 0xffffffffu) {
      *(uint2*)d = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (four >> (8 * e) & 1) d[e] = (bf16_t)y[e];
    }
  }
}

size_t scratch_words(const vlac_pages* p) { return PG_LISTS + 3 * (size_t)p->n_pages + 2 * (size_t)p->max_seqs; }

// Workgroups that copy up to `most` pages of `items` work items each
int copy_grid(long long most, long long items) { return (int)std::max(1LL, std::min(most * items, 2048LL)); }

int check_list(const vlac_pages* p, int n) {
  const int rc = check_pages(p, true);
  if (rc != VLAC_OK) return rc;
  return n < 0 || n > VLAC_PAGES_MAX_LIST ? VLAC_E_RANGE : VLAC_OK;
}

int launched() { return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP; }

}  // namespace

int check_pages(const vlac_pages* p, bool pointers) {
  if (!p) return VLAC_E_NULL;
  if (p->n_layers < 1 || p->n_layers > 512 || p->n_kv_heads < 1 || p->n_kv_heads > 1024 || p->n_pages < 1 ||
      p->n_pages > 1 << 24 || p->max_seqs < 1 || p->max_seqs > 65536 || p->max_pages < 1 || p->max_pages > 32768)
    return VLAC_E_RANGE;
  if (p->head_dim != 64 && p->head_dim != 128) return VLAC_E_SHAPE;
  if (p->operand_dtype != VLAC_OPERAND_BF16 && p->operand_dtype != VLAC_OPERAND_F16 && p->operand_dtype != VLAC_OPERAND_F16_W8)
    return VLAC_E_RANGE;
  if (pointers) {
    if (!p->data || !p->refs || !p->table || !p->len || !p->scratch) return VLAC_E_NULL;
    if ((uintptr_t)p->data % 16) return VLAC_E_SHAPE;
  }
  return VLAC_OK;
}

void launch_extend(const PoolView& p, const int* seqs, int n, int tokens, int want_len, int* out_pos, hipStream_t st) {
  const PlanArgs a = {p, nullptr, seqs, n, tokens, 0, want_len, out_pos};
  hipLaunchKernelGGL(pages_plan_kernel<EXTEND>, dim3(1), dim3(kPlan), 0, st, a);
}

static void launch_append(bool tiles, AppendArgs a, hipStream_t st) {
  a.blocks = (a.tokens + 14) / 8;
  const long long waves = (long long)a.n * a.blocks * a.p.n_kv_heads * (a.p.head_dim / 64);
  // (a launch of 2^32 threads and more would run only what is left of them modulo 2^32; a call has up to 2^28 waves)
  constexpr int kMost = 1 << 24;
  for (a.first = 0; a.first < waves; a.first += kMost) {
    const dim3 grid((unsigned)((std::min<long long>(waves - a.first, kMost) + 3) / 4));
    if (tiles) hipLaunchKernelGGL(pages_append_kernel<true>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(pages_append_kernel<false>, grid, dim3(256), 0, st, a);
  }
}

void launch_append_tiles(const PoolView& p, int layer, const int* seqs, const int* pos, int add, int n,
                         const bf16_t* tiles, hipStream_t st) {
  const AppendArgs a = {p, layer, n, 1, add, 0, seqs, pos, tiles, nullptr, 0, 0};
  launch_append(true, a, st);
}

extern "C" {

size_t vlac_page_bytes(const vlac_pages* pages) {
  return check_pages(pages, false) == VLAC_OK ? pool_view(pages).page() * sizeof(bf16_t) : 0;
}

size_t vlac_pages_scratch_bytes(const vlac_pages* pages) {
  return check_pages(pages, false) == VLAC_OK ? scratch_words(pages) * sizeof(int) : 0;
}

int vlac_pages_reset(const vlac_pages* pages, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  hipLaunchKernelGGL(pages_reset_kernel, dim3(512), dim3(256), 0, (hipStream_t)stream, pool_view(pages), (int)scratch_words(pages));
  return launched();
}

int vlac_pages_check(const vlac_pages* pages, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  int word = 0;
  if (hipMemcpyAsync(&word, pages->scratch + PG_STATUS, sizeof(int), hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return VLAC_E_HIP;
  if (!word) return VLAC_OK;
  if (hipMemsetAsync(pages->scratch + PG_STATUS, 0, sizeof(int), st) != hipSuccess || hipStreamSynchronize(st) != hipSuccess)
    return VLAC_E_HIP;
  return word & PAGES_NO_ROOM ? VLAC_E_NOMEM : VLAC_E_RANGE;
}

int vlac_pages_import(vlac_ctx* ctx, const void* kv_cache, int B, int L, const vlac_pages* pages, const int32_t* seqs,
                      void* stream) {
  if (!ctx || !kv_cache || !seqs) return VLAC_E_NULL;
  const int rc = check_list(pages, B);
  if (rc != VLAC_OK) return rc;
  const vlac_model_cfg& m = ctx->cfg;
  if (B < 1 || B > m.max_batch || L < 1) return VLAC_E_RANGE;
  if (L > m.max_seq || (long long)L > (long long)pages->max_pages * kPage || pages->n_layers != m.n_layers ||
      pages->n_kv_heads != m.n_kv_heads || pages->head_dim != m.head_dim || pages_f16(pages) != ctx->f16)
    return VLAC_E_SHAPE;
  for (int b = 0; b < B; ++b)
    if (!ctx->filled[b]) return VLAC_E_STATE;
  hipStream_t st = (hipStream_t)stream;
  const PoolView p = pool_view(pages);
  const PlanArgs a = {p, nullptr, seqs, B, L, 0, -1, nullptr};
  hipLaunchKernelGGL(pages_plan_kernel<IMPORT>, dim3(1), dim3(kPlan), 0, st, a);
  const long long stream16 = (long long)m.n_layers * 2 * m.n_kv_heads * m.max_seq * m.head_dim / 8;
  const int heads = p.n_layers * 2 * p.n_kv_heads;
  hipLaunchKernelGGL(pages_import_kernel, dim3(copy_grid((long long)B * ((L + 31) / 32), heads)), dim3(256), 0, st, p,
                     (const uint4*)kv_cache, stream16, m.max_seq);
  VLAC_HIP(hipGetLastError());
  return VLAC_OK;
}

int vlac_pages_fork(const vlac_pages* pages, const int32_t* src, const int32_t* dst, int n, int deep, void* stream) {
  const int rc = check_list(pages, n);
  if (rc != VLAC_OK) return rc;
  if (n == 0) return VLAC_OK;
  if (!src || !dst) return VLAC_E_NULL;
  hipStream_t st = (hipStream_t)stream;
  const PoolView p = pool_view(pages);
  const PlanArgs a = {p, src, dst, n, 0, deep != 0, -1, nullptr};
  hipLaunchKernelGGL(pages_plan_kernel<FORK>, dim3(1), dim3(kPlan), 0, st, a);
  const long long page16 = (long long)(p.page() / 8), most = std::min((long long)n * (deep ? p.max_pages : 1), (long long)p.n_pages);
  hipLaunchKernelGGL(pages_copy_kernel<false>, dim3(copy_grid(most, (page16 + kChunk - 1) / kChunk)), dim3(256), 0, st, p, page16);
  return launched();
}

int vlac_pages_extend(const vlac_pages* pages, const int32_t* seqs, int n, int tokens, int32_t* out_pos, void* stream) {
  const int rc = check_list(pages, n);
  if (rc != VLAC_OK) return rc;
  if (tokens < 1 || tokens > 1 << 20) return VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!seqs || !out_pos) return VLAC_E_NULL;
  launch_extend(pool_view(pages), seqs, n, tokens, -1, out_pos, (hipStream_t)stream);
  return launched();
}

int vlac_pages_append(const vlac_pages* pages, int layer, const int32_t* seqs, const int32_t* pos, int n, int tokens,
                      const void* k, const void* v, int64_t row_stride, void* stream) {
  const int rc = check_list(pages, n);
  if (rc != VLAC_OK) return rc;
  if (layer < 0 || layer >= pages->n_layers || tokens < 1 || (long long)n * tokens > 1 << 20) return VLAC_E_RANGE;
  if (row_stride < (int64_t)pages->n_kv_heads * pages->head_dim || row_stride % 8 || row_stride > 1 << 30) return VLAC_E_SHAPE;
  if (n == 0) return VLAC_OK;
  if (!seqs || !pos || !k || !v) return VLAC_E_NULL;
  if ((uintptr_t)k % 16 || (uintptr_t)v % 16) return VLAC_E_SHAPE;
  const AppendArgs a = {pool_view(pages), layer, n, tokens, 0, 0, seqs, pos, (const bf16_t*)k, (const bf16_t*)v, row_stride, 0};
  launch_append(false, a, (hipStream_t)stream);
  return launched();
}

int vlac_pages_free(const vlac_pages* pages, const int32_t* seqs, int n, void* stream) {
  const int rc = check_list(pages, n);
  if (rc != VLAC_OK) return rc;
  if (n == 0) return VLAC_OK;
  if (!seqs) return VLAC_E_NULL;
  hipLaunchKernelGGL(pages_free_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, pool_view(pages), seqs);
  return launched();
}

int vlac_pages_compact(const vlac_pages* pages, int32_t* out_live, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  if (!out_live) return VLAC_E_NULL;
  hipStream_t st = (hipStream_t)stream;
  const PoolView p = pool_view(pages);
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kPlan), 0, st, p, out_live);
  const long long page16 = (long long)(p.page() / 8);
  hipLaunchKernelGGL(pages_copy_kernel<true>,
                     dim3(copy_grid(std::max<long long>(p.n_pages / 2, 1), (page16 + kChunk - 1) / kChunk)), dim3(256), 0, st, p, page16);
  return launched();
}

}  // extern "C"
