// Attention of new tokens over pages, for sequences that share prefixes:
//   out[row] = sum_p exp(s_p - M) v_p / sum_p exp(s_p - M),  s_p = q . k_p / sqrt(head_dim), p <= position of the row.
// The pages that a group's tables have in common at the front (all of them wholly before every query of the group: no mask) are
// read once for all its columns (candidates x tokens x query heads of the kv head), 32 of them to a matrix product, where
// one pass per sequence reads them once for each; the pages behind them are each sequence's own.
//
// A column is a query (entry, token, head of the kv head's group); up to 32 columns are a column block, whose work is a list of key
// tiles: the shared pages, then the own pages of its entries, which only the entry's columns see.  S^T = K Q^T and O^T += V^T P^T
// as in the attention over the stream cache: a page's tiles are the operands as they lie, a lane owns a column.
// A workgroup of 8 waves takes an item: 1, 2 or 4 column blocks side by side (they share the pages) and the key tiles dealt
// to the waves of a block, which meet in LDS.  Where that leaves the chip empty the list is cut into parts, one item each,
// which leave (max, sum, output) in fp32, and a second kernel joins them in the order of the parts:
//   M = max m_i, out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i   (scores in units of log2).
//
// What bounds it, and what it takes (32 query and kv heads of 128, fp16, if not said otherwise):
// * long lists: memory.  48 candidates over 32801 shared positions (554 MB of K and V) 99 to 102 us, 5.5 TB/s, and 5.5 us to join.
// * many columns: what a CU moves into registers, 64 bytes per clock.  Every wave reads the K and V of a tile (16 KiB) for
//   its 32 columns: 16 candidates x 56 tokens over 1057 positions (16 GFLOP) 34 to 36 us, that path busy 73 % of the time, the
//   matrix cores 27 %, the softmax's instructions 37 %; two waves per SIMD overlap them in part.  (28 blocks x 32 heads in items of 4
//   are 224 items: 32 of the 256 CUs have none.)  (Pages staged in LDS for all
//   blocks of an item: 35 us as against 32 then, the meetings of the waves cost what the reads save; two column blocks per wave in 4
//   waves of 512 registers: 42, one wave per SIMD does not hide its own softmax; two per wave in 8 waves, queries in LDS: 36 to
//   46, no registers are left for K and V to be asked for ahead.)
// * short lists: the chain launch arguments - item - tables - pages, 2.6 us to the first product, then 1.4 us for every tile of
//   a wave (one after the other here; two at a time in the kernel for few columns), 1.5 us to meet and store: 12 query heads on 2 kv
//   heads, 32 groups of up to 8 candidates over 304 positions, bf16, 13 MB: 10 us, 8.5 with few columns; two candidates over 80
//   positions, 4 heads of 64: 5.5 and 5.2.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace {

constexpr int kWaves = 8;            // of a workgroup; one workgroup per CU (256 registers a wave)
constexpr int kCus = 256;
constexpr int kLong = 64;            // pages of a list from which on it may be cut
constexpr int kMaxParts = 64;
constexpr int kPartTiles = 2048;     // column blocks x parts that the workspace holds at most

// What a row has to know, per entry: row of the table (-1: the entry is ignored), position of its first query
struct Ent { int seq, pos; };
// A step over a page of an entry's own: page | valid positions of it << 24, tile | entry of the group << 16
struct Own { uint32_t page, what; };
// A work item: column blocks (of `width` columns) block0 .. block0 + waves_c - 1 of head `head` of the group that begins at entry
// e0, part `part` of `parts` of their key tiles: pages s0 .. s1 - 1 of sequence seq, and own_n[i] steps from own_at[i] on for block0 + i.
// tile: where block0's parts lie.
struct Item {
  int e0, seq, head, block0, waves_c, part, parts, cols, s0, s1, tile, width, own_at[4], own_n[4];
};
static_assert(sizeof(Item) == 80, "read as twenty words");
__device__ inline Item load_item(const Item* at) {
  Item x;
  x.e0 = ld_scalar(&at->e0); x.seq = ld_scalar(&at->seq); x.head = ld_scalar(&at->head); x.block0 = ld_scalar(&at->block0);
  x.waves_c = ld_scalar(&at->waves_c); x.part = ld_scalar(&at->part); x.parts = ld_scalar(&at->parts); x.cols = ld_scalar(&at->cols);
  x.s0 = ld_scalar(&at->s0); x.s1 = ld_scalar(&at->s1); x.tile = ld_scalar(&at->tile); x.width = ld_scalar(&at->width);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x.own_at[k] = ld_scalar(at->own_at + k);
    x.own_n[k] = ld_scalar(at->own_n + k);
  }
  return x;
}

struct Layout {
  size_t ent, own, item, ml, o, total;
  size_t max_items;
  int part_tiles;
  bool parts;  // there may be parts to join
  bool few;    // blocks of up to 16 columns
};
inline Layout layout_of(const PoolView& p, int n, int tokens, int n_q_heads) {
  Layout l;
  const size_t cols = (size_t)n * tokens * (n_q_heads / p.n_kv_heads);  // per kv head
  const size_t least = (cols + 31) / 32 * p.n_kv_heads;
  // Parts where the column blocks do not fill the chip by themselves and the tables have room for lists that are long
  // for 8 waves.  That is all that the host knows: it decides whether the second kernel is launched (2.5 us where it finds nothing to
  // join) and, below, which kernel the first is.  Short lists in wide tables pay for it: 8 candidates over 288 positions 7.3 us a
  // layer with up to 64 columns, 10.4 with more; 2 groups of up to 8 x 8 tokens over 601 11.9 and 14.7.
  l.parts = least < 2 * kCus && p.max_pages > kLong;
  // Blocks of up to 16 columns where one round of the chip holds all of them: 6.8 us, and 8.1 with blocks of 32, for 8 candidates
  // over 288 positions (32 heads of 128), 14.7 and 16.3 for 60 over 300, 19.2 and 21.3 for 100.  In more than a round the pages
  // are read too often: 150 over 300 34.1 and 28.1, grouped queries, 120 groups of up to 8 over 304, 24.7 and 21.3.
  l.few = !l.parts && cols <= (size_t)16 * n && (cols + 15) / 16 * p.n_kv_heads <= kCus;
  const size_t max_blocks = (l.few ? (cols + 15) / 16 * p.n_kv_heads : least) + (size_t)n * p.n_kv_heads;  // (a group ends in a block of its own)
  l.part_tiles = l.parts ? (int)std::min<size_t>(kPartTiles, max_blocks * kMaxParts) : 0;
  l.max_items = max_blocks + l.part_tiles;
  if (p.n_kv_heads < 8) l.max_items += l.max_items / 2;  // (runs of an XCD may leave places empty)
  l.max_items = (l.max_items + 7) / 8 * 8;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  l.ent = 256;
  l.own = l.ent + up(sizeof(Ent) * n);
  l.item = l.own + up(sizeof(Own) * n * p.max_pages);
  l.ml = l.item + up(sizeof(Item) * l.max_items);
  l.o = l.ml + (size_t)l.part_tiles * 64 * sizeof(float2);
  l.total = l.o + (size_t)l.part_tiles * 32 * p.head_dim * sizeof(float);
  return l;
}

// What a plan was made for, behind the number of items in the workspace: a workspace that holds another plan, or none, is
// not read any further.
struct Made { int v[15]; };
inline Made made_for(const PoolView& p, int n, int tokens, int n_q_heads) {
  const uint64_t d = (uint64_t)(uintptr_t)p.data, t = (uint64_t)(uintptr_t)p.table;
  return {{0x564c4150, n, tokens, n_q_heads, p.n_layers, p.n_kv_heads, p.head_dim, p.n_pages, p.max_seqs, p.max_pages, (int)d,
           (int)(d >> 32), (int)t, (int)(t >> 32), kWaves}};
}
__device__ inline int differs(const int* head, const Made& m) {
  int x = 0;
#pragma unroll
  for (int i = 0; i < 15; ++i) x |= ld_scalar(head + 1 + i) ^ m.v[i];
  return x;
}

struct PlanArgs {
  PoolView p;
  Made made;
  const int *seqs, *pos, *group;
  int add, n, tokens, n_q_heads, part_tiles, max_items, width;
  int* head;  // [0] places for items, [1] what it was made for
  Ent* ent;
  Own* own;
  Item* item;
};

// Sums of two numbers over the threads before this one, and over all
struct Two { int a, b; };
template <int NT>
__device__ inline Two scan_before(Two x, Two* sums, Two* total) {
  static_assert(NT <= 1024, "the waves' sums are a row of lanes");
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Two run = {wave_sums(x.a), wave_sums(x.b)};
  if (lane == 63) sums[w] = run;
  __syncthreads();
  // (every wave adds the sums of all of them for itself: no second meeting)
  const Two mine = (lane & 15) < NT / 64 ? sums[lane & 15] : Two{0, 0};
  const Two s = {row_sums(mine.a), row_sums(mine.b)};
  *total = {__builtin_amdgcn_readlane(s.a, 15), __builtin_amdgcn_readlane(s.b, 15)};
  const int last = max(w - 1, 0);
  const Two before = {(w > 0 ? __builtin_amdgcn_readlane(s.a, last) : 0) + run.a - x.a,
                      (w > 0 ? __builtin_amdgcn_readlane(s.b, last) : 0) + run.b - x.b};
  __syncthreads();
  return before;
}

// How a group is cut: column blocks, of which `waves_c` are side by side in an item
struct Cut { int blocks, waves_c, chunks, wk; };
__device__ inline Cut cut_of(int cols, int log_most, int width) {
  Cut x;
  x.blocks = (int)((unsigned)(cols + width - 1) / (unsigned)width);
  const int log = min(x.blocks >= 3 ? 2 : x.blocks >> 1, log_most);
  x.waves_c = 1 << log;
  x.chunks = (x.blocks + x.waves_c - 1) >> log;
  x.wk = kWaves >> log;
  return x;
}

// One workgroup.  Groups and their common pages, then the cut, then the items.  Memory is asked for in three rounds
// (lists, lengths, tables), all else is in LDS.  Bound by latency: two candidates 7.3 us, 32 groups of up to 8 candidates 9.2, 48
// entries of 1027 pages 20 to 23 (9 of them the comparison of the tables).
// (NT threads and room for N entries: a workgroup of 4 waves meets sooner than one of 16)
template <int NT, int N>
__global__ __launch_bounds__(NT) void attend_plan_kernel(PlanArgs a) {
  __shared__ Two sums[NT / 64];
  __shared__ int g_start[N + 1], g_lead[N], g_shared[N], g_own[N], q_item[N + 1], g_tile[N], l_seq[N], l_pos[N], l_own[N + 1];
  __shared__ unsigned short l_group[N];
  __shared__ int s_run[9], s_bad, s_width, s_steps, s_longest, s_blocks, s_area, s_own, s_cols;
  __shared__ unsigned long long s_work;
  const PoolView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  read_args(a.seqs, a.pos, a.group, a.add, a.n, a.tokens, a.n_q_heads, a.part_tiles, a.max_items, a.head, a.ent, a.own,
            a.item, p.table, p.len, p.max_seqs, p.max_pages, p.n_kv_heads);
  const int hkv = p.n_kv_heads, grp = a.n_q_heads / hkv, per_entry = a.tokens * grp;  // columns of an entry per kv head
  if (tid == 0) {
    s_bad = s_width = s_longest = s_blocks = s_area = s_own = 0;
    s_work = 0;
  }
  for (int g = tid; g < a.n; g += NT) g_own[g] = 0;

  int n_groups = 0;
  for (int base = 0; base < a.n; base += NT) {
    const int i = base + tid, ii = min(i, a.n - 1);
    const int label = a.group ? a.group[ii] : 0, label_before = a.group ? a.group[max(ii - 1, 0)] : 0;
    const int s = a.seqs[ii], p0 = a.pos[ii];
    const int l = checked_len(p, s);
    const bool start = i < a.n && (i == 0 || label != label_before);
    Two total;
    const Two before = scan_before<NT>({start ? 1 : 0, 0}, sums, &total);
    if (start) {
      const int g = n_groups + before.a;
      g_start[g] = i;
      g_lead[g] = g_shared[g] = 0x7fffffff;
    }
    if (i < a.n) {
      const long long at = (long long)p0 + a.add;
      const bool fits = p0 >= 0 && l >= 0 && at + a.tokens <= l;
      if (p0 >= 0 && !fits) s_bad = 1;
      l_seq[i] = fits ? s : -1;
      l_pos[i] = fits ? (int)at : 0;
      const int g = n_groups + before.a + (start ? 1 : 0) - 1;
      l_group[i] = (unsigned short)g;
      if (fits) atomicMax(&g_own[g], (int)at / kPage);  // (for a while: pages before the group's farthest query)
    }
    n_groups += total.a;
  }
  if (tid == 0) g_start[n_groups] = a.n;
  __syncthreads();
  if (tid == 0 && s_bad) report(p, PAGES_BAD_ENTRY);
  int widest = 0;
  for (int i = tid; i < a.n; i += NT)
    if (l_seq[i] >= 0) {
      atomicMin(&g_lead[l_group[i]], i);
      atomicMin(&g_shared[l_group[i]], l_pos[i] / kPage);
      widest = max(widest, l_pos[i] / kPage);
    }
  widest = wave_max(widest);
  auto group_cols = [&](int g) { return (g_start[g + 1] - g_start[g]) * per_entry; };
  int all_blocks = 0, area = 0;  // (of full width; blocks x pages: no more than the rule below asks for, so that no sum overflows)
  constexpr int kFull = kCus << 15;
  for (int g = tid; g < n_groups; g += NT) {
    const int blocks = (group_cols(g) + a.width - 1) / a.width * hkv;
    all_blocks += blocks;
    area = min(area + min(blocks, 2 * kCus) * g_own[g], kFull);
    g_own[g] = 0;
  }
  all_blocks = wave_sums(all_blocks);
  area = min(wave_sums(area), kFull);  // (of the last lane: all of them)
  if (lane == 63) {
    atomicMax(&s_width, widest);
    atomicAdd(&s_blocks, all_blocks);
    atomicAdd(&s_area, area);
  }
  __syncthreads();
  // Column blocks side by side in an item read their pages together, but have fewer waves each: where the tables have no
  // room for long lists (no parts) and the blocks do not fill the chip otherwise, each is an item by itself.
  // Lists are cut where they are long and the blocks would not fill the chip (half of it, up to 128 pages) while the longest runs:
  // 4 blocks side by side and a second kernel, instead of many blocks that read the same pages from the L2.  Uncut and cut, us: 20 groups
  // of up to 45 over 2300 positions (16 query heads on 4 of 64) 26 and 35, over 6000 55 and 61; 8 x 19 tokens over 2300 (32 heads of
  // 128) 24 and 31; 24 groups of up to 51 over 6000 (8 on 1 of 128, not quite a chip full of blocks) 87 and 66; up to 64 pages: 8
  // candidates over 1400 (32 heads) 12.4 and 14.9, over 2300 18.8 and 17.2.
  const int pages_most = s_width + (a.tokens + kPage - 1) / kPage + 1;
  const int filled = s_area;  // blocks that last as long as it, x its length
  const bool cut = a.part_tiles > 0 && pages_most > kLong &&
                   (filled < kCus / 2 * s_width || (pages_most > 2 * kLong && filled < kCus * s_width));
  const int log_most = a.width < 32 ? 0 : cut || s_blocks > 2 * kCus ? 2 : s_blocks > kCus ? 1 : 0;
  // And where the chip has room for more blocks than that, a block takes as few whole entries as one round of the chip holds:
  // fewer own pages are in its list then (up to 8 candidates a group, 6 columns each, 2 kv heads: 8 groups 10.6 us with blocks
  // of 32 columns, 5 and a third entries, 7.9 with one entry each; 32 groups 11.7, and 10.0 with two entries each and an
  // XCD's runs, below; blocks of 16 for 32 heads: 2 groups of up to 16 over 288 positions 13.2 and 10.0).
  if (w == NT / 64 - 1) {
    int each = 0;  // entries of a block (0: full width, whatever they are)
    if (log_most == 0 && per_entry <= 16 && n_groups * hkv <= kCus) {
      int lo = 1, hi = a.width / per_entry + 1;  // the least that fits, by halving (hi: none does)
      while (lo < hi) {
        const int k = (lo + hi) >> 1;
        const float per = 1.f / (float)k;
        int blocks = 0;
        for (int g = lane; g < n_groups; g += 64) blocks += (int)(((float)(g_start[g + 1] - g_start[g] + k - 1) + 0.5f) * per);
        blocks = __builtin_amdgcn_readlane(wave_sums(blocks), 63);
        if (blocks * hkv <= kCus) hi = k;
        else lo = k + 1;
      }
      each = lo * per_entry <= a.width ? lo : 0;
    }
    if (lane == 0) s_cols = each > 0 ? each * per_entry : a.width;
  }
  // The common pages: every entry's against its group's first.  A wave takes an entry's next 512 pages or, where tables
  // are short, as many entries as they leave lanes for; all of a turn's pages are asked for at once.
  const int width = s_width;
  if (width > 0) {
    const int lanes = width <= 32 ? 4 : width <= 64 ? 8 : width <= 256 ? 32 : 64, per_wave = 64 / lanes;
    const int spans = (width + 8 * lanes - 1) / (8 * lanes), blocks = (a.n + per_wave - 1) / per_wave;
    for (int k = w; k < blocks * spans; k += NT / 64) {
      const int span = k / blocks, i = min((k - span * blocks) * per_wave + lane / lanes, a.n - 1);  // (first spans first)
      const int seq = l_seq[i], g = l_group[i];
      const int lead = seq < 0 ? -1 : l_seq[g_lead[g]], end = g_shared[g], j0 = span * 8 * lanes + lane % lanes;
      if (lead == seq || j0 >= end) continue;
      const int* mine = p.table + (size_t)seq * p.max_pages;
      const int* other = p.table + (size_t)lead * p.max_pages;
      int x[8], y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = min(j0 + lanes * e, end - 1);
        x[e] = mine[j];
        y[e] = other[j];
      }
      int differ = 0x7fffffff;
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (x[e] != y[e]) differ = min(j0 + lanes * e, end - 1);
      if (differ != 0x7fffffff) atomicMin(&g_shared[g], differ);
    }
  }
  __syncthreads();

  for (int g = tid; g < n_groups; g += NT)
    if (g_lead[g] == 0x7fffffff) g_shared[g] = 0;
  __syncthreads();
  const int block_cols = s_cols, entry_blocks = (per_entry + block_cols - 1) / block_cols;
  // own pages of every entry, and where they begin in the list of all of them
  int owned = 0;
  for (int base = 0; base < a.n; base += NT) {
    const int i = base + tid;
    int own = 0;
    if (i < a.n) {
      const int seq = l_seq[i], pos = l_pos[i], g = l_group[i];
      a.ent[i] = {seq, pos};
      if (seq >= 0) {
        own = pages_of(pos + a.tokens) - g_shared[g];
        if (cut) atomicAdd(&g_own[g], own);
      }
    }
    const int longest = wave_max(own);
    if (lane == 0) atomicMax(&s_own, longest);
    Two total;
    const Two before = scan_before<NT>({own, 0}, sums, &total);
    if (i < a.n) l_own[i] = owned + before.a;
    owned += total.a;
  }
  if (tid == 0) l_own[a.n] = owned;
  __syncthreads();
  {
    const int lanes = s_own <= 2 ? 2 : s_own <= 16 ? 8 : 64;
    for (int i = tid / lanes; i < a.n; i += NT / lanes) {
      const int own = l_own[i + 1] - l_own[i], shared = g_shared[l_group[i]];
      for (int t = tid % lanes; t < own; t += lanes) {
        int pg = p.table[(size_t)l_seq[i] * p.max_pages + shared + t];
        if ((unsigned)pg >= (unsigned)p.n_pages) {  // (the table is the caller's)
          pg = 0;
          report(p, PAGES_BAD_ENTRY);
        }
        const int valid = min(l_pos[i] + a.tokens - kPage * (shared + t), kPage);
        a.own[l_own[i] + t] = {(uint32_t)pg | (uint32_t)valid << 24, (uint32_t)(shared + t) | (uint32_t)(i - g_start[l_group[i]]) << 16};
      }
    }
  }
  // Work in steps of a wave, a key tile of a column block: tiles of the list of a group's block.  (An entry's own tiles are dealt
  // to its blocks as if each had them all; a block of tokens before the last sees fewer.)
  if (cut) {
    unsigned long long work = 0;
    int longest = 0;
    for (int g = tid; g < n_groups; g += NT) {
      const Cut x = cut_of(group_cols(g), log_most, block_cols);
      const int tiles = g_shared[g] + (int)ceilf((float)g_own[g] * (float)entry_blocks / (float)max(x.blocks, 1));
      g_own[g] = tiles;  // (from here on: of the whole list of a block)
      work += (unsigned long long)x.blocks * tiles * hkv;
      longest = max(longest, (tiles + x.wk - 1) / x.wk);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) work += __shfl_xor(work, d);
    longest = wave_max(longest);
    if (lane == 0) {
      atomicAdd(&s_work, work);
      atomicMax(&s_longest, longest);
    }
    __syncthreads();
  }
  // Steps of a wave per item: the lanes of the first wave try the longest list in 1, 2, ... 64 parts, and take what
  // ends first: rounds of one item per CU x (steps + 3 for an item's start and end), + 3 for parts that have to be joined.
  // With many groups the chip is full anyhow, and the work per wave is the measure.
  const int most = cut ? max(1, a.part_tiles / max(s_blocks, 1)) : 1;  // parts that the workspace has room for
  auto parts_of = [&](int g, int steps) {
    if (most == 1) return 1;
    const unsigned per_item = (unsigned)min(steps, 1 << 16) * cut_of(group_cols(g), log_most, block_cols).wk;
    return max(1, min(min(most, kMaxParts), (int)((g_own[g] + per_item - 1) / per_item)));
  };
  if (most > 1 && w == 0) {
    int steps = max((s_longest + lane) / (lane + 1), 1), best;
    if (n_groups <= 64) {
      int items = 0, most_steps = 0;  // (the steps that come of it: parts are bounded)
      bool joined = false;
      for (int g = 0; g < n_groups; ++g) {
        const Cut x = cut_of(group_cols(g), log_most, block_cols);
        const int parts = parts_of(g, steps);
        items += hkv * x.chunks * parts;
        most_steps = max(most_steps, (g_own[g] + parts * x.wk - 1) / (parts * x.wk));
        joined |= parts > 1;
      }
      const float cost = (float)((items + kCus - 1) / kCus) * (float)(most_steps + 3) + (joined ? 3.f : 0.f);
      best = (int)fminf(cost, 1e9f);  // (ties: the fewest parts)
      int who = lane;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int c = __shfl_xor(best, d), o = __shfl_xor(who, d);
        if (c < best || (c == best && o < who)) { best = c; who = o; }
      }
      steps = __shfl(steps, who);
    } else {
      steps = (int)max(2ull, min((s_work + kCus * kWaves - 1) / (kCus * kWaves), 1ull << 30));
    }
    if (lane == 0) s_steps = steps;
  }
  if (most > 1) __syncthreads();
  const int steps = s_steps;

  // First item (per kv head) and first partial tile of every group.  Workgroup id % 8 is the XCD, and items that read the same
  // pages belong into one L2.  With 8 kv heads or a multiple of them it is enough that the heads are the fastest index.  With 1, 2
  // or 4 of them the groups are taken residue by residue (mod 8 / heads), and every XCD has a run of items of its own, if
  // the longest run takes no more rounds than the items dealt one by one.
  const int m = hkv < 8 && 8 % hkv == 0 ? 8 / hkv : 1, whole = n_groups / m, rest = n_groups - whole * m;
  auto group_at = [&](int q, int* residue) {  // the q-th group in that order
    *residue = 0;
    if (m == 1) return q;
    const bool longer = q < rest * (whole + 1);
    const int r = longer ? q / (whole + 1) : rest + (q - rest * (whole + 1)) / max(whole, 1);
    *residue = r;
    return (q - r * whole - min(r, rest)) * m + r;
  };
  int items = 0, tiles = 0;
  for (int base = 0; base < n_groups; base += NT) {
    const int q = base + tid;
    int g = 0, residue = 0;
    Two mine = {0, 0};
    if (q < n_groups) {
      g = group_at(q, &residue);
      const Cut x = cut_of(group_cols(g), log_most, block_cols);
      const int parts = parts_of(g, steps);
      mine = {x.chunks * parts, parts > 1 ? hkv * x.blocks * parts : 0};
    }
    Two total;
    const Two before = scan_before<NT>(mine, sums, &total);
    if (q < n_groups) {
      q_item[q] = items + before.a;
      g_tile[g] = tiles + before.b;
      if (g < m) s_run[residue] = items + before.a;  // (the first group of a residue)
    }
    items += total.a;
    tiles += total.b;
  }
  if (tid == 0)
    for (int r = min(m, n_groups); r <= m; ++r) s_run[r] = items;
  __syncthreads();
  int longest_run = 0;
  for (int r = 0; r < m; ++r) longest_run = max(longest_run, s_run[r + 1] - s_run[r]);
  const bool runs = m > 1 && (longest_run + kCus / 8 - 1) / (kCus / 8) <= (items * hkv + kCus - 1) / kCus && 2 * longest_run * m <= 3 * items;
  items *= hkv;
  // Workgroup i takes the items at i, i + grid, ..., so a place is its XCD + 8 x its number there.
  const int places = min(runs ? 8 * longest_run : items, a.max_items);
  items = min(items, a.max_items);
  if (tid < 16) a.head[tid] = tid == 0 ? places : a.made.v[tid - 1];
  if (runs)
    for (int it = tid; it < places; it += NT) {
      const int r = (it & 7) / hkv;
      if (it >> 3 >= s_run[r + 1] - s_run[r]) {  // (nobody's)
        a.item[it].cols = 0;
        a.item[it].parts = 1;
      }
    }
  for (int it = tid; it < items; it += NT) {
    const int u = it / hkv, h = it - u * hkv;
    int q = 0, hi = n_groups;  // the last group that begins at or before this item
    while (hi - q > 1) {
      const int mid = (q + hi) >> 1;
      if (q_item[mid] <= u) q = mid;
      else hi = mid;
    }
    int residue;
    const int g = group_at(q, &residue), c = group_cols(g), parts = parts_of(g, steps);
    const Cut x = cut_of(c, log_most, block_cols);
    const int r1 = u - q_item[q], run = s_run[residue];
    int part = 0, chunk = r1;
    if (most > 1) {
      chunk = r1 / parts;
      part = r1 - chunk * parts;
    }
    Item* im = a.item + (runs ? residue * hkv + h + 8 * (u - run) : it);
    const int e0 = g_start[g], shared = g_shared[g], block0 = chunk * x.waves_c;
    im->e0 = e0; im->seq = g_lead[g] == 0x7fffffff ? 0 : l_seq[g_lead[g]]; im->head = h;
    im->block0 = block0; im->waves_c = x.waves_c; im->part = part; im->parts = parts; im->cols = c; im->width = block_cols;
    im->s0 = part * shared / parts; im->s1 = (part + 1) * shared / parts;
    im->tile = g_tile[g] + (h * x.blocks + block0) * parts;
#pragma unroll 1
    for (int k = 0; k < x.waves_c; ++k) {
      // the own pages of the block's entries, one behind the other; of the last entry those that its tokens of
      // the block see; and the part's share of them
      const int block = block0 + k, last_col = min(block * block_cols + block_cols - 1, c - 1);
      if (block >= x.blocks) break;
      const int lo = e0 + (block * block_cols) / per_entry, e = last_col / per_entry, hi = e0 + e;
      const int seen = l_seq[hi] < 0 ? 0 : (l_pos[hi] + (last_col - e * per_entry) / grp) / kPage + 1 - shared;
      const int all = l_own[hi] + seen - l_own[lo], o0 = part * all / parts;
      im->own_at[k] = l_own[lo] + o0;
      im->own_n[k] = (part + 1) * all / parts - o0;
    }
  }
}

struct AttendArgs {
  PoolView p;
  Made made;
  const int* head;
  const Ent* ent;
  const Own* own;
  const Item* item;
  float2* ml;                // [part tiles][64 lanes] reference point of the exponentials (log2 units) and sum
  float4* o;                 // [part tiles][head_dim / 8][64 lanes] four of a lane's sums of the output
  const bf16_t* q;
  long long q_stride;
  bf16_t* out;
  int kc_out;
  int layer, n, tokens, n_q_heads;
  float scale_log2e;
};

template <bool F16>
__device__ inline uint32_t pack2(float lo, float hi) {
  // (no saturation as elsewhere: what is infinite stays it, and so does a NaN)
  if constexpr (F16) {
    const f32x2v v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2v));
  } else {
    return f2bf2(lo, hi);
  }
}

// How far above a column's maximum (log2) the reference point of its exponentials stands.  In fp32 a sum of weights times values of
// bf16 would pass 2^128 where V is near the end of the type: with weights of up to 2^(8 - 32) and at most 2^20 positions it
// stays below 2^124 (and a weight loses no bits: bf16 has fp32's range).  fp16 values end at 2^16, and its weights need their bits.
template <bool F16>
constexpr float kAbove = F16 ? 0.f : 32.f;

// Masks of the two values of a word that are infinite or NaN, where asked for
template <bool F16>
__device__ inline uint32_t far_values(uint32_t x, bool lo, bool hi) {
  constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;
  return (lo && (x & kExp) == kExp ? 0xffffu : 0u) | (hi && (x >> 16 & kExp) == kExp ? 0xffff0000u : 0u);
}

// Sums over their column's sum of weights (as 1 / sum).  Of finite values that is an average, which lies within their type; but the
// sums' weights are rounded and those of the divisor are not, so that it may come out up to half a step of a weight larger, and
// round to infinity where V is the largest value (an epilogue that saturates leaves those).  Sums that are infinite or NaN stay it.
// (Asked of all R at once, since none is so large as a rule: 56 tokens of 16 candidates over 1057 positions 34.2 to 34.9 us with the
// question and without.)
template <bool F16, int R>
__device__ inline void averages(float (&x)[R], float inv) {
  constexpr float kTop = F16 ? 65504.f : 0x1.fep127f;
  float y[R], most = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    y[r] = x[r] * inv;
    most = fmaxf(most, fabsf(y[r]));
  }
  if (__builtin_expect(__any(most > kTop), 0)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (fabsf(x[r]) < INFINITY && inv < INFINITY) y[r] = __builtin_amdgcn_fmed3f(y[r], -kTop, kTop);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) x[r] = y[r];
}

// The result of a column: features f .. f + 3 of its row
template <int HD, bool F16>
__device__ inline void store_out(const AttendArgs& a, int row, int f, const float* x, bool valid) {
  const uint2 y = valid ? make_uint2(pack2<F16>(x[0], x[1]), pack2<F16>(x[2], x[3])) : make_uint2(0, 0);
  *(uint2*)(a.kc_out > 0 ? a.out + frag_off(row, f, a.kc_out) : a.out + (size_t)row * a.n_q_heads * HD + f) = y;
}

// the first feature of sums 4 * quad .. + 3 of head h: 32 * ib + 8 * q4 + 4 * g, quad = 4 ib + q4
template <int HD>
__device__ inline int feature_of(int h, int quad, int g) { return h * HD + 32 * (quad >> 2) + 8 * (quad & 3) + 4 * g; }

template <int HD, bool F16>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(AttendArgs a) {
  constexpr int NC = HD / 16, NI = HD / 32, REGS = NI * 16;
  __shared__ float park[kWaves][2 + REGS][64];
  const PoolView& p = a.p;
  read_args(a.head, a.item, a.ent, a.q, a.q_stride, a.out, a.kc_out, a.layer, a.tokens, a.n_q_heads, a.scale_log2e, p.data, p.table,
            p.n_pages, p.max_pages, p.n_layers, p.n_kv_heads, a.ml, a.o, a.own);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 31, g = lane >> 5;
  const int grp = a.n_q_heads / p.n_kv_heads, per_entry = a.tokens * grp;
  // (asked for together with what says whether there is such an item)
  Item im = load_item(a.item + blockIdx.x);
  const int n_items = ld_scalar(a.head), differ = differs(a.head, a.made);
  read_args(n_items, differ, im.e0, im.seq, im.head, im.block0, im.waves_c, im.part, im.parts, im.cols, im.s0, im.s1, im.tile,
            im.width, im.own_at[0], im.own_at[1], im.own_at[2], im.own_at[3], im.own_n[0], im.own_n[1], im.own_n[2], im.own_n[3]);
  if (differ) {
    if (blockIdx.x == 0 && tid == 0) report(p, PAGES_BAD_ENTRY);
    return;
  }
  const size_t tile = (size_t)kPage * HD, page = (size_t)p.n_layers * 2 * p.n_kv_heads * tile;
  for (int it = blockIdx.x; it < n_items; it += gridDim.x) {
    if (it != (int)blockIdx.x) im = load_item(a.item + it);
    const int e0 = im.e0, lead = im.seq, hk = im.head, wc = im.waves_c, part = im.part, parts = im.parts, cols = im.cols;
    const int tile0 = im.tile;
    if (cols == 0) continue;
    // this wave's block and its place among the block's waves (neighbours, on SIMDs of their own, read the same page)
    const int wc_log = wc >> 1, wk_log = 3 - wc_log, wk = 1 << wk_log, bw = w & (wc - 1), phase = w >> wc_log;  // (wc: 1, 2 or 4)
    const int block = im.block0 + bw;
    const int width = im.width, cols_end = min(block * width + width, cols);
    const bool idle = block * width >= cols;

    // this lane's column
    const int c = block * width + j, cc = min(c, cols_end - 1);
    const int ei = cc / per_entry, ci = cc - ei * per_entry, ti = ci / grp, row = (e0 + ei) * a.tokens + ti;
    const int h = hk * grp + ci - ti * grp;
    const Ent mine = a.ent[e0 + ei];
    const int last = mine.pos + ti;  // its last visible position
    const bool valid = c < cols_end && mine.seq >= 0;
    uint4 qf[NC];
    {
      const bf16_t* q = a.q_stride < 0 ? a.q + ((size_t)(row >> 5) * a.n_q_heads + h) * (size_t)NC * 512 + (size_t)(((row & 31) + 32 * g) << 3)
                                       : a.q + (size_t)row * a.q_stride + (size_t)h * HD + 8 * g;
      const int q_step = a.q_stride < 0 ? 512 : 16;
#pragma unroll
      for (int x = 0; x < NC; ++x) qf[x] = *(const uint4*)(q + (size_t)x * q_step);
    }

    // The steps of this wave: every wk-th of the part's shared pages, then of its own pages (which go on where the shared ones
    // stopped, so that the waves' numbers of steps differ by one at most).  A lane holds one step.
    auto of_block = [&](int x0, int x1, int x2, int x3) { return bw < 2 ? (bw == 0 ? x0 : x1) : (bw == 2 ? x2 : x3); };
    const int own_at = of_block(im.own_at[0], im.own_at[1], im.own_at[2], im.own_at[3]);
    const int own_n = idle ? 0 : of_block(im.own_n[0], im.own_n[1], im.own_n[2], im.own_n[3]);
    const int s0 = im.s0, s1 = im.s1;
    const int sh0 = s0 + phase, ow0 = (phase - (s1 - s0)) & (wk - 1);
    const int n_shared = idle || sh0 >= s1 ? 0 : (s1 - sh0 + wk - 1) >> wk_log;
    const int n_steps = n_shared + (ow0 >= own_n ? 0 : (own_n - ow0 + wk - 1) >> wk_log);
    int st_page = 0, st_what = 0;  // page | valid positions << 24, tile | entry << 16 (an own page's)
    auto load_steps = [&](int first) {
      const int i = first + lane;
      st_what = 0;
      if (i < n_shared) {
        st_page = p.table[(size_t)lead * p.max_pages + sh0 + i * wk];
        if ((unsigned)st_page >= (unsigned)p.n_pages) {  // (the table is the caller's)
          st_page = 0;
          report(p, PAGES_BAD_ENTRY);
        }
      } else if (i < n_steps) {
        const Own x = a.own[own_at + ow0 + (i - n_shared) * wk];
        st_page = (int)x.page;
        st_what = (int)x.what;
      }
    };

    const bf16_t* kv = p.data + ((size_t)a.layer * 2 * p.n_kv_heads + hk) * tile + (size_t)lane * 8;
    const size_t v_off = (size_t)p.n_kv_heads * tile;
    uint4 kf[NC];
    auto tile_of = [&](int i) { return kv + (size_t)(__builtin_amdgcn_readlane(st_page, i) & 0xffffff) * page; };
    auto load_k = [&](const bf16_t* t) {
#pragma unroll
      for (int x = 0; x < NC; ++x) kf[x] = *(const uint4*)(t + x * 512);
    };
    f32x16 o[NI];
#pragma unroll
    for (int ib = 0; ib < NI; ++ib)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[ib][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    // Scores (minus infinity: not seen) -> the weights as the second product's operand, and the sums so far in their units.
    // (The weights are rounded to the type of the cache, half a step each: it is what the matrix core takes at its full rate, and
    // V has no more bits.  Their sum is that of the weights in fp32.)
    // Register 4*q4 + e of a lane is key 8*q4 + 4*g + e of the tile.  The reference point of a column's exponentials follows its
    // maximum only when that has grown by more than 8 (weights stay below 256, or 2^-24): then the rescaling of the sums is rare.  (The
    // decision is the column's own: its result does not depend on its neighbours.)
    auto weigh = [&](f32x16& s, uint4(&pb)[2]) {
      float tmax = -INFINITY;
#pragma unroll
      for (int x = 0; x < 16; ++x) tmax = fmaxf(tmax, s[x]);
      tmax = fmaf(fmaxf(tmax, __shfl_xor(tmax, 32)), a.scale_log2e, kAbove<F16>);  // (m is in units of log2)
      float alpha = 1.f;
      if (tmax > m + 8.f) {
        alpha = __builtin_amdgcn_exp2f(m - tmax);  // (the first time 2^-inf = 0)
        m = tmax;
      }
      const float m_use = m == -INFINITY ? 0.f : m;
      float psum = 0.f;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2e, -m_use));
        psum += s[x];
      }
      l = fmaf(l, alpha, psum);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        pb[t].x = pack2<F16>(s[8 * t + 0], s[8 * t + 1]);
        pb[t].y = pack2<F16>(s[8 * t + 2], s[8 * t + 3]);
        pb[t].z = pack2<F16>(s[8 * t + 4], s[8 * t + 5]);
        pb[t].w = pack2<F16>(s[8 * t + 6], s[8 * t + 7]);
      }
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int ib = 0; ib < NI; ++ib)
#pragma unroll
          for (int x = 0; x < 16; ++x) o[ib][x] *= alpha;
      }
    };

    // Two blocks side by side read the same pages, each page by two waves: those keep step (by a barrier that orders no memory, once
    // per shared step that every wave has), so that the second finds the page in this CU's L1.  48 candidates over 32801 positions
    // 112 us, and 118 without, 2 x 40 over 9000 79 and 83, short lists equal.  With heads of 64 the pages of all waves fit into the L1 anyway
    // (6 groups of 1 to 3 x 6 tokens over 18532 positions, 4 heads: 26.4 without, 28.0 with), and with four blocks the waves
    // lose by it (grouped queries, 24 x 17009 positions: 32.9 and 37.0).
    const int together = HD == 128 && wc == 2 && (im.block0 + 1) * width < cols ? (s1 - s0) >> wk_log : 0;
    bool odd = false;
    // Once as a rule.  Where a column comes out infinite or NaN once more, from the beginning and with care: V of a position may
    // hold that, columns that do not see the position have weight 0 there, and 0 x NaN is not 0.
    for (int care = 0; care < 2; ++care) {
      if (care) {
#pragma unroll
        for (int ib = 0; ib < NI; ++ib)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[ib][i] = 0.f;
        m = -INFINITY;
        l = 0.f;
      }
      // 64 steps at a time, and no branch around a load inside (the compiler would wait for all loads behind it): the last step
      // asks for a few words that are never used.  (Its own keys again instead: what a CU fetches is what bounds a list of few steps.)
      for (int first = 0; first < n_steps; first += 64) {
        load_steps(first);
        const bf16_t* now = tile_of(0);
        load_k(now);
        const int n64 = min(n_steps - first, 64);
        for (int i = 0; i < n64; ++i) {
          if (!care && first + i < together) __builtin_amdgcn_s_barrier();
          const bool own = first + i >= n_shared;
          const int what = __builtin_amdgcn_readlane(st_what, i), kt = what & 0xffff;
          const int held = __builtin_amdgcn_readlane(st_page, i) >> 24;  // positions of an own page that hold a token
          uint4 vf[NI * 2];
#pragma unroll
          for (int t = 0; t < NI * 2; ++t) vf[t] = *(const uint4*)(now + v_off + t * 512);
          __builtin_amdgcn_sched_barrier(0);
          f32x16 s;
#pragma unroll
          for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
          for (int x = 0; x < NC; ++x) s = mfma32<F16>(kf[x], qf[x], s);
          __builtin_amdgcn_sched_barrier(0);
          now = i + 1 < n64 ? tile_of(min(i + 1, n64 - 1)) : p.data;
          load_k(now);
          __builtin_amdgcn_sched_barrier(0);
          if (own) {
            const int see = ei == what >> 16 ? last - 32 * kt - 4 * g : -1;
#pragma unroll
            for (int x = 0; x < 16; ++x) s[x] = 8 * (x >> 2) + (x & 3) <= see ? s[x] : -INFINITY;
          }
          uint4 pb[2];
          weigh(s, pb);
          if (own && (care || held < kPage)) {
            // V of positions that hold no token may be anything
#pragma unroll
            for (int t = 0; t < NI * 2; ++t) {
              uint32_t* x = (uint32_t*)&vf[t];
#pragma unroll
              for (int d = 0; d < 4; ++d) {
                const int kp = 16 * (t & 1) + 8 * (d >> 1) + 4 * g + 2 * (d & 1);
                const uint32_t far = far_values<F16>(x[d], care, care);
                const uint32_t seen = kp + 1 < held ? ~0u : kp < held ? 0xffffu : 0u;
                odd |= (far & seen) != 0;
                x[d] &= seen & ~far;
              }
            }
          }
#pragma unroll
          for (int ib = 0; ib < NI; ++ib)
#pragma unroll
            for (int t = 0; t < 2; ++t) o[ib] = mfma32<F16>(vf[ib * 2 + t], pb[t], o[ib]);
        }
      }
      if (care) break;
      float worst = 0.f;  // (0 x infinity and 0 x NaN are NaN, and stay it)
#pragma unroll
      for (int ib = 0; ib < NI; ++ib)
#pragma unroll
        for (int x = 0; x < 16; ++x) worst = fmaf(o[ib][x], 0.f, worst);
      if (!__any(worst != 0.f)) break;
    }
    l += __shfl_xor(l, 32);
    if (__builtin_expect(__any(odd), 0)) {
      // key by key, added where it is seen
      for (int i = n_shared; i < n_steps; ++i) {
        const int at64 = (i - n_shared) & 63;
        if (at64 == 0) load_steps(i);
        const int what = __builtin_amdgcn_readlane(st_what, at64), kt = what & 0xffff, held = __builtin_amdgcn_readlane(st_page, at64) >> 24;
        const int see = ei == what >> 16 ? last - 32 * kt : -1;  // this column's last key of the tile
        const bf16_t* at = tile_of(at64);
        load_k(at);
        f32x16 s;
#pragma unroll
        for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
        for (int x = 0; x < NC; ++x) s = mfma32<F16>(kf[x], qf[x], s);
#pragma unroll
        for (int x = 0; x < 16; ++x)
          s[x] = 8 * (x >> 2) + 4 * g + (x & 3) <= see ? __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2e, m == -INFINITY ? 0.f : -m)) : 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint4 pb = {pack2<F16>(s[8 * t], s[8 * t + 1]), pack2<F16>(s[8 * t + 2], s[8 * t + 3]),
                            pack2<F16>(s[8 * t + 4], s[8 * t + 5]), pack2<F16>(s[8 * t + 6], s[8 * t + 7])};
#pragma unroll
          for (int ib = 0; ib < NI; ++ib) {
            const uint4 v = *(const uint4*)(at + v_off + (ib * 2 + t) * 512);
            const uint32_t* x = (const uint32_t*)&v;
            for (int k = 0; k < min(held - 16 * t, 16); ++k) {
              const bool here = g == (k >> 2 & 1);
              uint4 only;
              uint32_t* y = (uint32_t*)&only;
#pragma unroll
              for (int d = 0; d < 4; ++d)
                y[d] = here && d == 2 * (k >> 3) + (k >> 1 & 1) ? x[d] & far_values<F16>(x[d], !(k & 1), k & 1) : 0u;
              f32x16 z;
#pragma unroll
              for (int r = 0; r < 16; ++r) z[r] = 0.f;
              z = mfma32<F16>(only, pb, z);
#pragma unroll
              for (int r = 0; r < 16; ++r) o[ib][r] += 16 * t + k <= see ? z[r] : 0.f;
            }
          }
        }
      }
    }

    // The waves of a block meet in LDS, a share of the sums each, in the order of the waves; then the result, or the part.
    auto meet = [&](auto count) {
      constexpr int R = decltype(count)::value;
      constexpr int WK = REGS / R;
      park[w][0][lane] = m;
      park[w][1][lane] = l;
#pragma unroll
      for (int ib = 0; ib < NI; ++ib)
#pragma unroll
        for (int i = 0; i < 16; ++i) park[w][2 + ib * 16 + i][lane] = o[ib][i];
      __syncthreads();
      const int r0 = phase * R;
      float M = -INFINITY, L = 0.f, x[R];
#pragma unroll
      for (int y = 0; y < WK; ++y) M = fmaxf(M, park[bw + y * wc][0][lane]);
      const float m_use = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = 0.f;
#pragma unroll
      for (int y = 0; y < WK; ++y) {
        const float f = __builtin_amdgcn_exp2f(park[bw + y * wc][0][lane] - m_use);
        L = fmaf(f, park[bw + y * wc][1][lane], L);
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = fmaf(f, park[bw + y * wc][2 + r0 + r][lane], x[r]);
      }
      if (!idle) {
        if (parts > 1) {
          const size_t at = (size_t)tile0 + bw * parts + part;
#pragma unroll
          for (int r = 0; r < R; r += 4)
            a.o[(at * (REGS / 4) + (r0 + r) / 4) * 64 + lane] = make_float4(x[r], x[r + 1], x[r + 2], x[r + 3]);
          if (r0 == 0) a.ml[at * 64 + lane] = make_float2(M, L);
        } else if (c < cols_end) {
          averages<F16>(x, 1.f / L);
#pragma unroll
          for (int r = 0; r < R; r += 4) store_out<HD, F16>(a, row, feature_of<HD>(h, (r0 + r) / 4, g), x + r, valid);
        }
      }
      __syncthreads();  // (the next item parks here)
    };
    if (wc == 1) meet(std::integral_constant<int, REGS / 8>{});
    else if (wc == 2) meet(std::integral_constant<int, REGS / 4>{});
    else meet(std::integral_constant<int, REGS / 2>{});
  }
}

// The same for short lists of blocks of up to 16 columns, no parts: products of 16 x 16 x 32, half the registers per column
// block, and so two tiles at a time per wave.  A row of K is the key that the second product wants there: the row m = 4 * q + e of
// product rb is key 16 * (q >> 1) + 8 * rb + 4 * (q & 1) + e, so that the 8 scores of a lane are, in order, the 8 weights that it owes
// as the second operand, for the 16 bytes of V that lie together in the page.  Bound by latency, then by what a CU fetches: one
// token of 8 candidates over 288 positions, 32 heads of 128, 6.8 us; 2 groups of up to 8 x 8 tokens over 601 (36 MB) 11.6.
template <int HD, bool F16>
__global__ __launch_bounds__(64 * kWaves) void attend_few_kernel(AttendArgs a) {
  constexpr int NB = HD / 32, NF = HD / 16, U = 2;
  __shared__ float park[kWaves][2 + 4 * NF][64];
  const PoolView& p = a.p;
  read_args(a.head, a.item, a.ent, a.q, a.q_stride, a.out, a.kc_out, a.layer, a.tokens, a.n_q_heads, a.scale_log2e, p.data, p.table,
            p.n_pages, p.max_pages, p.n_layers, p.n_kv_heads, a.own);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, q4 = lane >> 4;
  const int grp = a.n_q_heads / p.n_kv_heads, per_entry = a.tokens * grp;
  // (asked for together with what says whether there is such an item)
  Item im = load_item(a.item + blockIdx.x);
  const int n_items = ld_scalar(a.head), differ = differs(a.head, a.made);
  read_args(n_items, differ, im.e0, im.seq, im.head, im.block0, im.cols, im.s0, im.s1, im.width, im.own_at[0], im.own_n[0]);
  if (differ) {
    if (blockIdx.x == 0 && tid == 0) report(p, PAGES_BAD_ENTRY);
    return;
  }
  const size_t tile = (size_t)kPage * HD, page = (size_t)p.n_layers * 2 * p.n_kv_heads * tile;
  const int half = (q4 >> 1) * 512 + (q4 & 1) * 256;  // where 8 features, or 8 positions, of a lane lie
  for (int it = blockIdx.x; it < n_items; it += gridDim.x) {
    if (it != (int)blockIdx.x) im = load_item(a.item + it);
    const int e0 = im.e0, lead = im.seq, hk = im.head, cols = im.cols, width = im.width;
    if (cols == 0) continue;
    const int c0 = im.block0 * width, cols_end = min(c0 + width, cols);

    // this lane's column
    const int c = c0 + j, cc = min(c, cols_end - 1);
    const int ei = cc / per_entry, ci = cc - ei * per_entry, ti = ci / grp, row = (e0 + ei) * a.tokens + ti;
    const int h = hk * grp + ci - ti * grp;
    const Ent mine = a.ent[e0 + ei];
    const int last = mine.pos + ti;  // its last visible position
    const bool valid = c < cols_end && mine.seq >= 0;
    uint4 qf[NB];
    {
      const bf16_t* q = a.q_stride < 0 ? a.q + ((size_t)(row >> 5) * a.n_q_heads + h) * (size_t)(HD / 16) * 512 + (size_t)((row & 31) << 3) + half
                                       : a.q + (size_t)row * a.q_stride + (size_t)h * HD + 8 * q4;
      const int q_step = a.q_stride < 0 ? 1024 : 32;
#pragma unroll
      for (int x = 0; x < NB; ++x) qf[x] = *(const uint4*)(q + (size_t)x * q_step);
    }

    // The steps of this wave: every eighth of the shared pages, then of the block's own.  A lane holds one step.
    const int own_at = im.own_at[0], own_n = im.own_n[0], s0 = im.s0, s1 = im.s1;
    const int sh0 = s0 + w, ow0 = (w - (s1 - s0)) & (kWaves - 1);
    const int n_shared = sh0 >= s1 ? 0 : (s1 - sh0 + kWaves - 1) / kWaves;
    const int n_steps = n_shared + (ow0 >= own_n ? 0 : (own_n - ow0 + kWaves - 1) / kWaves);
    int st_page = 0, st_what = 0;  // page | valid positions << 24, tile | entry << 16 (an own page's)
    auto load_steps = [&](int first) {
      const int i = first + lane;
      st_what = 0;
      if (i < n_shared) {
        st_page = p.table[(size_t)lead * p.max_pages + sh0 + i * kWaves];
        if ((unsigned)st_page >= (unsigned)p.n_pages) {  // (the table is the caller's)
          st_page = 0;
          report(p, PAGES_BAD_ENTRY);
        }
      } else if (i < n_steps) {
        const Own x = a.own[own_at + ow0 + (i - n_shared) * kWaves];
        st_page = (int)x.page;
        st_what = (int)x.what;
      }
    };

    const bf16_t* kv = p.data + ((size_t)a.layer * 2 * p.n_kv_heads + hk) * tile + half;
    const size_t v_off = (size_t)p.n_kv_heads * tile + 8 * j;
    const int k_off = 8 * (16 * (j >> 3) + (j & 7));
    auto tile_of = [&](int i) { return kv + (size_t)(__builtin_amdgcn_readlane(st_page, i) & 0xffffff) * page; };
    f32x4v o[NF];
    float m, l;
    auto clear = [&] {
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[f] = f32x4v{0.f, 0.f, 0.f, 0.f};
    };
    clear();
    auto load_k = [&](uint4(&kf)[2 * NB], const bf16_t* t) {
#pragma unroll
      for (int x = 0; x < 2 * NB; ++x) kf[x] = *(const uint4*)(t + k_off + (x >> 1) * 1024 + (x & 1) * 64);
    };
    auto v_at = [&](const bf16_t* t, int f) { return t + v_off + (f >> 1) * 1024 + (f & 1) * 128; };
    auto scores = [&](const uint4(&kf)[2 * NB], float(&s)[8]) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        f32x4v y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NB; ++x) y = mfma16<F16>(kf[2 * x + rb], qf[x], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * rb + e] = y[e];
      }
    };
    // score 4 * rb + e is key first_key + 8 * rb + e of the tile
    const int first_key = 16 * (q4 >> 1) + 4 * (q4 & 1);
    auto weights = [&](const float(&s)[8]) {
      return make_uint4(pack2<F16>(s[0], s[1]), pack2<F16>(s[2], s[3]), pack2<F16>(s[4], s[5]), pack2<F16>(s[6], s[7]));
    };
    bool odd = false;
    for (int care = 0; care < 2; ++care) {  // (as above: twice only where a column comes out infinite or NaN)
      if (care) clear();
      for (int first = 0; first < n_steps; first += 64) {
        load_steps(first);
        const int n64 = min(n_steps - first, 64);
        for (int i = 0; i < n64; i += U) {
          uint4 kf[U][2 * NB], vf[U][NF];
#pragma unroll
          for (int u = 0; u < U; ++u) load_k(kf[u], i + u < n64 ? tile_of(min(i + u, n64 - 1)) : kv);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const bf16_t* t = i + u < n64 ? tile_of(min(i + u, n64 - 1)) : kv;
#pragma unroll
            for (int f = 0; f < NF; ++f) vf[u][f] = *(const uint4*)v_at(t, f);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (i + u >= n64) break;
            const bool own = first + i + u >= n_shared;
            const int what = __builtin_amdgcn_readlane(st_what, min(i + u, 63)), kt = what & 0xffff;
            const int held = __builtin_amdgcn_readlane(st_page, min(i + u, 63)) >> 24;  // positions of an own page that hold a token
            float s[8];
            scores(kf[u], s);
            if (own) {
              const int see = ei == what >> 16 ? last - 32 * kt - first_key : -1;
#pragma unroll
              for (int x = 0; x < 8; ++x) s[x] = 8 * (x >> 2) + (x & 3) <= see ? s[x] : -INFINITY;
            }
            // (the reference point as above)
            float tmax = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
            tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
            tmax = fmaf(fmaxf(tmax, __shfl_xor(tmax, 32)), a.scale_log2e, kAbove<F16>);
            float alpha = 1.f;
            if (tmax > m + 8.f) {
              alpha = __builtin_amdgcn_exp2f(m - tmax);
              m = tmax;
            }
            const float m_use = m == -INFINITY ? 0.f : m;
            float psum = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2e, -m_use));
              psum += s[x];
            }
            l = fmaf(l, alpha, psum);
            const uint4 pb = weights(s);
            if (__any(alpha != 1.f)) {
#pragma unroll
              for (int f = 0; f < NF; ++f) o[f] *= alpha;
            }
            if (own && (care || held < kPage)) {
              // V of positions that hold no token may be anything
#pragma unroll
              for (int f = 0; f < NF; ++f) {
                uint32_t* x = (uint32_t*)&vf[u][f];
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                  const int kp = first_key + 8 * (d >> 1) + 2 * (d & 1);
                  const uint32_t far = far_values<F16>(x[d], care, care);
                  const uint32_t seen = kp + 1 < held ? ~0u : kp < held ? 0xffffu : 0u;
                  odd |= (far & seen) != 0;
                  x[d] &= seen & ~far;
                }
              }
            }
#pragma unroll
            for (int f = 0; f < NF; ++f) o[f] = mfma16<F16>(vf[u][f], pb, o[f]);
          }
        }
      }
      if (care) break;
      float worst = 0.f;  // (0 x infinity and 0 x NaN are NaN, and stay it)
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) worst = fmaf(o[f][e], 0.f, worst);
      if (!__any(worst != 0.f)) break;
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (__builtin_expect(__any(odd), 0)) {
      // key by key, added where it is seen
      for (int i = n_shared; i < n_steps; ++i) {
        const int at64 = (i - n_shared) & 63;
        if (at64 == 0) load_steps(i);
        const int what = __builtin_amdgcn_readlane(st_what, at64), kt = what & 0xffff, held = __builtin_amdgcn_readlane(st_page, at64) >> 24;
        const int see = ei == what >> 16 ? last - 32 * kt : -1;  // this column's last key of the tile
        const bf16_t* at = tile_of(at64);
        uint4 kf[2 * NB];
        load_k(kf, at);
        float s[8];
        scores(kf, s);
#pragma unroll
        for (int x = 0; x < 8; ++x)
          s[x] = first_key + 8 * (x >> 2) + (x & 3) <= see ? __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2e, m == -INFINITY ? 0.f : -m)) : 0.f;
        const uint4 pb = weights(s);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const uint4 v = *(const uint4*)v_at(at, f);
          const uint32_t* x = (const uint32_t*)&v;
          for (int k = 0; k < held; ++k) {
            const bool here = q4 == 2 * (k >> 4) + (k >> 2 & 1);
            uint4 only;
            uint32_t* y = (uint32_t*)&only;
#pragma unroll
            for (int d = 0; d < 4; ++d)
              y[d] = here && d == 2 * (k >> 3 & 1) + (k >> 1 & 1) ? x[d] & far_values<F16>(x[d], !(k & 1), k & 1) : 0u;
            const f32x4v z = mfma16<F16>(only, pb, f32x4v{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) o[f][e] += k <= see ? z[e] : 0.f;
          }
        }
      }
    }

    // The waves meet in LDS; four sums of a lane each, in the order of the waves.
    park[w][0][lane] = m;
    park[w][1][lane] = l;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e) park[w][2 + 4 * f + e][lane] = o[f][e];
    __syncthreads();
    if (w < NF && c < cols_end) {
      float M = -INFINITY, L = 0.f;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < kWaves; ++y) M = fmaxf(M, park[y][0][lane]);
      const float m_use = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int y = 0; y < kWaves; ++y) {
        const float f = __builtin_amdgcn_exp2f(park[y][0][lane] - m_use);
        L = fmaf(f, park[y][1][lane], L);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(f, park[y][2 + 4 * w + e][lane], x[e]);
      }
      averages<F16>(x, 1.f / L);
      store_out<HD, F16>(a, row, h * HD + 16 * w + 4 * q4, x, valid);
    }
    __syncthreads();  // (the next item parks here)
  }
}

// Joins the parts.  The items of a (head, column blocks) deal its sums among themselves: a wave takes four sums of a block's
// lanes, over all parts.
template <int HD, bool F16>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int QUADS = HD / 8;
  const PoolView& p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, g = lane >> 5;
  const int grp = a.n_q_heads / p.n_kv_heads, per_entry = a.tokens * grp;
  if (differs(a.head, a.made)) return;
  const int n_items = ld_scalar(a.head);
  for (int it = blockIdx.x; it < n_items; it += gridDim.x) {
    const Item* im = a.item + it;
    const int parts = ld_scalar(&im->parts), part = ld_scalar(&im->part), wc = ld_scalar(&im->waves_c), cols = ld_scalar(&im->cols);
    const int e0 = ld_scalar(&im->e0), hk = ld_scalar(&im->head), block0 = ld_scalar(&im->block0), tile0 = ld_scalar(&im->tile);
    const int width = ld_scalar(&im->width);
    if (parts < 2) continue;
    for (int u = part + w * parts; u < wc * QUADS; u += 4 * parts) {
      const int bw = u / QUADS, quad = u - bw * QUADS, block = block0 + bw;
      if (block * width >= cols) continue;
      const size_t at = (size_t)tile0 + bw * parts;
      float M = -INFINITY, L = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s0 = 0; s0 < parts; s0 += 8) {  // eight parts in flight
        float2 y[8];
        float4 z[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          const size_t t = at + min(s0 + s, parts - 1);
          y[s] = a.ml[t * 64 + lane];
          z[s] = a.o[(t * QUADS + quad) * 64 + lane];
        }
        float top = M;
#pragma unroll
        for (int s = 0; s < 8; ++s) top = fmaxf(top, y[s].x);
        const float m_use = top == -INFINITY ? 0.f : top, back = __builtin_amdgcn_exp2f(M - m_use);
        M = top;
        L *= back;
        x.x *= back; x.y *= back; x.z *= back; x.w *= back;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          const float f = s0 + s < parts ? __builtin_amdgcn_exp2f(y[s].x - m_use) : 0.f;
          if (s0 + s < parts) {
            L = fmaf(f, y[s].y, L);
            x.x = fmaf(f, z[s].x, x.x); x.y = fmaf(f, z[s].y, x.y); x.z = fmaf(f, z[s].z, x.z); x.w = fmaf(f, z[s].w, x.w);
          }
        }
      }
      const int c = block * width + j;
      if (j >= width || c >= cols) continue;
      const int ei = c / per_entry, ci = c - ei * per_entry, ti = ci / grp;
      float y[4] = {x.x, x.y, x.z, x.w};
      averages<F16>(y, 1.f / L);
      store_out<HD, F16>(a, (e0 + ei) * a.tokens + ti, feature_of<HD>(hk * grp + ci - ti * grp, quad, g), y, a.ent[e0 + ei].seq >= 0);
    }
  }
}

bool sizes_ok(const vlac_pages* p, int n, int tokens, int n_q_heads) {
  return n >= 0 && n <= VLAC_PAGES_MAX_LIST && tokens >= 1 && tokens <= 65536 && (long long)n * tokens <= 1 << 20 && n_q_heads >= 1 &&
         n_q_heads <= 1024 && n_q_heads >= p->n_kv_heads && n_q_heads % p->n_kv_heads == 0;
}

int check_attend(const vlac_pages* pages, int n, int tokens, int n_q_heads, const void* ws, size_t ws_bytes) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  if (!sizes_ok(pages, n, tokens, n_q_heads)) return n_q_heads >= 1 && n_q_heads % pages->n_kv_heads ? VLAC_E_SHAPE : VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!ws) return VLAC_E_NULL;
  if ((uintptr_t)ws % 16) return VLAC_E_SHAPE;
  const size_t need = attend_workspace(pool_view(pages), n, tokens, n_q_heads);
  return need == 0 || ws_bytes < need ? VLAC_E_RANGE : VLAC_OK;
}

}  // namespace

size_t attend_workspace(const PoolView& p, int n, int tokens, int n_q_heads) {
  return layout_of(p, n > 0 ? n : 1, tokens, n_q_heads).total;
}

void launch_attend_plan(const PoolView& p, const int* seqs, const int* pos, int add, int n, int tokens, int n_q_heads,
                        const int* group, void* ws, hipStream_t st) {
  const Layout l = layout_of(p, n, tokens, n_q_heads);
  char* b = (char*)ws;
  const PlanArgs a = {p, made_for(p, n, tokens, n_q_heads), seqs, pos, group, add, n, tokens, n_q_heads, l.part_tiles,
                      (int)l.max_items, l.few ? 16 : 32, (int*)b, (Ent*)(b + l.ent), (Own*)(b + l.own), (Item*)(b + l.item)};
  // (4 waves or 16: one token of 2 candidates 7.3 and 8.2 us, 16 candidates x 56 tokens over 1057 positions 8.0 and 8.6; 48
  // candidates with tables of 1027 pages 40 and 20 when both were tried.  More entries than 128 are a second round for 4 waves.)
  if (n <= 128 && (long long)n * p.max_pages <= 4096)
    hipLaunchKernelGGL((attend_plan_kernel<256, 128>), dim3(1), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((attend_plan_kernel<1024, VLAC_PAGES_MAX_LIST>), dim3(1), dim3(1024), 0, st, a);
}

void launch_attend(const PoolView& p, bool f16, int layer, int n, int tokens, int n_q_heads, const AttendIo& io, void* ws,
                   hipStream_t st) {
  const Layout l = layout_of(p, n, tokens, n_q_heads);
  char* b = (char*)ws;
  const AttendArgs a = {p, made_for(p, n, tokens, n_q_heads), (const int*)b, (const Ent*)(b + l.ent), (const Own*)(b + l.own),
                        (const Item*)(b + l.item),
                        (float2*)(b + l.ml), (float4*)(b + l.o), io.q, io.q_stride, io.out, io.kc_out, layer, n, tokens,
                        n_q_heads, 1.4426950408889634f / sqrtf((float)p.head_dim)};
  const dim3 grid((unsigned)std::min<size_t>(l.max_items, kCus)), join((unsigned)std::min<size_t>(l.max_items, 4 * kCus));
#define VLAC_ATTEND(HD_, F16_)                                                                        \
  {                                                                                                   \
    if (l.few) hipLaunchKernelGGL((attend_few_kernel<HD_, F16_>), grid, dim3(64 * kWaves), 0, st, a); \
    else hipLaunchKernelGGL((attend_kernel<HD_, F16_>), grid, dim3(64 * kWaves), 0, st, a);           \
    if (l.parts) hipLaunchKernelGGL((attend_join_kernel<HD_, F16_>), join, dim3(256), 0, st, a);      \
  }
  if (p.head_dim == 128) {
    if (f16) VLAC_ATTEND(128, true) else VLAC_ATTEND(128, false)
  } else {
    if (f16) VLAC_ATTEND(64, true) else VLAC_ATTEND(64, false)
  }
#undef VLAC_ATTEND
}

extern "C" {

size_t vlac_attend_workspace_bytes(const vlac_pages* pages, int n, int tokens, int n_q_heads) {
  if (check_pages(pages, false) != VLAC_OK || !sizes_ok(pages, n, tokens, n_q_heads)) return 0;
  return attend_workspace(pool_view(pages), n, tokens, n_q_heads);
}

int vlac_attend_plan(const vlac_pages* pages, const int32_t* seqs, const int32_t* pos, int n, int tokens, int n_q_heads,
                     const int32_t* group, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_attend(pages, n, tokens, n_q_heads, workspace, workspace_bytes);
  if (rc != VLAC_OK || n == 0) return rc;
  if (!seqs || !pos) return VLAC_E_NULL;
  launch_attend_plan(pool_view(pages), seqs, pos, 0, n, tokens, n_q_heads, group, workspace, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

int vlac_attend_shared(const vlac_pages* pages, int layer, int n, int tokens, int n_q_heads, const void* q, int64_t q_stride,
                       void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_attend(pages, n, tokens, n_q_heads, workspace, workspace_bytes);
  if (rc != VLAC_OK) return rc;
  if (layer < 0 || layer >= pages->n_layers) return VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!q || !out) return VLAC_E_NULL;
  if (q_stride < (int64_t)n_q_heads * pages->head_dim || q_stride % 8 || q_stride > 1 << 30 || (uintptr_t)q % 16 || (uintptr_t)out % 8)
    return VLAC_E_SHAPE;
  const AttendIo io = {(const bf16_t*)q, q_stride, (bf16_t*)out, 0};
  launch_attend(pool_view(pages), pages_f16(pages), layer, n, tokens, n_q_heads, io, workspace, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
