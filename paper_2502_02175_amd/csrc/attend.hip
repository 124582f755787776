// Attention of new tokens over pages, for sequences that share prefixes:
//   out[row] = sum_p exp(s_p - M) v_p / sum_p exp(s_p - M),  s_p = q . k_p / sqrt(head_dim), p <= position of the row.
// The keys of a row are cut into segments: the pages that its group has in common at the front (all of them wholly
// before every query of the group: no mask), and its own behind them.  A segment is cut further over the keys, and
// every part leaves (max, sum, output) of its columns in fp32; a second kernel joins a row's parts:
//   M = max m_i, out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i   (scores in units of log2).
// What is gained: a shared page is read once for all columns of its group (candidates x tokens x query heads of the kv
// head), 32 of them to a matrix product, where one pass per sequence reads it once for each.
//
// A column is a query (entry, token, head of the group); 32 columns are a column block.  S^T = K Q^T and O^T += V^T P^T as in
// the attention over the stream cache: a page's tiles are the operands as they lie, a lane owns a column.
// A workgroup of 4 waves takes a work item: of a segment with one column block the waves take every
// 4th key tile, with two every 2nd, and with more a column block each; or (short segments of one block, the usual
// decode step) four such segments, one per wave.
#include <algorithm>

#include "pages.h"

namespace {

constexpr int kPlan = 1024;          // threads of the planning workgroup
constexpr int kMaxSplit = 64;        // parts of a segment (a lane each when they are joined)
constexpr int kSlots = 512;          // workgroups that the chip holds at a time (two per CU)
constexpr int kWaveTiles = 4;        // own segments of at most this many pages are a wave's work

// What a row has to know, per entry
struct Ent {
  int seq, pos;          // row of the table (-1: the entry is ignored), position of its first query
  int shared;            // pages that its group reads together
  int sh_parts, sh_base; // parts of that segment, first partial column of head 0, part 0
  int c0, cols;          // first column of the entry in its group's segment, columns of the segment
  int own_parts, own_base;
  int group;             // index of its group (for the planning kernel)
  int pad[2];
};
// A work item.  what: 0 shared, 1 own, 2 own segments of four (entry, kv head) pairs
struct Item {
  int what, e0, seq, head, block, t0, t1, base, cols, waves_c, pad[2];
};
static_assert(sizeof(Ent) == 48 && sizeof(Item) == 48, "read as three 16-byte words");

struct Layout {
  size_t ent, item, ml, o, total;
  size_t max_items, max_cols;
  int split_shared, split_own;  // most parts of a segment
};
// Parts are bounded so that what they leave is bounded: as many as give every slot of the chip an item twice over where
// the batch has the fewest column blocks that its rows can make
inline Layout layout_of(int n, int tokens, int n_q_heads, int n_kv_heads, int head_dim) {
  Layout l;
  const size_t rows = (size_t)n * tokens * n_q_heads, per_kv = rows / n_kv_heads;
  const size_t own_cols = (size_t)tokens * (n_q_heads / n_kv_heads);
  const size_t blocks = (per_kv + 31) / 32 * n_kv_heads, own_blocks = (own_cols + 31) / 32 * n * n_kv_heads;
  auto split = [](size_t b) { return (int)std::max<size_t>(1, std::min<size_t>(kMaxSplit, (2 * kSlots + b - 1) / b)); };
  l.split_shared = split(blocks);
  l.split_own = split(own_blocks);
  l.max_cols = rows * (l.split_shared + l.split_own);
  // (a group of few columns is a block of its own: at most n groups)
  l.max_items = (blocks + (size_t)n * n_kv_heads) * l.split_shared + own_blocks * l.split_own + n_kv_heads;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  l.ent = 256;
  l.item = l.ent + up(sizeof(Ent) * n);
  l.ml = l.item + up(sizeof(Item) * l.max_items);
  l.o = l.ml + up(8 * l.max_cols);
  l.total = l.o + up(4 * l.max_cols * head_dim);
  return l;
}

struct PlanArgs {
  PoolView p;
  const int *seqs, *pos, *group;
  int add, n, tokens, n_q_heads, split_shared, split_own, max_items;
  int* head;  // [0] number of items
  Ent* ent;
  Item* item;
};

// Sums of two numbers over the threads before this one, and over all
struct Two { int a, b; };
__device__ inline Two scan_before(Two x, Two* sums, Two* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Two run = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int ya = __shfl_up(run.a, d), yb = __shfl_up(run.b, d);
    if (lane >= d) { run.a += ya; run.b += yb; }
  }
  if (lane == 63) sums[w] = run;
  __syncthreads();
  if (threadIdx.x == 0) {
    Two s = {0, 0};
    for (int i = 0; i < kPlan / 64; ++i) {
      const Two t = sums[i];
      sums[i] = s;
      s.a += t.a; s.b += t.b;
    }
    sums[kPlan / 64] = s;
  }
  __syncthreads();
  const Two before = {sums[w].a + run.a - x.a, sums[w].b + run.b - x.b};
  *total = sums[kPlan / 64];
  __syncthreads();
  return before;
}

// How the waves of a workgroup share a segment: column blocks side by side
__device__ inline int waves_over_columns(int blocks) { return blocks >= 3 ? 4 : blocks; }

struct Cut { int waves_c, chunks, parts; };

// One workgroup.  Groups and their common pages, then the cut, then the items.
__global__ __launch_bounds__(kPlan) void attend_plan_kernel(PlanArgs a) {
  __shared__ Two sums[kPlan / 64 + 1];
  constexpr int N = VLAC_PAGES_MAX_LIST;
  __shared__ int g_start[N + 1], g_lead[N], g_shared[N], g_item[N], g_base[N], o_item[N];
  __shared__ int s_own_most;
  __shared__ unsigned long long s_work[2];
  const PoolView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int hkv = p.n_kv_heads, per_entry = a.tokens * (a.n_q_heads / hkv);  // columns of an entry per kv head
  if (tid == 0) {
    s_own_most = 0;
    s_work[0] = s_work[1] = 0;
  }

  int n_groups = 0;
  for (int base = 0; base < a.n; base += kPlan) {
    const int i = base + tid;
    const bool start = i < a.n && (i == 0 || (a.group && a.group[i] != a.group[i - 1]));
    Two total;
    const Two before = scan_before({start ? 1 : 0, 0}, sums, &total);
    if (start) g_start[n_groups + before.a] = i;
    if (i < a.n) a.ent[i].group = n_groups + before.a + (start ? 1 : 0) - 1;
    n_groups += total.a;
  }
  for (int g = tid; g < n_groups; g += kPlan) {
    g_lead[g] = 0x7fffffff;
    g_shared[g] = 0x7fffffff;
  }
  if (tid == 0) g_start[n_groups] = a.n;
  __syncthreads();
  bool bad = false;
  for (int i = tid; i < a.n; i += kPlan) {
    const int s = a.seqs[i], p0 = a.pos[i];
    const int l = checked_len(p, s);
    const long long at = (long long)p0 + a.add;
    const bool fits = p0 >= 0 && l >= 0 && at + a.tokens <= l;
    bad |= p0 >= 0 && !fits;
    a.ent[i].seq = fits ? s : -1;
    a.ent[i].pos = fits ? (int)at : 0;
    if (fits) {
      const int g = a.ent[i].group;
      atomicMin(&g_lead[g], i);
      atomicMin(&g_shared[g], (int)(at / kPage));
    }
  }
  if (bad) report(p, PAGES_BAD_ENTRY);
  __syncthreads();
  // the common pages: every entry against its group's first, 512 pages in flight
  for (int i = w; i < a.n; i += kPlan / 64) {
    const int seq = a.ent[i].seq, g = a.ent[i].group;
    if (seq < 0) continue;
    const int lead = a.ent[g_lead[g]].seq;
    if (lead == seq) continue;
    const int* mine = p.table + (size_t)seq * p.max_pages;
    const int* other = p.table + (size_t)lead * p.max_pages;
    for (int j0 = 0; j0 < g_shared[g]; j0 += 512) {
      const int end = g_shared[g];
      int x[8], y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = j0 + 64 * e + lane;
        x[e] = j < end ? mine[j] : -1;
        y[e] = j < end ? other[j] : -1;
      }
      int differ = 0x7fffffff;
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (x[e] != y[e]) differ = j0 + 64 * e + lane;
      if (__any(differ != 0x7fffffff)) {
        if (differ != 0x7fffffff) atomicMin(&g_shared[g], differ);
        break;
      }
    }
  }
  __syncthreads();

  // work in steps of a wave: a key tile of a column block
  unsigned long long work = 0;
  for (int g = tid; g < n_groups; g += kPlan) {
    if (g_lead[g] == 0x7fffffff) g_shared[g] = 0;
    const int blocks = ((g_start[g + 1] - g_start[g]) * per_entry + 31) / 32;
    work += (unsigned long long)blocks * g_shared[g] * hkv;
  }
  atomicAdd(&s_work[0], work);
  __syncthreads();
  const int own_blocks = (per_entry + 31) / 32;
  work = 0;
  for (int i = tid; i < a.n; i += kPlan)
    if (a.ent[i].seq >= 0) {
      const int own = pages_of(a.ent[i].pos + a.tokens) - g_shared[a.ent[i].group];
      atomicMax(&s_own_most, own);
      work += (unsigned long long)own * own_blocks * hkv;
    }
  atomicAdd(&s_work[1], work);
  __syncthreads();
  const bool by_wave = own_blocks == 1 && s_own_most <= kWaveTiles;
  // steps of a wave per item: what fills the chip's slots, and no fewer than two, so that a part is worth its columns
  const int steps = (int)max(2ull, (s_work[0] + s_work[1] + 4ull * kSlots - 1) / (4ull * kSlots));
  auto cut = [&](int c, int tiles, int most) {  // c columns per kv head, `tiles` pages
    Cut x;
    const int blocks = (c + 31) / 32;
    x.waves_c = waves_over_columns(blocks);
    x.chunks = (blocks + x.waves_c - 1) / x.waves_c;
    const long long per_item = (long long)steps * (4 / x.waves_c);
    x.parts = (int)min((long long)most, (tiles + per_item - 1) / per_item);
    return x;
  };
  auto group_cols = [&](int g) { return (g_start[g + 1] - g_start[g]) * per_entry; };

  // first item and first partial column of every segment
  int items = 0, cols = 0;
  for (int base = 0; base < n_groups; base += kPlan) {
    const int g = base + tid;
    Two mine = {0, 0};
    if (g < n_groups) {
      const Cut x = cut(group_cols(g), g_shared[g], a.split_shared);
      mine = {hkv * x.chunks * x.parts, hkv * group_cols(g) * x.parts};
    }
    Two total;
    const Two before = scan_before(mine, sums, &total);
    if (g < n_groups) {
      g_item[g] = items + before.a;
      g_base[g] = cols + before.b;
    }
    items += total.a;
    cols += total.b;
  }
  const int shared_items = items;
  for (int base = 0; base < a.n; base += kPlan) {
    const int i = base + tid;
    Two mine = {0, 0};
    int parts = 0;
    if (i < a.n) {
      Ent& e = a.ent[i];
      const int g = e.group, c = group_cols(g);
      e.shared = g_shared[g];
      e.sh_parts = cut(c, g_shared[g], a.split_shared).parts;
      e.sh_base = g_base[g];
      e.c0 = (i - g_start[g]) * per_entry;
      e.cols = c;
      if (by_wave) {  // (entry, kv head) pairs in order, whose partial columns lie in the same order
        parts = e.seq >= 0;
        mine = {0, hkv * per_entry};
      } else if (e.seq >= 0) {
        const Cut x = cut(per_entry, pages_of(e.pos + a.tokens) - g_shared[g], a.split_own);
        parts = x.parts;
        mine = {hkv * x.chunks * parts, hkv * per_entry * parts};
      }
    }
    Two total;
    const Two before = scan_before(mine, sums, &total);
    if (i < a.n) {
      a.ent[i].own_parts = parts;
      a.ent[i].own_base = cols + before.b;
      o_item[i] = items + before.a;
    }
    items += total.a;
    cols += total.b;
  }
  if (by_wave) items += (a.n * hkv + 3) / 4;
  if (tid == 0) a.head[0] = min(items, a.max_items);
  __syncthreads();

  // the last of first[0 .. n) that is at most x (ascending; a segment without items begins where the next one does)
  auto segment_of = [](const int* first, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  for (int it = tid; it < min(items, a.max_items); it += kPlan) {
    Item im = {};
    if (it < shared_items) {
      const int g = segment_of(g_item, n_groups, it), c = group_cols(g), tiles = g_shared[g];
      const Cut x = cut(c, tiles, a.split_shared);
      const int r = it - g_item[g], hs = r / x.chunks, h = hs / x.parts, s = hs - h * x.parts;
      im.what = 0; im.e0 = g_start[g]; im.seq = a.ent[g_lead[g]].seq; im.head = h;
      im.block = (r - hs * x.chunks) * x.waves_c;
      im.t0 = (int)((long long)s * tiles / x.parts); im.t1 = (int)((long long)(s + 1) * tiles / x.parts);
      im.base = g_base[g] + hs * c; im.cols = c; im.waves_c = x.waves_c;
    } else if (by_wave) {
      im.what = 2; im.e0 = 4 * (it - shared_items); im.seq = a.n * hkv; im.cols = per_entry; im.waves_c = 1;
    } else {
      const int i = segment_of(o_item, a.n, it), own = pages_of(a.ent[i].pos + a.tokens) - a.ent[i].shared, from = a.ent[i].shared;
      const Cut x = cut(per_entry, own, a.split_own);
      const int r = it - o_item[i], hs = r / x.chunks, h = hs / x.parts, s = hs - h * x.parts;
      im.what = 1; im.e0 = i; im.seq = a.ent[i].seq; im.head = h;
      im.block = (r - hs * x.chunks) * x.waves_c;
      im.t0 = from + (int)((long long)s * own / x.parts); im.t1 = from + (int)((long long)(s + 1) * own / x.parts);
      im.base = a.ent[i].own_base + hs * per_entry; im.cols = per_entry; im.waves_c = x.waves_c;
    }
    a.item[it] = im;
  }
}

struct AttendArgs {
  PoolView p;
  const int* head;
  const Ent* ent;
  const Item* item;
  float2* ml;  // [columns] reference point of the exponentials (log2 units) and sum
  float* o;    // [columns][head_dim] unnormalised output
  const bf16_t* q;
  long long q_stride;
  bf16_t* out;
  int kc_out;
  int layer, n, tokens, n_q_heads;
  float scale_log2e;
};

template <bool F16>
__device__ inline uint32_t pack2(float lo, float hi) {
  // (no saturation as elsewhere: values are sums of cache values with weights of sum 1, and a NaN stays one)
  if constexpr (F16) {
    const f32x2v v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2v));
  } else {
    return f2bf2(lo, hi);
  }
}

// Masks of the two values of a word that are infinite or NaN, where asked for
template <bool F16>
__device__ inline uint32_t far_values(uint32_t x, bool lo, bool hi) {
  constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;
  return (lo && (x & kExp) == kExp ? 0xffffu : 0u) | (hi && (x >> 16 & kExp) == kExp ? 0xffff0000u : 0u);
}

template <int HD, bool F16>
__global__ __launch_bounds__(256, 2) void attend_kernel(AttendArgs a) {
  constexpr int NC = HD / 16, NI = HD / 32;
  __shared__ float park[4][2 + NI * 16][64];
  const PoolView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 31, g = lane >> 5;
  const int grp = a.n_q_heads / p.n_kv_heads, per_entry = a.tokens * grp;
  const int n_items = ld_scalar(a.head);
  const size_t tile = (size_t)kPage * HD, page = p.page();
  for (int it = blockIdx.x; it < n_items; it += gridDim.x) {
    const Item* im = a.item + it;
    const int what = ld_scalar(&im->what);
    int e0 = ld_scalar(&im->e0), seq = ld_scalar(&im->seq), hk = ld_scalar(&im->head), t0 = ld_scalar(&im->t0), t1 = ld_scalar(&im->t1);
    int base = ld_scalar(&im->base);
    const int cols = ld_scalar(&im->cols), wc = ld_scalar(&im->waves_c), wk = 4 / wc;
    int block = ld_scalar(&im->block), step = 1, pos = 0;
    bool idle = false;
    if (what == 2) {
      const int pair = e0 + w;
      idle = pair >= seq;
      e0 = idle ? 0 : pair / p.n_kv_heads;
      hk = idle ? 0 : pair - e0 * p.n_kv_heads;
      const Ent* e = a.ent + e0;
      seq = ld_scalar(&e->seq);
      idle = idle || seq < 0;
      pos = ld_scalar(&e->pos);
      t0 = ld_scalar(&e->shared);
      t1 = idle ? t0 : (pos + a.tokens + kPage - 1) / kPage;
      base = ld_scalar(&e->own_base) + hk * per_entry;
    } else {
      if (what == 1) pos = ld_scalar(&a.ent[e0].pos);
      block += w & (wc - 1);
      t0 += w / wc;
      step = wk;
      idle = block * 32 >= cols;
      if (idle) t1 = t0;
    }
    // this lane's column
    const int c = block * 32 + j, cc = min(c, cols - 1);
    const int ei = cc / per_entry, ci = cc - ei * per_entry, ti = ci / grp, row = (e0 + ei) * a.tokens + ti;
    const int h = hk * grp + ci - ti * grp;
    const bool masked = what != 0;
    const int last = pos + ti;                 // own segments: this column's last visible position
    const int end = pos + a.tokens;            // positions from here on were never written
    uint4 qf[NC];
    if (t0 < t1) {
      const bf16_t* q = a.q_stride < 0 ? a.q + ((size_t)(row >> 5) * a.n_q_heads + h) * (size_t)NC * 512 + (size_t)(((row & 31) + 32 * g) << 3)
                                       : a.q + (size_t)row * a.q_stride + (size_t)h * HD + 8 * g;
      const int q_step = a.q_stride < 0 ? 512 : 16;
#pragma unroll
      for (int x = 0; x < NC; ++x) qf[x] = *(const uint4*)(q + (size_t)x * q_step);
    }
    const bf16_t* kv = p.data + ((size_t)a.layer * 2 * p.n_kv_heads + hk) * tile + (size_t)lane * 8;
    const size_t v_off = (size_t)p.n_kv_heads * tile;
    const int* table = p.table + (size_t)max(seq, 0) * p.max_pages;

    f32x16 o[NI];
#pragma unroll
    for (int ib = 0; ib < NI; ++ib)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[ib][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    // pages of the next 64 tiles, one per lane (an index out of range reads page 0: the table is the caller's)
    int ids = 0;
    auto load_ids = [&](int kt) {
      const int at = kt + lane * step;
      ids = at < t1 ? table[at] : 0;
      if ((unsigned)ids >= (unsigned)p.n_pages) {
        ids = 0;
        report(p, PAGES_BAD_ENTRY);
      }
    };
    uint4 kf[NC];
    auto tile_of = [&](int n) { return kv + (size_t)__builtin_amdgcn_readlane(ids, n) * page; };
    auto load_k = [&](const bf16_t* t) {
#pragma unroll
      for (int x = 0; x < NC; ++x) kf[x] = *(const uint4*)(t + x * 512);
    };
    const bf16_t* now = nullptr;
    if (t0 < t1) {
      load_ids(t0);
      now = tile_of(0);
      load_k(now);
    }
    int n_at = 0;
    bool odd = false;
    for (int kt = t0; kt < t1; kt += step) {
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int x = 0; x < NC; ++x) s = mfma32<F16>(kf[x], qf[x], s);
      __builtin_amdgcn_sched_barrier(0);
      uint4 vf[NI * 2];
#pragma unroll
      for (int t = 0; t < NI * 2; ++t) vf[t] = *(const uint4*)(now + v_off + t * 512);
      if (kt + step < t1) {
        if (++n_at == 64) {
          load_ids(kt + step);
          n_at = 0;
        }
        now = tile_of(n_at);
        load_k(now);
      }
      __builtin_amdgcn_sched_barrier(0);
      // register 4*q4 + e of a lane is key 32*kt + 8*q4 + 4*g + e
      float tmax = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int kp = 32 * kt + 8 * (i >> 2) + 4 * g + (i & 3);
        s[i] = (!masked || kp <= last) ? s[i] * a.scale_log2e : -INFINITY;
        tmax = fmaxf(tmax, s[i]);
      }
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
      const float m_new = fmaxf(m, tmax);
      const float alpha = (m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
      m = m_new;
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(s[i] - m_use);
        psum += s[i];
      }
      l = l * alpha + psum;
      uint4 pb[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        pb[t].x = pack2<F16>(s[8 * t + 0], s[8 * t + 1]);
        pb[t].y = pack2<F16>(s[8 * t + 2], s[8 * t + 3]);
        pb[t].z = pack2<F16>(s[8 * t + 4], s[8 * t + 5]);
        pb[t].w = pack2<F16>(s[8 * t + 6], s[8 * t + 7]);
      }
      if (masked && 32 * kt + 31 > pos) {
        // V of positions that hold no token may be anything, NaN among it, and 0 x NaN is not 0.  Positions behind the
        // first query are seen by some columns only: what is not finite there is left for behind the loop.
#pragma unroll
        for (int t = 0; t < NI * 2; ++t) {
          uint32_t* x = (uint32_t*)&vf[t];
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int kp = 32 * kt + 16 * (t & 1) + 8 * (d >> 1) + 4 * g + 2 * (d & 1);
            const uint32_t far = far_values<F16>(x[d], kp > pos, kp + 1 > pos);
            const uint32_t seen = kp + 1 < end ? ~0u : kp < end ? 0xffffu : 0u;
            odd |= (far & seen) != 0;
            x[d] &= seen & ~far;
          }
        }
      }
#pragma unroll
      for (int ib = 0; ib < NI; ++ib) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[ib][i] *= alpha;
#pragma unroll
        for (int t = 0; t < 2; ++t) o[ib] = mfma32<F16>(vf[ib * 2 + t], pb[t], o[ib]);
      }
    }
    l += __shfl_xor(l, 32);
    if (masked && __any(odd)) {
      // infinities and NaN of V where some columns see them and some do not: key by key, added where they are seen
      for (int kt = t0; kt < t1; kt += step) {
        if (32 * kt + 31 <= pos) continue;
        const int pg = table[kt];
        const bf16_t* at = kv + (size_t)((unsigned)pg < (unsigned)p.n_pages ? pg : 0) * page;
        load_k(at);
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int x = 0; x < NC; ++x) s = mfma32<F16>(kf[x], qf[x], s);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int kp = 32 * kt + 8 * (i >> 2) + 4 * g + (i & 3);
          s[i] = kp <= last ? __builtin_amdgcn_exp2f(s[i] * a.scale_log2e - (m == -INFINITY ? 0.f : m)) : 0.f;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint4 pb = {pack2<F16>(s[8 * t], s[8 * t + 1]), pack2<F16>(s[8 * t + 2], s[8 * t + 3]),
                            pack2<F16>(s[8 * t + 4], s[8 * t + 5]), pack2<F16>(s[8 * t + 6], s[8 * t + 7])};
#pragma unroll
          for (int ib = 0; ib < NI; ++ib) {
            const uint4 v = *(const uint4*)(at + v_off + (ib * 2 + t) * 512);
            const uint32_t* x = (const uint32_t*)&v;
            for (int k = max(pos + 1 - 32 * kt - 16 * t, 0); k < min(end - 32 * kt - 16 * t, 16); ++k) {
              const bool here = g == (k >> 2 & 1), sees = 32 * kt + 16 * t + k <= last;
              uint4 only;
              uint32_t* y = (uint32_t*)&only;
#pragma unroll
              for (int d = 0; d < 4; ++d)
                y[d] = here && d == 2 * (k >> 3) + (k >> 1 & 1) ? x[d] & far_values<F16>(x[d], !(k & 1), k & 1) : 0u;
              f32x16 z;
#pragma unroll
              for (int i = 0; i < 16; ++i) z[i] = 0.f;
              z = mfma32<F16>(only, pb, z);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[ib][i] += sees ? z[i] : 0.f;
            }
          }
        }
      }
    }

    auto store = [&](int ib, const f32x16& x) {
      float* d = a.o + (size_t)(base + c) * HD + 32 * ib + 4 * g;
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *(float4*)(d + 8 * q4) = make_float4(x[4 * q4], x[4 * q4 + 1], x[4 * q4 + 2], x[4 * q4 + 3]);
    };
    if (what == 2 || wk == 1) {
      if (!idle && c < cols) {
#pragma unroll
        for (int ib = 0; ib < NI; ++ib) store(ib, o[ib]);
        if (g == 0) a.ml[base + c] = make_float2(m, l);
      }
    } else {
      // the waves of a column block meet in LDS, a share of the feature blocks each, in the order of the waves
      park[w][0][lane] = m;
      park[w][1][lane] = l;
#pragma unroll
      for (int ib = 0; ib < NI; ++ib)
#pragma unroll
        for (int i = 0; i < 16; ++i) park[w][2 + ib * 16 + i][lane] = o[ib][i];
      __syncthreads();
      const int w0 = w & (wc - 1), share = w / wc;
      float M = -INFINITY;
      for (int x = 0; x < wk; ++x) M = fmaxf(M, park[w0 + x * wc][0][lane]);
      const float m_use = M == -INFINITY ? 0.f : M;
      float L = 0.f, f[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f[x] = x < wk ? __builtin_amdgcn_exp2f(park[w0 + x * wc][0][lane] - m_use) : 0.f;
        if (x < wk) L = fmaf(f[x], park[w0 + x * wc][1][lane], L);
      }
      if (!idle && c < cols) {
        for (int ib = share; ib < NI; ib += wk) {
          f32x16 x;
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (y < wk) {
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = fmaf(f[y], park[w0 + y * wc][2 + ib * 16 + i][lane], x[i]);
            }
          store(ib, x);
        }
        if (share == 0 && g == 0) a.ml[base + c] = make_float2(M, L);
      }
      __syncthreads();
    }
  }
}

// A wave per row: the parts of its segments, shared ones first, in their order
template <int HD, bool F16>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  const PoolView& p = a.p;
  const int lane = threadIdx.x & 63;
  const long long rh = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (rh >= (long long)a.n * a.tokens * a.n_q_heads) return;
  const int grp = a.n_q_heads / p.n_kv_heads, per_entry = a.tokens * grp;
  const int row = (int)(rh / a.n_q_heads), h = (int)(rh - (long long)row * a.n_q_heads);
  const int i = row / a.tokens, t = row - i * a.tokens, hk = h / grp, ci = t * grp + h - hk * grp;
  const Ent* e = a.ent + i;
  const bool valid = ld_scalar(&e->seq) >= 0;
  const int sp = valid ? ld_scalar(&e->sh_parts) : 0, op = valid ? ld_scalar(&e->own_parts) : 0;
  const int cols = ld_scalar(&e->cols);
  const size_t sh = ld_scalar(&e->sh_base) + (size_t)hk * sp * cols + ld_scalar(&e->c0) + ci;
  const size_t ow = ld_scalar(&e->own_base) + (size_t)hk * op * per_entry + ci;
  float2 s = make_float2(-INFINITY, 0.f), w = make_float2(-INFINITY, 0.f);
  if (lane < sp) s = a.ml[sh + (size_t)lane * cols];
  if (lane < op) w = a.ml[ow + (size_t)lane * per_entry];
  float M = fmaxf(s.x, w.x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) M = fmaxf(M, __shfl_xor(M, d));
  const float m_use = M == -INFINITY ? 0.f : M;
  const float fs = __builtin_amdgcn_exp2f(s.x - m_use), fw = __builtin_amdgcn_exp2f(w.x - m_use);
  float L = fs * s.y + fw * w.y;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) L += __shfl_xor(L, d);
  constexpr int PER = HD / 64;
  float acc[PER] = {};
  auto add = [&](size_t col, float f) {
    const float* o = a.o + col * HD + lane * PER;
#pragma unroll
    for (int x = 0; x < PER; ++x) acc[x] = fmaf(f, o[x], acc[x]);
  };
  for (int x = 0; x < sp; ++x) add(sh + (size_t)x * cols, __shfl(fs, x));
  for (int x = 0; x < op; ++x) add(ow + (size_t)x * per_entry, __shfl(fw, x));
  const float inv = valid ? 1.f / L : 0.f;
  bf16_t* d = a.kc_out > 0 ? a.out + frag_off(row, h * HD + lane * PER, a.kc_out) : a.out + (size_t)rh * HD + lane * PER;
  if (PER == 2) *(uint32_t*)d = pack2<F16>(acc[0] * inv, acc[PER - 1] * inv);
  else *d = (bf16_t)pack2<F16>(acc[0] * inv, 0.f);
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

// 0: more partial columns than an int counts
size_t attend_workspace(const PoolView& p, int n, int tokens, int n_q_heads) {
  const Layout l = layout_of(n > 0 ? n : 1, tokens, n_q_heads, p.n_kv_heads, p.head_dim);
  return l.max_cols > 0x7fffffffu || l.max_items > 0x7fffffffu ? 0 : l.total;
}

void launch_attend_plan(const PoolView& p, const int* seqs, const int* pos, int add, int n, int tokens, int n_q_heads,
                        const int* group, void* ws, hipStream_t st) {
  const Layout l = layout_of(n, tokens, n_q_heads, p.n_kv_heads, p.head_dim);
  char* b = (char*)ws;
  const PlanArgs a = {p, seqs, pos, group, add, n, tokens, n_q_heads, l.split_shared, l.split_own, (int)l.max_items,
                      (int*)b, (Ent*)(b + l.ent), (Item*)(b + l.item)};
  hipLaunchKernelGGL(attend_plan_kernel, dim3(1), dim3(kPlan), 0, st, a);
}

void launch_attend(const PoolView& p, bool f16, int layer, int n, int tokens, int n_q_heads, const AttendIo& io, void* ws,
                   hipStream_t st) {
  const Layout l = layout_of(n, tokens, n_q_heads, p.n_kv_heads, p.head_dim);
  char* b = (char*)ws;
  const AttendArgs a = {p, (const int*)b, (const Ent*)(b + l.ent), (const Item*)(b + l.item), (float2*)(b + l.ml), (float*)(b + l.o),
                        io.q, io.q_stride, io.out, io.kc_out, layer, n, tokens, n_q_heads,
                        1.4426950408889634f / sqrtf((float)p.head_dim)};
  const dim3 grid((unsigned)std::min<size_t>(l.max_items, 2 * kSlots));
  const long long rows = (long long)n * tokens * n_q_heads;
  const dim3 join((unsigned)((rows + 3) / 4));
#define VLAC_ATTEND(HD_, F16_)                                                             \
  {                                                                                        \
    hipLaunchKernelGGL((attend_kernel<HD_, F16_>), grid, dim3(256), 0, st, a);             \
    hipLaunchKernelGGL((attend_join_kernel<HD_, F16_>), join, dim3(256), 0, st, a);        \
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
  if (q_stride < (int64_t)n_q_heads * pages->head_dim || q_stride % 8 || q_stride > 1 << 30 || (uintptr_t)q % 16 || (uintptr_t)out % 4)
    return VLAC_E_SHAPE;
  const AttendIo io = {(const bf16_t*)q, q_stride, (bf16_t*)out, 0};
  launch_attend(pool_view(pages), pages_f16(pages), layer, n, tokens, n_q_heads, io, workspace, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
