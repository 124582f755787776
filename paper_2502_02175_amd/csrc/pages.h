// Pages of the cache: what the kernels on tables, pages and attention over them share.
#pragma once
#include "common.h"

static const int kPage = 32;  // positions of a page
enum { PAGES_BAD_ENTRY = 1, PAGES_NO_ROOM = 2 };

// scratch of a pool: [0] status bits, [1] pages to copy, [2] free, then from 16 on
//   copy_src [n_pages], copy_dst [n_pages] (fork and import: the fresh pages in the order they are given out),
//   moved_to [n_pages] (compact), is_dst [max_seqs], is_src [max_seqs] (zero between calls)
enum { PG_STATUS = 0, PG_COPIES = 1, PG_LISTS = 16 };

// What the kernels see of a pool (head_dim and type are template arguments or in the strides)
struct PoolView {
  bf16_t* data;
  int *refs, *table, *len, *scratch;
  int n_pages, max_seqs, max_pages;
  int n_layers, n_kv_heads, head_dim;
  __host__ __device__ size_t tile() const { return (size_t)kPage * head_dim; }   // a head's K or V of a page
  __host__ __device__ size_t page() const { return (size_t)n_layers * 2 * n_kv_heads * tile(); }
  __host__ __device__ int* copy_src() const { return scratch + PG_LISTS; }
  __host__ __device__ int* copy_dst() const { return copy_src() + n_pages; }
  __host__ __device__ int* moved_to() const { return copy_dst() + n_pages; }
  __host__ __device__ int* is_dst() const { return moved_to() + n_pages; }
  __host__ __device__ int* is_src() const { return is_dst() + max_seqs; }
};

static inline PoolView pool_view(const vlac_pages* p) {
  PoolView v;
  v.data = (bf16_t*)p->data;
  v.refs = p->refs; v.table = p->table; v.len = p->len; v.scratch = p->scratch;
  v.n_pages = p->n_pages; v.max_seqs = p->max_seqs; v.max_pages = p->max_pages;
  v.n_layers = p->n_layers; v.n_kv_heads = p->n_kv_heads; v.head_dim = p->head_dim;
  return v;
}

// host checks: sizes, and (pointers = true) the buffers
int check_pages(const vlac_pages* p, bool pointers);
static inline bool pages_f16(const vlac_pages* p) { return p->operand_dtype != VLAC_OPERAND_BF16; }

#ifdef __HIPCC__
__device__ inline int pages_of(int len) { return (len + kPage - 1) / kPage; }
// the length of a sequence, or -1 where the index or the length is out of range
__device__ inline int checked_len(const PoolView& p, int s) {
  if ((unsigned)s >= (unsigned)p.max_seqs) return -1;
  const int l = p.len[s];
  return l < 0 || l > p.max_pages * kPage ? -1 : l;
}
__device__ inline void report(const PoolView& p, int bit) { atomicOr(p.scratch + PG_STATUS, bit); }

// Sums over the lanes up to this one, and a maximum over all, by moves between lanes inside the vector ALU (shifts within rows
// of 16 lanes, then the last lane of a row into the next, and of the first half into the second): 6 dependent instructions where
// shuffles through LDS take 6 round trips, and the planning kernels, which are chains of such sums, 1 to 3 us less.
template <int HOW, int ROWS>
__device__ inline int lanes_moved(int x) { return __builtin_amdgcn_update_dpp(0, x, HOW, ROWS, 0xf, false); }
__device__ inline int row_sums(int x) {  // (of 16 lanes)
  x += lanes_moved<0x111, 0xf>(x);
  x += lanes_moved<0x112, 0xf>(x);
  x += lanes_moved<0x114, 0xf>(x);
  return x + lanes_moved<0x118, 0xf>(x);
}
__device__ inline int wave_sums(int x) {
  x = row_sums(x);
  x += lanes_moved<0x142, 0xa>(x);
  return x + lanes_moved<0x143, 0xc>(x);
}
__device__ inline int wave_max(int x) {  // (x >= 0)
  x = max(x, lanes_moved<0x111, 0xf>(x));
  x = max(x, lanes_moved<0x112, 0xf>(x));
  x = max(x, lanes_moved<0x114, 0xf>(x));
  x = max(x, lanes_moved<0x118, 0xf>(x));
  x = max(x, lanes_moved<0x142, 0xa>(x));
  x = max(x, lanes_moved<0x143, 0xc>(x));
  return __builtin_amdgcn_readlane(x, 63);
}
#endif

// pages.hip
void launch_extend(const PoolView& p, const int* seqs, int n, int tokens, int want_len, int* out_pos, hipStream_t st);
// K and V of one token per entry, at pos[i] + add, from tiles [n][K, V][n_kv_heads][32 * head_dim] (row (pos + add) % 32 of each)
void launch_append_tiles(const PoolView& p, int layer, const int* seqs, const int* pos, int add, int n,
                         const bf16_t* tiles, hipStream_t st);

// attend.hip: where the query rows come from and where the results go
struct AttendIo {
  const bf16_t* q;
  long long q_stride;  // elements between rows; < 0: fragment order per head (the QKV epilogue's), rows as slots
  bf16_t* out;
  int kc_out;          // > 0: fragment order with this many k-tiles, else [rows][n_q_heads][head_dim]
};
size_t attend_workspace(const PoolView& p, int n, int tokens, int n_q_heads);
void launch_attend_plan(const PoolView& p, const int* seqs, const int* pos, int add, int n, int tokens, int n_q_heads,
                        const int* group, void* ws, hipStream_t st);
void launch_attend(const PoolView& p, bool f16, int layer, int n, int tokens, int n_q_heads, const AttendIo& io, void* ws,
                   hipStream_t st);
