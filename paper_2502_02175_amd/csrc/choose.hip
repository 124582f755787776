// What may be chosen, and at what price: the rules of vlac_token_rules over rows of logits, and the greatest of each row.
//   l -> l > 0 ? l / repetition : l * repetition, - presence   where the row's text holds the token,
//   l -> l - frequency * count, l -> l + bias, l -> -infinity where it is not allowed; every step rounded to fp32.
// A workgroup takes a piece of a row: how often its text holds each token of the piece is counted in LDS (whole numbers, so
// that the order of the atomics decides nothing), then the piece goes by once.  The greatest logits of the pieces meet in a
// second launch (of 2 us; a workspace that has to be zero before a call would save it).
// Large calls are bound by memory: 1024 rows of 100000 (0.82 GB) 157 us, 5.2 TB/s; 256 rows of 32000 with texts of 1057 tokens
// (67 MB) 19.8.  Small ones by the chain arguments - logits and length - text - counts - second launch: one row of 32000 6.6.
#include <algorithm>
#include <cmath>

#include "choose.h"
#include "trees.h"

namespace {

constexpr int NT = 256;  // threads of a workgroup

// A logit's store, non-temporal in large calls (256 rows of 32000 21.2 -> 19.8 us, 96 of 150001 39 -> 33; loads marked so as well: 20 and 42)
template <bool STREAM>
__device__ inline void put(float* to, float x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, to);
  else *to = x;
}

// The greatest of a row so far, and its token; what is not above -infinity (a NaN among it) is never taken
struct Best { float v; int at; };
__device__ inline void take(Best& b, float v, int at) {
  if (v > b.v || (v == b.v && at < b.at)) { b.v = v; b.at = at; }
}
constexpr int kNobody = 0x7fffffff;

// Over the workgroup, in every thread of the first wave
__device__ inline Best best_of_all(Best b, float* sv, int* si) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float v = __shfl_xor(b.v, d);
    const int i = __shfl_xor(b.at, d);
    take(b, v, i);
  }
  if ((tid & 63) == 0) { sv[tid >> 6] = b.v; si[tid >> 6] = b.at; }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NT / 64; ++k) take(b, sv[k], si[k]);
  return b;
}

// -infinity is the start of every search: equal values do not replace it, so a row of nothing but -infinity has no token
__device__ inline int token_of(const Best& b) { return b.v > -INFINITY ? b.at : -1; }

// A logit under the rules, every step rounded by itself (a multiply-add would round product and difference at once)
__device__ inline float priced(float y, int n, float repetition, float presence, float frequency) {
#pragma clang fp contract(off)
  if (__builtin_expect(n > 0, 0)) {
    y = y > 0.f ? __fdiv_rn(y, repetition) : y * repetition;
    y = y - presence;
    y = y - frequency * (float)n;
  }
  return y;
}

// A workgroup takes PER logits per thread, all of which (and the bias and the mask) are asked for before the text is counted: the
// chain of the counting (lengths, tokens, LDS) hides behind them.
template <bool COUNTS, int PER>
__global__ __launch_bounds__(NT) void choose_kernel(ChooseArgs a) {
  constexpr int PIECE = NT * PER;
  __shared__ __align__(16) int counts[COUNTS ? PIECE : 4];
  __shared__ short above[COUNTS ? VLAC_TREE_MAX_NODES : 1];
  __shared__ int drafts[COUNTS ? VLAC_TREE_MAX_NODES : 1];
  __shared__ float sv[NT / 64];
  __shared__ int si[NT / 64];
  read_args(a.logits, a.rows, a.vocab, a.stride, a.out, a.out_stride, a.token, a.token_stride, a.best, a.repetition, a.presence, a.frequency,
            a.bias, a.bias_stride, a.allowed, a.allowed_stride, a.history, a.history_len, a.history_stride, a.tokens, a.parents,
            a.drafted, a.more, a.more_stride, a.more_n, a.one, a.pieces, a.row0, a.rule_row0, a.rule_rows);
  const int tid = threadIdx.x, local = blockIdx.x / a.pieces, piece = blockIdx.x - local * a.pieces, row = a.row0 + local;
  const int c0 = piece * PIECE, entry = row / a.tokens, node = row - entry * a.tokens;
  const size_t rule_row = (size_t)row * a.rule_rows + a.rule_row0;
  const float* const x = a.logits + row * a.stride;
  const float* const bias = a.bias ? a.bias + rule_row * a.bias_stride : nullptr;
  const bool whole = c0 + PIECE <= a.vocab;  // (else: past the end the last again)
  float l[PER], add[PER];
  auto load = [&](float(&to)[PER], const float* from) {
    if (whole) {
#pragma unroll
      for (int u = 0; u < PER; ++u) to[u] = (from + c0)[(unsigned)(u * NT + tid)];
    } else {
#pragma unroll
      for (int u = 0; u < PER; ++u) to[u] = from[(unsigned)min(c0 + u * NT + tid, a.vocab - 1)];
    }
  };
  load(l, x);
  if (bias) load(add, bias);
  // The mask: a wave's 64 tokens are two words, and a lane has one of the 2 PER words of them all
  const uint32_t* const allowed = a.allowed ? a.allowed + rule_row * a.allowed_stride : nullptr;
  uint32_t mask = ~0u;
  if (allowed) {
    const int lane = tid & 63, at = ((c0 + (lane >> 1) * NT + (tid & ~63)) >> 5) + (lane & 1), words = (a.vocab + 31) >> 5;
    mask = lane < 2 * PER && at < words ? allowed[at] : 0u;
  }
  if (COUNTS) {
    constexpr int U = 8;  // of the text's tokens in flight
    const unsigned n = a.history ? (unsigned)min((long long)max(a.history_len[entry], 0), a.history_stride) : 0u;  // (up to 2^31 - 1)
    const int* text = a.history + entry * a.history_stride;
    for (int k = tid; k < PIECE / 4; k += NT) ((int4*)counts)[k] = make_int4(0, 0, 0, 0);
    if (a.parents)
      for (int t = tid; t < a.tokens; t += NT) {
        const int up = a.parents[(size_t)entry * a.tokens + t];
        drafts[t] = a.drafted[(size_t)entry * a.tokens + t];
        above[t] = (short)(up < -2 || up >= t ? -2 : up);
      }
    __syncthreads();
    auto count = [&](int token) {
      const unsigned at = (unsigned)token - (unsigned)c0;
      if (at < (unsigned)PIECE) atomicAdd(&counts[at], 1);
    };
    for (unsigned k0 = tid; k0 < n; k0 += U * NT) {
      int token[U];
#pragma unroll
      for (int u = 0; u < U; ++u) token[u] = k0 + u * NT < n ? text[k0 + u * NT] : -1;
#pragma unroll
      for (int u = 0; u < U; ++u) count(token[u]);
    }
    for (int k = tid; k < a.more_n; k += NT) count(a.more[(size_t)entry * a.more_stride + k]);
    if (a.one && tid == 0) count(a.one[entry]);
    if (a.parents && tid >= NT - 64) {  // (the last wave: the drafts of the row's node and of those above it)
      uint64_t way;
      const int end = follow<true>(node, [&](int t) { return t < a.tokens ? (int)above[t] : -2; }, way);
      if (end == -1)
        for (int k = 0; 64 * k <= node; ++k)
          if (part_of(way, k) >> (tid & 63) & 1) count(drafts[64 * k + (tid & 63)]);
    }
    __syncthreads();
  }
  float best = -INFINITY;
  int best_u = -1;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (COUNTS) {
      const int n = counts[u * NT + tid];
      if (__any(n > 0)) l[u] = priced(l[u], n, a.repetition, a.presence, a.frequency);
    }
    if (bias) l[u] = l[u] + add[u];
    const uint64_t words = (uint64_t)__builtin_amdgcn_readlane(mask, 2 * u + 1) << 32 | (uint32_t)__builtin_amdgcn_readlane(mask, 2 * u);
    l[u] = __builtin_amdgcn_inverse_ballot_w64(words) ? l[u] : -INFINITY;
    // (a thread's tokens ascend: of equal ones the first stays)
    if (l[u] > best && (whole || c0 + u * NT + tid < a.vocab)) {
      best = l[u];
      best_u = u;
    }
  }
  if (a.out) {
    float* const out = a.out + row * a.out_stride + c0;
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (whole || c0 + u * NT + tid < a.vocab) put<(PER > 4)>(out + (unsigned)(u * NT + tid), l[u]);
  }
  if (!a.token) return;
  const Best b = best_of_all({best, best_u < 0 ? kNobody : c0 + best_u * NT + tid}, sv, si);
  if (tid == 0) {
    if (a.pieces > 1) a.best[(size_t)row * a.pieces + piece] = make_float2(b.v, __int_as_float(b.at));
    else a.token[(size_t)row * a.token_stride] = token_of(b);
  }
}

// The pieces' best, a wave per row
__global__ __launch_bounds__(NT) void choose_join_kernel(ChooseArgs a) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * (NT / 64) + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  Best b = {-INFINITY, kNobody};
  for (int k = lane; k < a.pieces; k += 64) {
    const float2 x = a.best[(size_t)row * a.pieces + k];
    take(b, x.x, __float_as_int(x.y));
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float v = __shfl_xor(b.v, d);
    const int i = __shfl_xor(b.at, d);
    take(b, v, i);
  }
  if (lane == 0) a.token[(size_t)row * a.token_stride] = token_of(b);
}

// Logits of a workgroup of 256 threads: 4 per thread where there are few, so that many workgroups share the counting and the
// chain before it, 16 where the chip is full anyhow (us with 1024 and with 4096, texts of 1000 tokens, 32000 logits a row: 1 row 6.8
// and 9.5, 16 rows 7.6 and 9.9, 64 rows 12.3 and 11.4, 256 rows 27 and 19; 8 rows of 150001 11.3 and 12.0; 1920 rows of 1000 10.2 and 12.5).
// (8192 by 512 threads: 1 to 3 us more than 4096 throughout.)
constexpr int kSmall = 4 * NT, kLarge = 16 * NT;
int piece_of(int rows, int vocab) { return vocab <= 2 * kSmall || (long long)rows * vocab < 3 << 19 ? kSmall : kLarge; }
int pieces_of(int vocab, int piece) { return (vocab + piece - 1) / piece; }

}  // namespace

int check_rules(const vlac_token_rules* r, int vocab) {
  if (!r) return VLAC_E_NULL;
  if (!(std::isfinite(r->repetition) && r->repetition > 0.f && std::isfinite(r->presence) && std::isfinite(r->frequency)))
    return VLAC_E_RANGE;
  if (r->tokens < 1 || r->tokens > VLAC_TREE_MAX_NODES) return VLAC_E_RANGE;
  if ((r->history == nullptr) != (r->history_len == nullptr) || (r->parents == nullptr) != (r->drafted == nullptr)) return VLAC_E_NULL;
  if (!r->parents && r->tokens > 1) return VLAC_E_NULL;
  if (r->bias && r->bias_stride != 0 && r->bias_stride < vocab) return VLAC_E_SHAPE;
  if (r->allowed && r->allowed_stride != 0 && r->allowed_stride < (vocab + 31) / 32) return VLAC_E_SHAPE;
  if (r->history && (r->history_stride < 0 || r->history_stride > 1LL << 31)) return VLAC_E_SHAPE;
  if ((r->bias && r->bias_stride > 1LL << 31) || (r->allowed && r->allowed_stride > 1LL << 31)) return VLAC_E_SHAPE;
  if ((uintptr_t)r->bias % 4 || (uintptr_t)r->allowed % 4 || (uintptr_t)r->history % 4 || (uintptr_t)r->history_len % 4 ||
      (uintptr_t)r->parents % 4 || (uintptr_t)r->drafted % 4)
    return VLAC_E_SHAPE;
  return VLAC_OK;
}

size_t choose_workspace(int rows, int vocab) { return ((size_t)std::max(rows, 1) * pieces_of(vocab, kSmall) * sizeof(float2) + 255) / 256 * 256; }

ChooseArgs choose_args(const float* logits, int rows, int vocab, int64_t stride, const vlac_token_rules& r, float* out, int64_t out_stride,
                       int32_t* token, void* ws) {
  ChooseArgs a = {};
  a.logits = logits; a.rows = rows; a.vocab = vocab; a.stride = stride;
  a.out = out; a.out_stride = out_stride;
  a.token = token; a.token_stride = 1;
  a.best = (float2*)ws;
  a.repetition = r.repetition; a.presence = r.presence; a.frequency = r.frequency;
  a.bias = r.bias; a.bias_stride = r.bias_stride;
  a.allowed = r.allowed; a.allowed_stride = r.allowed_stride;
  a.history = r.history; a.history_len = r.history_len; a.history_stride = r.history_stride;
  a.tokens = r.tokens; a.parents = r.parents; a.drafted = r.drafted;
  a.rule_rows = 1;
  return a;
}

void launch_choose(ChooseArgs a, hipStream_t st) {
  const int piece = piece_of(a.rows, a.vocab);
  a.pieces = pieces_of(a.vocab, piece);
  const bool prices = a.repetition != 1.f || a.presence != 0.f || a.frequency != 0.f;
  const bool counts = prices && (a.history || a.parents || a.more_n > 0 || a.one);
  const int most = std::max(1, (1 << 23) / a.pieces);  // rows of a launch (one of 2^32 threads would not run whole)
  for (a.row0 = 0; a.row0 < a.rows; a.row0 += most) {
    const dim3 grid((unsigned)(std::min(a.rows - a.row0, most) * a.pieces));
    if (piece == kSmall) {
      if (counts) hipLaunchKernelGGL((choose_kernel<true, 4>), grid, dim3(NT), 0, st, a);
      else hipLaunchKernelGGL((choose_kernel<false, 4>), grid, dim3(NT), 0, st, a);
    } else {
      if (counts) hipLaunchKernelGGL((choose_kernel<true, 16>), grid, dim3(NT), 0, st, a);
      else hipLaunchKernelGGL((choose_kernel<false, 16>), grid, dim3(NT), 0, st, a);
    }
  }
  if (a.token && a.pieces > 1)
    hipLaunchKernelGGL(choose_join_kernel, dim3((unsigned)((a.rows + NT / 64 - 1) / (NT / 64))), dim3(NT), 0, st, a);
}

extern "C" {

size_t vlac_choose_workspace_bytes(int rows, int vocab) {
  return rows < 0 || rows > VLAC_CHOOSE_MAX_ROWS || vocab < 1 || vocab > 1 << 24 ? 0 : choose_workspace(rows, vocab);
}

int vlac_choose_tokens(const float* logits, int rows, int vocab, int64_t stride, const vlac_token_rules* rules, float* out_logits,
                       int64_t out_stride, int32_t* out_token, void* workspace, size_t workspace_bytes, void* stream) {
  if (rows < 0 || rows > VLAC_CHOOSE_MAX_ROWS || vocab < 1 || vocab > 1 << 24) return VLAC_E_RANGE;
  const int rc = check_rules(rules, vocab);
  if (rc != VLAC_OK) return rc;
  if (rows % rules->tokens) return VLAC_E_SHAPE;
  if (stride < vocab || stride > 1LL << 31) return VLAC_E_SHAPE;
  if (out_logits && (out_stride < vocab || out_stride > 1LL << 31 || (out_logits == logits && out_stride != stride))) return VLAC_E_SHAPE;
  if (rows == 0) return VLAC_OK;
  if (!logits || (out_token && !workspace)) return VLAC_E_NULL;
  if ((uintptr_t)logits % 4 || (uintptr_t)out_logits % 4 || (uintptr_t)out_token % 4 || (out_token && (uintptr_t)workspace % 16))
    return VLAC_E_SHAPE;
  if (out_token && workspace_bytes < choose_workspace(rows, vocab)) return VLAC_E_RANGE;
  if (!out_logits && !out_token) return VLAC_OK;
  launch_choose(choose_args(logits, rows, vocab, stride, *rules, out_logits, out_stride, out_token, workspace), (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
