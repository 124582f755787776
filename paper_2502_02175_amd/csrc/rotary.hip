// Queries, keys and values of new tokens on their way into the pages: the norm of every head and the rotation of its position
// in the same pass,
//   q' = R(place) N(q), k' = R(place) N(k), v' = v,   N(x) = x rsqrt(mean x^2 + eps) gain,
//   R turns pair f by 2 pi turns[f] place (in 64 bits up to the fraction of a turn: 32 lose it at far places).
#include <algorithm>
#include <cmath>

#include "pages.h"

namespace {

struct RotaryArgs {
  PoolView p;
  int layer, n, tokens, blocks;  // blocks: of 8 positions that an entry's tokens may touch
  const int *seqs, *pos, *places;
  int n_q_heads;
  const bf16_t *q, *k, *v;
  long long q_stride, kv_stride;
  bf16_t* q_out;
  long long q_out_stride;
  const bf16_t *q_gain, *k_gain;
  float eps;
  int dims, pairs;  // rotated features (0: none); pairs: neighbours are a pair
  float amplitude;
  const double* turns;
  int first;  // wave of the call that this launch begins with
};

template <bool F16>
__device__ inline void widen(uint32_t x, float& lo, float& hi) {
  if constexpr (F16) {
    const f16x2v h = __builtin_bit_cast(f16x2v, x);
    lo = (float)h[0];
    hi = (float)h[1];
  } else {
    lo = __uint_as_float(x << 16);
    hi = __uint_as_float(x & 0xffff0000u);
  }
}
// Rounded once, half a step; in fp16 finite values beyond its range saturate, what is infinite or NaN stays it
template <bool F16>
__device__ inline uint32_t narrow2(float lo, float hi) {
  if constexpr (F16) {
    const float a = fabsf(lo) < INFINITY ? __builtin_amdgcn_fmed3f(lo, -65504.f, 65504.f) : lo;
    const float b = fabsf(hi) < INFINITY ? __builtin_amdgcn_fmed3f(hi, -65504.f, 65504.f) : hi;
    const f32x2v v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2v));
  } else {
    return f2bf2(lo, hi);
  }
}

// Sum over the GROUP lanes (8 or 16, aligned) that share a row
template <int GROUP>
__device__ inline float row_sum(float x) {
#pragma unroll
  for (int d = 1; d < GROUP; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// A wave takes one head (of the queries, the keys or the values) at 8 positions that lie side by side in a page: one page to
// look up, and a K store of 8 rows is a line.  A lane holds 8 features of a row, so head_dim / 8 lanes hold a row; the partners of a
// pair, and V's 4 neighbouring positions, meet in LDS.
template <int HD, bool F16>
__global__ __launch_bounds__(256) void rotary_append_kernel(RotaryArgs a) {
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, STEPS = 8 / ROWS;  // rows at a time
  __shared__ float meet[4][8 * HD];
  const PoolView& p = a.p;
  read_args(a.layer, a.n, a.tokens, a.blocks, a.seqs, a.pos, a.places, a.n_q_heads, a.q, a.k, a.v, a.q_stride, a.kv_stride, a.q_out,
            a.q_out_stride, a.q_gain, a.k_gain, a.eps, a.dims, a.pairs, a.amplitude, a.turns, a.first, p.data, p.refs, p.table, p.len,
            p.n_pages, p.max_seqs, p.max_pages, p.n_layers, p.n_kv_heads);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & (LANES - 1), r0 = lane / LANES;
  const int units = a.n_q_heads + 2 * p.n_kv_heads;
  const int u = a.first + blockIdx.x * 4 + w;  // (a call has less than 2^29 waves)
  const int ib = u / units, unit = u - ib * units, i = ib / a.blocks, blk = ib - i * a.blocks;
  if (i >= a.n) return;
  const int p0 = ld_scalar(a.pos + i), s = ld_scalar(a.seqs + i);
  if (p0 < 0) return;
  const long long at8 = ((long long)p0 / 8 + blk) * 8;  // the block's first position
  if (at8 >= (long long)p0 + a.tokens) return;
  const int t0 = (int)(at8 - p0);                        // the token of its first row (negative: before the first)
  const int what = unit < a.n_q_heads ? 0 : unit < a.n_q_heads + p.n_kv_heads ? 1 : 2;  // queries, keys, values
  const int h = what == 0 ? unit : unit - a.n_q_heads - (what - 1) * p.n_kv_heads;

  // the rows, asked for before it is known whether they have a place
  const bf16_t* src = what == 0 ? a.q : what == 1 ? a.k : a.v;
  const long long stride = what == 0 ? a.q_stride : a.kv_stride;
  uint4 x16[STEPS];
  int place[STEPS];
#pragma unroll
  for (int y = 0; y < STEPS; ++y) {
    const int t = t0 + r0 + y * ROWS;
    const bool mine = t >= 0 && t < a.tokens;
    const size_t row = (size_t)i * a.tokens + (mine ? t : 0);
    x16[y] = mine ? *(const uint4*)(src + row * stride + (size_t)h * HD + 8 * c) : make_uint4(0, 0, 0, 0);
    place[y] = !mine ? -1 : a.places ? a.places[row] : (int)min((long long)p0 + t, 0x7fffffffLL);
  }

  // where K and V go
  bf16_t* tile = nullptr;
  int l = 0;
  if (what > 0) {
    const bool known = (unsigned)s < (unsigned)p.max_seqs;
    l = known ? ld_scalar(p.len + s) : -1;
    const long long j = at8 / kPage;
    int pg = known && j < p.max_pages ? ld_scalar(p.table + (size_t)s * p.max_pages + j) : -1;
    const bool fits = l >= 0 && l <= p.max_pages * kPage;
    const bool whole = fits && min(at8 + 8, (long long)p0 + a.tokens) <= l;  // (all of the block's tokens lie inside)
    if ((unsigned)pg >= (unsigned)p.n_pages || ld_scalar(p.refs + pg) != 1) pg = -1;
    if (lane == 0 && (pg < 0 || !whole)) report(p, PAGES_BAD_ENTRY);
    if (pg < 0 || !fits) return;
    tile = p.data + (size_t)pg * p.page() + ((size_t)a.layer * 2 * p.n_kv_heads + (what - 1) * p.n_kv_heads + h) * p.tile();
  }
  float* const mine_lds = meet[w];

  if (what == 2) {
    // [position][feature] in LDS, then a feature per lane
#pragma unroll
    for (int y = 0; y < STEPS; ++y)
      ((uint4*)mine_lds)[(r0 + y * ROWS) * LANES + c] = place[y] >= 0 ? x16[y] : make_uint4(0, 0, 0, 0);
    asm volatile("" ::: "memory");  // (read as another type below: the order is the wave's own, if the compiler keeps it)
    const bf16_t* rows = (const bf16_t*)mine_lds;
    const int from = max(-t0, 0), to = (int)min(min((long long)a.tokens - t0, l - at8), 8LL);  // rows that are stored
#pragma unroll
    for (int half = 0; half < HD / 64; ++half) {
      const int f = 64 * half + lane;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = rows[(4 * g + e) * HD + f];
        bf16_t* d = tile + (size_t)(f >> 5) * 1024 + (((int)at8 & 31) >> 4) * 512 + g * 256 + (f & 31) * 8 + (((int)at8 >> 3) & 1) * 4;
        if (from <= 4 * g && to >= 4 * g + 4) {
          *(uint2*)d = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * g + e >= from && 4 * g + e < to) d[e] = (bf16_t)y[e];
        }
      }
    }
    return;
  }

  const bf16_t* gain = what == 0 ? a.q_gain : a.k_gain;
  if (gain || a.dims > 0) {
    float g8[8];
    if (gain) {
      const uint4 x = *(const uint4*)(gain + 8 * c);
      widen<false>(x.x, g8[0], g8[1]);
      widen<false>(x.y, g8[2], g8[3]);
      widen<false>(x.z, g8[4], g8[5]);
      widen<false>(x.w, g8[6], g8[7]);
    }
    const int half = a.dims >> 1;
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      const int r = r0 + y * ROWS;
      float x[8];
      widen<F16>(x16[y].x, x[0], x[1]);
      widen<F16>(x16[y].y, x[2], x[3]);
      widen<F16>(x16[y].z, x[4], x[5]);
      widen<F16>(x16[y].w, x[6], x[7]);
      if (gain) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
        const float scale = rsqrtf(row_sum<LANES>(sum) * (1.f / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * scale * g8[e];
      }
      if (a.dims > 0) {
        float* row = mine_lds + r * HD;
        *(float4*)(row + 8 * c) = make_float4(x[0], x[1], x[2], x[3]);
        *(float4*)(row + 8 * c + 4) = make_float4(x[4], x[5], x[6], x[7]);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int f = 8 * c + e;
          if (f >= a.dims) continue;
          const bool second = a.pairs ? f & 1 : f >= half;
          const int pair = a.pairs ? f >> 1 : second ? f - half : f;
          const float other = row[a.pairs ? f ^ 1 : second ? f - half : f + half];
          const double turn = (double)place[y] * a.turns[pair];
          const float part = (float)(turn - floor(turn));
          const float co = __builtin_amdgcn_cosf(part) * a.amplitude, si = __builtin_amdgcn_sinf(part) * a.amplitude;
          x[e] = second ? fmaf(x[e], co, other * si) : fmaf(x[e], co, -(other * si));
        }
      }
      x16[y] = make_uint4(narrow2<F16>(x[0], x[1]), narrow2<F16>(x[2], x[3]), narrow2<F16>(x[4], x[5]), narrow2<F16>(x[6], x[7]));
    }
  }
#pragma unroll
  for (int y = 0; y < STEPS; ++y) {
    const int r = r0 + y * ROWS, t = t0 + r;
    if (t < 0 || t >= a.tokens) continue;
    const uint4 x = place[y] >= 0 ? x16[y] : make_uint4(0, 0, 0, 0);
    if (what == 0) *(uint4*)(a.q_out + ((size_t)i * a.tokens + t) * a.q_out_stride + (size_t)h * HD + 8 * c) = x;
    else if (at8 + r < l) *(uint4*)(tile + (size_t)(c >> 1) * 512 + (c & 1) * 256 + (((int)at8 & 31) + r) * 8) = x;
  }
}

__global__ __launch_bounds__(64) void rotary_fill_kernel(int dims, double base, double factor, double original, double low,
                                                         double high, double* __restrict__ turns) {
  const int f = threadIdx.x;
  if (f >= dims / 2) return;
  const double w = pow(base, -2.0 * f / dims) * 0.15915494309189533577;  // 1 / (2 pi)
  const double r = original * w;
  double keep = 0.0;
  if (original > 0.0) keep = r <= low ? 0.0 : r >= high ? 1.0 : (r - low) / (high - low);
  turns[f] = w * (keep + (1.0 - keep) / factor);
}

}  // namespace

extern "C" {

int vlac_rotary_fill(int dims, double base, double factor, double original, double low, double high, double* turns, void* stream) {
  if (dims < 2 || dims > 128 || dims % 2) return VLAC_E_SHAPE;
  if (!std::isfinite(base) || !std::isfinite(factor) || !std::isfinite(original) || !std::isfinite(low) || !std::isfinite(high) ||
      base <= 1.0 || factor < 1.0 || original < 0.0 || low < 0.0 || low >= high)
    return VLAC_E_RANGE;
  if (!turns) return VLAC_E_NULL;
  if ((uintptr_t)turns % 8) return VLAC_E_SHAPE;
  hipLaunchKernelGGL(rotary_fill_kernel, dim3(1), dim3(64), 0, (hipStream_t)stream, dims, base, factor, original, low, high, turns);
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

int vlac_pages_append_rotated(const vlac_pages* pages, int layer, const int32_t* seqs, const int32_t* pos, int n, int tokens,
                              const vlac_rotary* rot, const int32_t* places, int n_q_heads, const void* q, int64_t q_stride,
                              const void* k, const void* v, int64_t kv_stride, void* q_out, int64_t q_out_stride,
                              const void* q_gain, const void* k_gain, float eps, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc != VLAC_OK) return rc;
  if (n < 0 || n > VLAC_PAGES_MAX_LIST || layer < 0 || layer >= pages->n_layers || tokens < 1 || (long long)n * tokens > 1 << 20 ||
      n_q_heads < 0 || n_q_heads > 1024)
    return VLAC_E_RANGE;
  const int64_t q_width = (int64_t)n_q_heads * pages->head_dim, kv_width = (int64_t)pages->n_kv_heads * pages->head_dim;
  if (kv_stride < kv_width || kv_stride % 8 || kv_stride > 1 << 30) return VLAC_E_SHAPE;
  if (n_q_heads > 0 && (q_stride < q_width || q_stride % 8 || q_stride > 1 << 30 || q_out_stride < q_width || q_out_stride % 8 ||
                        q_out_stride > 1 << 30 || (q == q_out && q_stride != q_out_stride)))
    return VLAC_E_SHAPE;
  if (rot) {
    if (rot->dims < 2 || rot->dims > pages->head_dim || rot->dims % 2) return VLAC_E_SHAPE;
    if ((rot->layout != VLAC_ROTARY_HALF && rot->layout != VLAC_ROTARY_PAIRS) || !std::isfinite(rot->amplitude)) return VLAC_E_RANGE;
    if (!rot->turns) return VLAC_E_NULL;
    if ((uintptr_t)rot->turns % 8) return VLAC_E_SHAPE;
  }
  if ((q_gain || k_gain) && !(std::isfinite(eps) && eps >= 0.f)) return VLAC_E_RANGE;
  if (n == 0) return VLAC_OK;
  if (!seqs || !pos || !k || !v || (n_q_heads > 0 && (!q || !q_out))) return VLAC_E_NULL;
  if ((uintptr_t)k % 16 || (uintptr_t)v % 16 || (uintptr_t)q_gain % 16 || (uintptr_t)k_gain % 16 ||
      (n_q_heads > 0 && ((uintptr_t)q % 16 || (uintptr_t)q_out % 16)))
    return VLAC_E_SHAPE;
  RotaryArgs a = {pool_view(pages), layer, n, tokens, (tokens + 14) / 8, seqs, pos, places, n_q_heads, (const bf16_t*)q, (const bf16_t*)k,
                  (const bf16_t*)v, q_stride, kv_stride, (bf16_t*)q_out, q_out_stride, (const bf16_t*)q_gain, (const bf16_t*)k_gain, eps,
                  rot ? rot->dims : 0, rot ? rot->layout == VLAC_ROTARY_PAIRS : 0, rot ? rot->amplitude : 1.f,
                  rot ? rot->turns : nullptr, 0};
  const long long waves = (long long)n * a.blocks * (n_q_heads + 2 * pages->n_kv_heads);
  // (a launch of 2^32 threads and more would run only what is left of them modulo 2^32)
  constexpr int kMost = 1 << 24;
  hipStream_t st = (hipStream_t)stream;
  for (a.first = 0; a.first < waves; a.first += kMost) {
    const dim3 grid((unsigned)((std::min<long long>(waves - a.first, kMost) + 3) / 4));
    if (pages->head_dim == 128) {
      if (pages_f16(pages)) hipLaunchKernelGGL((rotary_append_kernel<128, true>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((rotary_append_kernel<128, false>), grid, dim3(256), 0, st, a);
    } else {
      if (pages_f16(pages)) hipLaunchKernelGGL((rotary_append_kernel<64, true>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((rotary_append_kernel<64, false>), grid, dim3(256), 0, st, a);
    }
  }
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
