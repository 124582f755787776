// Queries, keys and values of new tokens on their way into the pages: the norm of every head and the rotation of its position
// in the same pass,
//   q' = R(place) N(q), k' = R(place) N(k), v' = v,   N(x) = x rsqrt(mean x^2 + eps) gain,
//   R turns pair f by 2 pi turns[f] place.
// Norm and rotation in fp32, rounded once.  The turn is worked out in 64 bits and its fraction rounded to 32 (which lose it
// at far places otherwise); the chip's sine and cosine of a fraction of a turn are off by 1.3e-7 at most, a 3000th of
// a half step of fp16 of the larger value.
//
// Bound by latency up to some MB (arguments - position and sequence - rows, page and table of turns - stores: one token of
// two sequences 3.1 us, 8 x 31 tokens of 32 heads of 128, 12 MB, 7.4), then by memory: 1024 tokens of 32 heads (50 MB read and written) 12.0
// us, 4096 49, 4.1 TB/s.  Whole rows of a head would be longer pieces than a wave's, but a page stores K by 8 features of 32 positions and V
// by 8 positions of a feature, so a wave takes 8 positions of queries and keys, and 16 of values: a line of K, or a word of
// every feature, is written at once.  (V by 8 positions through LDS: 9.2 us instead of 7.4; its last rows by single values
// instead of four at a time: 16 x 64 tokens of 32 heads 23 us instead of 15.)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pages.h"

namespace {

struct RotaryArgs {
  PoolView p;
  int layer, n, tokens;
  const int *seqs, *pos, *places;
  int n_q_heads;
  const bf16_t *q, *k, *v;
  long long q_stride, kv_stride;
  bf16_t* q_out;
  long long q_out_stride;
  const bf16_t *q_gain, *k_gain;
  float eps;
  int dims;  // rotated features (0: none)
  float amplitude;
  const double* turns;
  int first;  // wave of the call that this launch begins with
  // a wave takes up to G heads: of queries and keys (the first qk_waves waves of an entry, in qk_groups groups per block of 8
  // positions), or of values (v_waves, v_groups per block of 16)
  int qk_groups, v_groups, qk_waves, v_waves;
};
enum Turning { COPY, PAIRS, HALVES, ANY_HALVES };  // (HALVES: dims / 2 is a multiple of 8, so that a lane's 8 partners are another lane's)

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

// Sum over the GROUP lanes (8 or 16, aligned) that share a row, by moves inside the vector ALU: neighbours, pairs of them, the other
// quads of a half row (mirrored), the other half (mirrored)
template <int HOW>
__device__ inline float moved(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), HOW, 0xf, 0xf, true));
}
template <int GROUP>
__device__ inline float row_sum(float x) {
  x += moved<0xb1>(x);    // (quad: 1 0 3 2)
  x += moved<0x4e>(x);    // (quad: 2 3 0 1)
  x += moved<0x141>(x);   // (half row mirrored)
  if constexpr (GROUP == 16) x += moved<0x140>(x);  // (row mirrored)
  return x;
}

// A store of 16 bytes, non-temporal in large calls: with 2 heads of 128 or more to a wave, 1024 tokens of 32 heads 15.1 -> 12.0 us, 4
// x 1057 of 12 on 2 12.5 -> 11.0, 32 x 2 tokens' equal.  (V's stores marked so as well: 17 us.)
template <bool STREAM>
__device__ inline void put(bf16_t* to, const uint4& x) {
  if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4*)to);
  else *(uint4*)to = x;
}

// Where the tokens of an entry lie that a wave takes: rows from .. to - 1 of the block of positions that begins at `at`, the first of them
// token t0 + from; and the page, if they may be stored there (rows before `last` lie inside the sequence).
struct Block {
  int i, seq, t0, from, to, last;
  long long at;
  bf16_t* page;  // of the layer
};
// The block blk of `size` positions of entry i: false if no token lies in it
__device__ inline bool block_of(const RotaryArgs& a, int i, int blk, int size, Block& b) {
  const int p0 = ld_scalar(a.pos + i);
  b.i = i;
  b.seq = ld_scalar(a.seqs + i);
  b.at = ((long long)p0 / size + blk) * size;
  if (p0 < 0 || b.at >= (long long)p0 + a.tokens) return false;
  b.t0 = (int)(b.at - p0);
  b.from = max(-b.t0, 0);
  b.to = min(a.tokens - b.t0, size);
  return true;
}
__device__ inline void find_page(const RotaryArgs& a, Block& b, int size, int lane) {
  const PoolView& p = a.p;
  const bool known = (unsigned)b.seq < (unsigned)p.max_seqs;
  const int l = known ? ld_scalar(p.len + b.seq) : -1;
  const long long j = b.at / kPage;
  int pg = known && j < p.max_pages ? ld_scalar(p.table + (size_t)b.seq * p.max_pages + j) : -1;
  const bool fits = l >= 0 && l <= p.max_pages * kPage;
  if ((unsigned)pg >= (unsigned)p.n_pages || ld_scalar(p.refs + pg) != 1) pg = -1;
  if (lane == 0 && (pg < 0 || !fits || b.at + b.to > l)) report(p, PAGES_BAD_ENTRY);
  b.page = pg >= 0 && fits ? p.data + (size_t)pg * p.page() + (size_t)a.layer * 2 * p.n_kv_heads * p.tile() : nullptr;
  b.last = fits ? (int)min(l - b.at, (long long)size) : 0;
}

// Values: 16 positions, whose words of a page (8 of them, of one feature) a wave has together.  A lane loads 8 features of a
// row and changes places with the lanes 16, 32 and 48 further, which have them of the next three rows: two swaps of registers between
// halves and two between quarters of the wave transpose 4 x 4 words, without LDS.
template <int HD, int G>
__device__ inline void value_rows(const RotaryArgs& a, Block& b, int group, int lane) {
  constexpr int LANES = HD / 8, SIDE = 16 / LANES, STEPS = 4 / SIDE;  // groups of 4 rows side by side, and behind one another
  const PoolView& p = a.p;
  const int c = lane & (LANES - 1), side = (lane & 15) / LANES, e4 = lane >> 4, hkv = p.n_kv_heads;
  const int h0 = group * G;
  size_t row[STEPS];
  bool mine[STEPS];
#pragma unroll
  for (int y = 0; y < STEPS; ++y) {
    const int r = 4 * (y * SIDE + side) + e4;
    mine[y] = r >= b.from && r < b.to;
    row[y] = (size_t)b.i * a.tokens + (mine[y] ? b.t0 + r : 0);
  }
  auto load = [&](uint4(&x)[STEPS], int h) {
#pragma unroll
    for (int y = 0; y < STEPS; ++y)
      x[y] = mine[y] ? *(const uint4*)(a.v + row[y] * a.kv_stride + (size_t)h * HD + 8 * c) : make_uint4(0, 0, 0, 0);
  };
  uint4 all[G][STEPS];
#pragma unroll
  for (int k = 0; k < G; ++k) load(all[k], min(h0 + k, hkv - 1));
  bool gone[STEPS];  // (rows that are not there are zeros)
#pragma unroll
  for (int y = 0; y < STEPS; ++y) gone[y] = a.places && mine[y] && a.places[row[y]] < 0;
  find_page(a, b, 16, lane);
  if (!b.page) return;
  const int end = min(b.to, b.last), r16 = ((int)b.at & 31) >> 4;
#pragma unroll
  for (int head = 0; head < G; ++head) {
    const int h = h0 + head;
    if (h >= hkv) break;
    const uint4(&x)[STEPS] = all[head];
    uint2 out[STEPS][2];  // the two features of this lane: the group's 4 rows
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      uint32_t w0 = gone[y] ? 0u : x[y].x, w1 = gone[y] ? 0u : x[y].y, w2 = gone[y] ? 0u : x[y].z, w3 = gone[y] ? 0u : x[y].w;
      // word k of row r (the lane's quarter) -> word r of quarter k
      auto s = __builtin_amdgcn_permlane32_swap(w0, w2, false, false);
      w0 = s[0]; w2 = s[1];
      s = __builtin_amdgcn_permlane32_swap(w1, w3, false, false);
      w1 = s[0]; w3 = s[1];
      s = __builtin_amdgcn_permlane16_swap(w0, w1, false, false);
      w0 = s[0]; w1 = s[1];
      s = __builtin_amdgcn_permlane16_swap(w2, w3, false, false);
      w2 = s[0]; w3 = s[1];
      out[y][0] = make_uint2((w0 & 0xffffu) | w1 << 16, (w2 & 0xffffu) | w3 << 16);
      out[y][1] = make_uint2(w0 >> 16 | (w1 & 0xffff0000u), w2 >> 16 | (w3 & 0xffff0000u));
    }
    bf16_t* const tile = b.page + ((size_t)hkv + h) * p.tile() + r16 * 512;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int f = 8 * c + 2 * e4 + k;
      bf16_t* const at = tile + (size_t)(f >> 5) * 1024 + (f & 31) * 8;
#pragma unroll
      for (int y = 0; y < STEPS / 2; ++y) {
        // rows r .. r + 3 and r + 8 .. r + 11 make up a word
        const int four = y * SIDE + side, r = 4 * four;
        bf16_t* const d = at + four * 256;
        const uint2 lo = out[y][k], hi = out[y + STEPS / 2][k];
        if (r >= b.from && r + 12 <= end) {
          *(uint4*)d = make_uint4(lo.x, lo.y, hi.x, hi.y);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint2 four_rows = i ? hi : lo;
            const int r4 = r + 8 * i;
            if (r4 >= b.from && r4 + 4 <= end) {
              *(uint2*)(d + 4 * i) = four_rows;
            } else if (r4 + 4 > b.from && r4 < end) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (r4 + e >= b.from && r4 + e < end) d[4 * i + e] = (bf16_t)((e < 2 ? four_rows.x : four_rows.y) >> (16 * (e & 1)));
            }
          }
        }
      }
    }
  }
}

// Queries and keys: 8 positions that lie side by side in a page (one page to look up, and a K store of 8 rows is a line) and one or
// more heads there: the angles are worked out once for all of them.  A lane holds 8 features of a row, so head_dim / 8 lanes
// hold a row.
template <int HD, bool F16, int TURN, int G>
__device__ inline void query_key_rows(const RotaryArgs& a, Block& b, int group, int lane, float* meet) {
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, STEPS = 8 / ROWS;  // rows at a time
  constexpr int ANGLES = TURN == COPY ? 1 : TURN == PAIRS ? 4 : 8;
  const PoolView& p = a.p;
  const int c = lane & (LANES - 1), r0 = lane / LANES;
  const int units = a.n_q_heads + p.n_kv_heads, unit0 = group * G;
  size_t row[STEPS];
  bool mine[STEPS];
#pragma unroll
  for (int y = 0; y < STEPS; ++y) {
    const int r = r0 + y * ROWS;
    mine[y] = r >= b.from && r < b.to;
    row[y] = (size_t)b.i * a.tokens + (mine[y] ? b.t0 + r : 0);
  }
  auto load = [&](uint4(&x)[STEPS], int unit) {
    const bool is_q = unit < a.n_q_heads;
    const bf16_t* src = (is_q ? a.q : a.k) + (size_t)(is_q ? unit : unit - a.n_q_heads) * HD + 8 * c;
    const long long stride = is_q ? a.q_stride : a.kv_stride;
#pragma unroll
    for (int y = 0; y < STEPS; ++y) x[y] = mine[y] ? *(const uint4*)(src + row[y] * stride) : make_uint4(0, 0, 0, 0);
  };
  // everything that has an address already is asked for first
  uint4 all[G][STEPS];
#pragma unroll
  for (int k = 0; k < G; ++k) load(all[k], min(unit0 + k, units - 1));
  const int half = a.dims >> 1;
  double turns[ANGLES];
  if constexpr (TURN != COPY) {
#pragma unroll
    for (int e = 0; e < ANGLES; ++e) {
      const int f = TURN == PAIRS ? 8 * c + 2 * e : 8 * c + e, pair = TURN == PAIRS ? f >> 1 : f >= half ? f - half : f;
      turns[e] = a.turns[f < a.dims ? pair : 0];
    }
  }
  int place[STEPS];
#pragma unroll
  for (int y = 0; y < STEPS; ++y)
    place[y] = !mine[y] ? -1 : a.places ? a.places[row[y]] : (int)min(b.at + r0 + y * ROWS, 0x7fffffffLL);
  b.page = nullptr;
  b.last = 0;
  if (min(unit0 + G, units) > a.n_q_heads) find_page(a, b, 8, lane);

  // the angles of this lane's rows and features
  float co[STEPS][ANGLES], si[STEPS][ANGLES];
  if constexpr (TURN != COPY) {
#pragma unroll
    for (int y = 0; y < STEPS; ++y)
#pragma unroll
      for (int e = 0; e < ANGLES; ++e) {
        const float part = (float)__builtin_amdgcn_fract((double)place[y] * turns[e]);
        co[y][e] = __builtin_amdgcn_cosf(part) * a.amplitude;
        si[y][e] = __builtin_amdgcn_sinf(part) * a.amplitude;
        // the second of a pair turns the other way
        if (TURN != PAIRS && 8 * c + e < half) si[y][e] = -si[y][e];
      }
  }

#pragma unroll
  for (int head = 0; head < G; ++head) {
    const int unit = unit0 + head;
    if (unit >= units) break;
    uint4(&x16)[STEPS] = all[head];
    const bool is_q = unit < a.n_q_heads;
    const int h = is_q ? unit : unit - a.n_q_heads;
    const bf16_t* gain = is_q ? a.q_gain : a.k_gain;
    if (TURN != COPY || gain) {
      float g8[8];
      if (gain) {
        const uint4 x = *(const uint4*)(gain + 8 * c);
        widen<false>(x.x, g8[0], g8[1]);
        widen<false>(x.y, g8[2], g8[3]);
        widen<false>(x.z, g8[4], g8[5]);
        widen<false>(x.w, g8[6], g8[7]);
      }
#pragma unroll
      for (int y = 0; y < STEPS; ++y) {
        float x[8];
        widen<F16>(x16[y].x, x[0], x[1]);
        widen<F16>(x16[y].y, x[2], x[3]);
        widen<F16>(x16[y].z, x[4], x[5]);
        widen<F16>(x16[y].w, x[6], x[7]);
        if (gain) {
          auto mean_of_squares = [&] {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
            return row_sum<LANES>(sum) * (1.f / HD);
          };
          float mean = mean_of_squares() + a.eps;
          if constexpr (!F16) {
            // Squares of bf16 leave fp32's range at both ends: once more for such a row, brought nearer to 1 by a power of two
            // (which all lanes of the row do, and which the quotient does not see)
            if (__builtin_expect(mean == INFINITY || mean < 0x1p-100f, 0)) {
              const float nearer = mean == INFINITY ? 0x1p-70f : 0x1p70f;
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] *= nearer;
              mean = mean_of_squares() + a.eps * nearer * nearer;
            }
          }
          const float scale = rsqrtf(mean);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * scale * g8[e];
        }
        if constexpr (TURN == PAIRS) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (8 * c + 2 * e < a.dims) {
              const float x0 = x[2 * e], x1 = x[2 * e + 1];
              x[2 * e] = fmaf(x0, co[y][e], -(x1 * si[y][e]));
              x[2 * e + 1] = fmaf(x1, co[y][e], x0 * si[y][e]);
            }
        } else if constexpr (TURN == HALVES) {
          const int partner = lane + (8 * c < half ? half >> 3 : -(half >> 3));  // (of lanes beyond the rotated ones: nobody looks)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float other = __shfl(x[e], partner);
            if (8 * c < a.dims) x[e] = fmaf(x[e], co[y][e], other * si[y][e]);
          }
        } else if constexpr (TURN == ANY_HALVES) {
          float* const row32 = meet + (r0 + y * ROWS) * HD;
          *(float4*)(row32 + 8 * c) = make_float4(x[0], x[1], x[2], x[3]);
          *(float4*)(row32 + 8 * c + 4) = make_float4(x[4], x[5], x[6], x[7]);
          asm volatile("" ::: "memory");  // (the order is the wave's own, if the compiler keeps it)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int f = 8 * c + e;
            if (f < a.dims) x[e] = fmaf(x[e], co[y][e], row32[f < half ? f + half : f - half] * si[y][e]);
          }
          asm volatile("" ::: "memory");
        }
        x16[y] = make_uint4(narrow2<F16>(x[0], x[1]), narrow2<F16>(x[2], x[3]), narrow2<F16>(x[4], x[5]), narrow2<F16>(x[6], x[7]));
      }
    }
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      if (!mine[y]) continue;
      const int r = r0 + y * ROWS;
      const uint4 x = place[y] >= 0 ? x16[y] : make_uint4(0, 0, 0, 0);
      if (is_q) put<(G > 1)>(a.q_out + row[y] * a.q_out_stride + (size_t)h * HD + 8 * c, x);
      else if (b.page && r < b.last) put<(G > 1)>(b.page + h * p.tile() + (size_t)(c >> 1) * 512 + (c & 1) * 256 + (((int)b.at & 31) + r) * 8, x);
    }
  }
}

template <int HD, bool F16, int TURN, int G>
__global__ __launch_bounds__(256, 4) void rotary_append_kernel(RotaryArgs a) {
  __shared__ float4 meet[4][TURN == ANY_HALVES ? 8 * HD / 4 : 1];  // (the partners of a pair, where they are in no one lane)
  const PoolView& p = a.p;
  read_args(a.layer, a.n, a.tokens, a.seqs, a.pos, a.places, a.n_q_heads, a.q, a.k, a.v, a.q_stride, a.kv_stride, a.q_out,
            a.q_out_stride, a.q_gain, a.k_gain, a.eps, a.dims, a.amplitude, a.turns, a.first, a.qk_groups, a.v_groups, a.qk_waves,
            a.v_waves, p.data, p.refs, p.table, p.len, p.n_pages, p.max_seqs, p.max_pages, p.n_layers, p.n_kv_heads);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = a.first + blockIdx.x * 4 + w, per_entry = a.qk_waves + a.v_waves;  // (a call has less than 2^29 waves)
  const int i = u / per_entry, k = u - i * per_entry;
  if (i >= a.n) return;
  Block b;
  if (k < a.qk_waves) {
    const int blk = k / a.qk_groups;
    if (block_of(a, i, blk, 8, b)) query_key_rows<HD, F16, TURN, G>(a, b, k - blk * a.qk_groups, lane, (float*)meet[w]);
  } else {
    const int blk = (k - a.qk_waves) / a.v_groups;
    if (block_of(a, i, blk, 16, b)) value_rows<HD, G>(a, b, k - a.qk_waves - blk * a.v_groups, lane);
  }
}

// Waves that a call should have before they take more than one head each (8 per CU), us per layer with this many, half and twice
// as many: 8 x 31 tokens of 32 heads 7.4, 10.0, 7.4; 4 x 1057 of 12 on 2 11.0, 13.0, 12.5; 64 x 1 of 32 6.8, 8.2, 7.4.
constexpr int kWavesWanted = 2048;

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
  RotaryArgs a = {pool_view(pages), layer, n, tokens, seqs, pos, places, n_q_heads, (const bf16_t*)q, (const bf16_t*)k,
                  (const bf16_t*)v, q_stride, kv_stride, (bf16_t*)q_out, q_out_stride, (const bf16_t*)q_gain, (const bf16_t*)k_gain, eps,
                  rot ? rot->dims : 0, rot ? rot->amplitude : 1.f, rot ? rot->turns : nullptr, 0, 0, 0, 0, 0};
  const int qk = n_q_heads + pages->n_kv_heads, blocks8 = (tokens + 14) / 8, blocks16 = (tokens + 30) / 16;
  const long long work = (long long)n * blocks8 * qk;
  const int per_wave = work >= 4 * kWavesWanted ? 4 : work >= 2 * kWavesWanted ? 2 : 1;
  a.qk_groups = (qk + per_wave - 1) / per_wave;
  a.v_groups = (pages->n_kv_heads + per_wave - 1) / per_wave;
  a.qk_waves = blocks8 * a.qk_groups;
  a.v_waves = blocks16 * a.v_groups;
  const long long waves = (long long)n * (a.qk_waves + a.v_waves);
  const int turn = !rot ? COPY : rot->layout == VLAC_ROTARY_PAIRS ? PAIRS : rot->dims % 16 == 0 ? HALVES : ANY_HALVES;
  hipStream_t st = (hipStream_t)stream;
  // (a launch of 2^32 threads and more would run only what is left of them modulo 2^32)
  constexpr int kMost = 1 << 24;
  for (a.first = 0; a.first < waves; a.first += kMost) {
    const dim3 grid((unsigned)((std::min<long long>(waves - a.first, kMost) + 3) / 4));
    auto launch = [&](auto hd, auto f16, auto how, auto heads) {
      hipLaunchKernelGGL((rotary_append_kernel<decltype(hd)::value, decltype(f16)::value, decltype(how)::value, decltype(heads)::value>), grid,
                         dim3(256), 0, st, a);
    };
    auto by_heads = [&](auto hd, auto f16, auto how) {
      if (per_wave == 4) launch(hd, f16, how, std::integral_constant<int, 4>{});
      else if (per_wave == 2) launch(hd, f16, how, std::integral_constant<int, 2>{});
      else launch(hd, f16, how, std::integral_constant<int, 1>{});
    };
    auto by_turn = [&](auto hd, auto f16) {
      if (turn == COPY) by_heads(hd, f16, std::integral_constant<int, COPY>{});
      else if (turn == PAIRS) by_heads(hd, f16, std::integral_constant<int, PAIRS>{});
      else if (turn == HALVES) by_heads(hd, f16, std::integral_constant<int, HALVES>{});
      else by_heads(hd, f16, std::integral_constant<int, ANY_HALVES>{});
    };
    auto typed = [&](auto hd) {
      if (pages_f16(pages)) by_turn(hd, std::true_type{});
      else by_turn(hd, std::false_type{});
    };
    if (pages->head_dim == 128) typed(std::integral_constant<int, 128>{});
    else typed(std::integral_constant<int, 64>{});
  }
  return hipGetLastError() == hipSuccess ? VLAC_OK : VLAC_E_HIP;
}

}  // extern "C"
