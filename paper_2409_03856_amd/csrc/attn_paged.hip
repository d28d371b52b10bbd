// Attention over the paged cache, on gfx950.
//
// Token i of sequence b stands at cache row p + i (p = cache_pos[b]); its H query heads read key/value
// head h / G (G = H / Hkv) of rows 0 .. p + i, less what a window or a mask of the chunk hides:
//   s_j = scale q . k_j, capped (cap tanh(s / cap)), less slope (p + i - j);  out = sum_j softmax(s)_j v_j.
// The G n query rows of a sequence that share a key/value head (r = i G + h % G) are processed together.
//
// The rows of a call are cut into units (a sequence, a range of its visible rows) on the device, where
// the lengths are: units are as long as makes about kTargetWgs workgroups of equal work, so ragged
// batches stay balanced. A sequence of one unit is written out directly; the others leave (max, sum,
// output) per unit and row, and attn_paged_merge_kernel joins them in order.
//
// attn_rows_kernel: up to 16 query rows per workgroup, four waves that take every fourth tile of
// 32 positions each and are merged at the end. Scores are K Q^T on the matrix units, whose result (a lane
// holds one query row and, by the order in which key rows are dealt to the operand's rows, eight
// consecutive positions) is the operand of V^T P^T as it is. Keys lie row by row and values column by
// column in the cache, so that both operands are 16-byte loads straight into registers, one tile ahead in
// flight: LDS holds the page entries of 4096 positions, staged behind a barrier, and the pieces of fp32 queries, and
// no tile waits for another wave. fp32 queries and their probabilities go in as three
// bf16 pieces that hold every bit; bf16 ones in one piece and probabilities in two.
// Bound: HBM. 48 sequences of up to 30000 rows, 32 / 8 heads of 128, bf16: 350 us for 1.85 GB of keys and values,
// 5.3 TB/s (a plain read's rate here); fp32 queries 365 us. One token over 2048 rows: 9.8 us, a chain of launch,
// plan, page entries, one tile, and the waves' joining; its merge 5.
//
// attn_tiles_kernel: more rows, in tiles of LDS that four waves share (below).
// Bound: the matrix units and the vector instructions between their products, which two waves of a SIMD only
// partly overlap. Prompts of 4500 and 1124 tokens, bf16: 206 us, 855 TFLOP/s (a large library product reaches
// 1140 to 1360), matrix units busy 41 % at the clock that a counter run keeps; the same with fp32 queries, three products
// for one, 590 us, 299 TFLOP/s; eight trees of 40 nodes over 6000
// rows, fp32, capped: 155 us and the merge 9, matrix units busy 25 % (six products a tile, then 48 exponentials' and
// pieces' instructions a lane). Row groups and cuts are made for max_n tokens of every sequence: beside a long prompt a
// decoded token is one workgroup's per head, from its first row to its last (a prompt of 4096 tokens and 32 tokens over up to
// 30000 rows, bf16: 1086 us in one call, 178 and 293 in two).
#include <float.h>
#include <math.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "paged.h"
#include "profile.h"

namespace sirius {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4_t;

typedef unsigned long long u64;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = kPlanTile;    // positions per wave step
constexpr int kStep = kPlanStep;
static_assert(kStep == kTile * kWaves, "a step is a tile of each wave");
constexpr int kTargetWgs = 512;     // workgroups wanted: two per CU, what their registers allow
constexpr int kMaxUnits = 256;      // units of a round at most
constexpr int kGroups = 512;        // 8-position groups whose pages are staged at a time

struct Args {
  PagedView pg;
  const void* q;
  long ldq;
  int H, Hkv, hd, G, rgroups, units, rounds;  // units: ranges of a round (1: every sequence whole); rounds: 1 or 2
  float scale, cap;
  const float* slopes;
  int window;
  const uint64_t* mask;
  void* out;
  float* pm;
  float* pl;
  float* po;
  int2* info;  // [B]: first slot of the partials, units
};

__device__ __forceinline__ uint32_t high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float rest(float x) {  // less its truncation to bf16; 0 for infinities
  const float h = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  return h == x ? 0.f : x - h;
}
__device__ __forceinline__ float rest_finite(float x) {
  return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}

// e^x for x <= 4 to about one ulp: exp2 of the rounded x log2(e), times the first order of what the
// rounding left off. Below -200 (hidden: -inf) 0; a NaN stays one.
__device__ __forceinline__ float exp_neg(float x) {
  constexpr float kHi = 1.44269502162933349609375f, kLo = 1.9259629911e-8f, kLn2 = 0.693147180559945f;
  x = __builtin_elementwise_maximum(x, -200.f);
  const float t = x * kHi;
  const float d = fmaf(x, kLo, fmaf(x, kHi, -t));
  return __builtin_amdgcn_exp2f(t) * fmaf(d, kLn2, 1.f);
}

// cap tanh(x / cap) as x (1 - y^2 / 3 + ..), y = x / cap: the series of tanh, whose next term is 1e-8 at 0.35.
__device__ __forceinline__ float cap_near(float x, float inv) {
  const float y = x * inv, z = y * y;
  return x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -8.86323553e-3f, 2.18694885e-2f), -5.39682540e-2f), 0.133333333f), -0.333333333f), 1.f);
}
// The same anywhere: beyond 0.35 cap 1 - 2 / (e^2y + 1).
__device__ __forceinline__ float capped(float x, float cap, float inv) {
  const float y = x * inv, a = fabsf(y);
  const float far = cap * copysignf(1.f - 2.f / (__builtin_amdgcn_exp2f(fminf(a, 40.f) * 2.88539008f) + 1.f), y);
  return a > 0.35f ? far : cap_near(x, inv);
}

// A workgroup's share: positions [c0, c1) of sequence b, whose first seen row is lo.
struct Unit {
  int b, c0, c1, lo, slot, count, part;  // unit `part` of the sequence's `count`; slot: of its first partial
  int first, n, p;                 // its tokens, its position
};

// Rows that a sequence's tokens see: from the first token's window to the last token, from a tile's start.
__device__ __forceinline__ int first_seen(const Args& a, int p) {
  return a.window > 0 ? max(0, p + 1 - a.window) : 0;
}
__device__ __forceinline__ bool valid(const Args& a, int p, int n) { return n <= a.pg.n && rows_fit(a.pg, p, n); }

__device__ __forceinline__ int span_of(const Args& a, int b) {
  const int n = tokens_of(a.pg, b).y, p = a.pg.pos[b];
  if (n == 0) return 0;
  if (!valid(a, p, n)) return 1;
  return p + n - (first_seen(a, p) & ~(kTile - 1));
}

__device__ __forceinline__ int wave_add(int v) {
  for (int m = 1; m < kWave; m <<= 1) v += __shfl_xor(v, m, kWave);
  return v;
}

// How the call's sequences are cut. Every workgroup counts for itself, one sequence per lane.
struct Plan {
  int every;          // rows per unit at most
  int span, cnt;      // up to 64 sequences: this lane's
  int ic, is;         // and the units and the partial slots up to its end
};

// Inclusive sums over the wave.
__device__ __forceinline__ void scan2(int lane, int& a, int& b) {
  for (int o = 1; o < kWave; o <<= 1) {
    const int c = __shfl_up(a, o, kWave), d = __shfl_up(b, o, kWave);
    if (lane >= o) {
      a += c;
      b += d;
    }
  }
}

// Up to 64 sequences every wave plans alone; more take the whole workgroup, 256 at a time.
__device__ __forceinline__ Plan make_plan(const Args& a) {
  constexpr int kOvh = 256;  // what a unit costs besides its rows, in rows
  __shared__ int s_w[kWaves];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, B = a.pg.B;
  Plan p{1 << 30, 0, 0, 0, 0};
  if (a.units <= 1) return p;
  if (B > kWave) {
    long total = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
      // spans are at most 2^20: a block's sum fits an int
      const int s = wave_add(b0 + tid < B ? span_of(a, b0 + tid) : 0);
      if (lane == 0) s_w[wave] = s;
      __syncthreads();
      total += (long)s_w[0] + s_w[1] + s_w[2] + s_w[3];
      __syncthreads();
    }
    p.every = whole_steps((total + a.units * a.rounds - 1) / (a.units * a.rounds));
    return p;
  }
  p.span = lane < B ? span_of(a, lane) : 0;
  const int total = wave_add(p.span);
  p.every = whole_steps((total + a.units - 1) / a.units);
  if (a.rounds > 1 && B > 1) {
    // One or two rounds of a.units units of equal length, or as many units for every sequence as one
    // round has room for: what ends first. 8 sequences of 6000 rows in 21 units go by two each, not by three
    // in 24 (213 -> 181 us).
    int most = p.span;
    for (int m = 1; m < kWave; m <<= 1) most = max(most, __shfl_xor(most, m, kWave));
    const int half = whole_steps((total + 2 * a.units - 1) / (2 * a.units));
    const int one = wave_add(units_of(p.span, p.every)), two = wave_add(units_of(p.span, half));
    auto cost = [&](int units, int rows) { return (units + a.units - 1) / a.units * (rows + kOvh); };
    int best = cost(one, p.every);
    if (cost(two, half) < best) {
      best = cost(two, half);
      p.every = half;
    }
    const int fit = B <= a.units ? whole_steps((most + a.units / B - 1) / (a.units / B)) : INT32_MAX / 2;
    if (fit + kOvh < best) p.every = fit;
  }
  p.cnt = units_of(p.span, p.every);
  p.ic = p.cnt;
  p.is = p.cnt > 1 ? p.cnt : 0;
  scan2(lane, p.ic, p.is);
  return p;
}

// The unit with this number, b = -1 behind the last.
__device__ __forceinline__ Unit unit_at(const Args& a, const Plan& p, int number) {
  __shared__ int s_w[2][kWaves];
  __shared__ int s_hit[5];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int B = a.pg.B;
  Unit u{};
  int length = 1 << 30;  // rows per unit
  auto cut = [&](int span, int count) { return whole_steps((span + count - 1) / count); };
  if (a.units <= 1) {
    u.b = number < B ? number : -1;
    u.count = 1;
  } else if (B <= kWave) {
    const uint64_t hit = __ballot(number >= p.ic - p.cnt && number < p.ic);
    if (hit == 0) {
      u.b = -1;
      return u;
    }
    u.b = __builtin_ctzll(hit);
    u.count = __shfl(p.cnt, u.b, kWave);
    u.slot = __shfl(p.is, u.b, kWave) - (u.count > 1 ? u.count : 0);
    u.part = number - (__shfl(p.ic, u.b, kWave) - u.count);
    length = cut(__shfl(p.span, u.b, kWave), u.count);
  } else {
    int before = 0, slots = 0;  // units and partial slots before this block
    if (tid == 0) s_hit[0] = -1;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
      const int s = b0 + tid < B ? span_of(a, b0 + tid) : 0;
      const int cnt = units_of(s, p.every), sl = cnt > 1 ? cnt : 0;
      int ic = cnt, is = sl;
      scan2(lane, ic, is);
      if (lane == kWave - 1) {
        s_w[0][wave] = ic;
        s_w[1][wave] = is;
      }
      __syncthreads();
      int ec = before + ic - cnt, es = slots + is - sl;
      for (int w = 0; w < wave; ++w) {
        ec += s_w[0][w];
        es += s_w[1][w];
      }
      if (number >= ec && number < ec + cnt) {
        s_hit[0] = b0 + tid;
        s_hit[1] = number - ec;
        s_hit[2] = cnt;
        s_hit[3] = es;
        s_hit[4] = s;
      }
      before += s_w[0][0] + s_w[0][1] + s_w[0][2] + s_w[0][3];
      slots += s_w[1][0] + s_w[1][1] + s_w[1][2] + s_w[1][3];
      __syncthreads();
      if (number < before) break;
    }
    u.b = s_hit[0];
    if (u.b < 0) return u;
    u.part = s_hit[1];
    u.count = s_hit[2];
    u.slot = s_hit[3];
    length = cut(s_hit[4], u.count);
  }
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.part = __builtin_amdgcn_readfirstlane(u.part);
  u.count = __builtin_amdgcn_readfirstlane(u.count);
  u.slot = __builtin_amdgcn_readfirstlane(u.slot);
  length = __builtin_amdgcn_readfirstlane(length);
  if (u.b < 0) return u;
  const int2 tk = tokens_of(a.pg, u.b);
  u.first = tk.x;
  u.n = tk.y;
  u.p = a.pg.pos[u.b];
  u.lo = first_seen(a, u.p);
  if (u.n == 0 || !valid(a, u.p, u.n)) return u;  // c0 = c1
  const int base = u.lo & ~(kTile - 1);
  u.c0 = (int)min((long)base + (long)u.part * length, (long)u.p + u.n);
  u.c1 = (int)min((long)u.c0 + length, (long)u.p + u.n);
  return u;
}

__device__ __forceinline__ void put(float* p, float f) { *p = f; }
__device__ __forceinline__ void put(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ void put4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void put4(uint16_t* p, float4 v) {
  uint2 w;
  w.x = __builtin_bit_cast(uint16_t, (__bf16)v.x) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v.y) << 16;
  w.y = __builtin_bit_cast(uint16_t, (__bf16)v.z) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v.w) << 16;
  *reinterpret_cast<uint2*>(p) = w;
}
__device__ __forceinline__ float value_at(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float value_at(const uint16_t* p, int i) { return bf16_lo(p[i]); }

// What a query row sees.
struct RowLimits {
  int low, last, p;  // rows low .. last, of those from p on the ones whose bit is set
  uint64_t bits;
  // Without branches: five instructions a position (and with short circuits this compiler has lost the
  // assignment that hides a position)
  __device__ __forceinline__ bool sees(int pos) const {
    const int k = pos - p;
    return (pos >= low) & (pos <= last) & ((k < 0) | (((bits >> (k & 63)) & 1) != 0));
  }
};
template <bool MOD>
__device__ __forceinline__ RowLimits limits(const Args& a, const Unit& u, int r, int nrows) {
  RowLimits l{0, -1, 0x7fffffff, 0};
  if (r < nrows) {
    const int i = r / a.G;
    l.last = u.p + i;
    if (MOD) {
      if (a.window > 0) l.low = max(0, u.p + i + 1 - a.window);
      if (a.mask != nullptr) {
        l.p = u.p;
        l.bits = a.mask[u.first + i];
      }
    }
  }
  return l;
}

__device__ __forceinline__ float element(const uint4& w, int e) {  // of eight bf16 values
  const uint32_t v = e < 4 ? (e < 2 ? w.x : w.y) : (e < 6 ? w.z : w.w);
  return e & 1 ? bf16_hi(v) : bf16_lo(v);
}

// One query row over the unit's positions in plain fp32 products, by one wave: what the matrix units'
// pieces make NaN of (an infinite key or value times a zero piece; a hidden row's infinity times a zero
// probability) although the formula does not. One bad value that many rows see sends them all here, so keys are
// read by eight columns, values by eight positions of a column, four loads at once, and a row that sees a NaN or +infinity
// as a score stops there. (A prompt of 4500 tokens with an infinite value in its fourth row: 37 ms, with a NaN key 13,
// 415 each by single elements; 0.24 without them. 40 tokens over 6000 rows of eight sequences: 7 and 2, 42.)
template <typename TQ>
__device__ __forceinline__ void whole_row(const Args& a, const Unit& u, int r, int kvh, float* po, float* pm, float* pl) {
  constexpr int kAhead = 4;  // groups of positions whose values are on their way together
  const int lane = threadIdx.x & (kWave - 1), hd = a.hd, hd8 = hd >> 3, ps = a.pg.page_size;
  const int i = r / a.G, h = kvh * a.G + (r - i * a.G);
  const TQ* q = static_cast<const TQ*>(a.q) + (long)(u.first + i) * a.ldq + (long)h * hd;
  const RowLimits lim = limits<true>(a, u, r, 0x7fffffff);
  auto place = [&](int pos, int& off) {
    const int pg = page_of(a.pg, pos);
    off = pos - pg * ps;
    return (long)a.pg.table[(size_t)u.b * a.pg.max_pages + pg] * a.Hkv + kvh;
  };
  auto score = [&](int pos) {
    int off;
    const long head = place(pos, off);
    const uint4* k = reinterpret_cast<const uint4*>(a.pg.k_pages) + (head * ps + off) * hd8;
    float s = 0.f;
#pragma unroll 4
    for (int c = 0; c < hd8; ++c) {
      const uint4 w = k[c];
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(value_at(q, 8 * c + e), element(w, e), s);
    }
    s *= a.scale;
    if (a.cap > 0.f) s = capped(s, a.cap, 1.f / a.cap);
    if (a.slopes != nullptr) s -= a.slopes[h] * (float)(u.p + i - pos);
    return s;
  };
  float m = -INFINITY;
  bool nan = false;
  for (int pos = u.c0 + lane; pos < u.c1; pos += kWave)
    if (lim.sees(pos)) {
      const float s = score(pos);
      m = fmaxf(m, s);
      nan |= s != s;
    }
  for (int k = 1; k < kWave; k <<= 1) m = fmaxf(m, __shfl_xor(m, k, kWave));
  float l = 0.f, o0 = 0.f, o1 = 0.f;  // columns lane and lane + 64
  if (__ballot(nan) != 0 || m == INFINITY) {  // uniform: every weight is a NaN
    l = __builtin_nanf("");
  } else {
    for (int base = u.c0; base < u.c1; base += kWave) {
      float w = 0.f;
      if (base + lane < u.c1 && lim.sees(base + lane)) {
        const float s = score(base + lane);
        w = s == -INFINITY ? 0.f : expf(s - m);
      }
      l += w;
      const uint64_t some = __ballot(w != 0.f);
      // where each group of eight starts: what has a weight is on a page of the pool, the others read the first one
      long from = 0;
      if (some >> (lane & ~7) & 0xff) {
        int off;
        const long head = place(base + (lane & ~7), off);
        from = head * hd * ps + off;
      }
      for (int g0 = 0; g0 < kWave; g0 += 8 * kAhead) {
        if ((some >> g0) == 0) break;  // uniform
        uint4 v0[kAhead], v1[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const uint16_t* v = a.pg.v_pages + __shfl(from, g0 + 8 * k, kWave);
          v0[k] = *reinterpret_cast<const uint4*>(v + (long)min(lane, hd - 1) * ps);
          v1[k] = *reinterpret_cast<const uint4*>(v + (long)min(lane + kWave, hd - 1) * ps);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float we = __shfl(w, g0 + 8 * k + e, kWave);
            o0 = we != 0.f ? fmaf(we, element(v0[k], e), o0) : o0;
            o1 = we != 0.f ? fmaf(we, element(v1[k], e), o1) : o1;
          }
      }
    }
    l = wave_sum(l);
  }
  if (po != nullptr) {
    if (lane < hd) po[lane] = o0;
    if (lane + kWave < hd) po[lane + kWave] = o1;
    if (lane == 0) {
      *pm = m;
      *pl = l;
    }
  } else {
    TQ* out = static_cast<TQ*>(a.out) + ((long)(u.first + i) * a.H + h) * hd;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (lane < hd) put(out + lane, l == 0.f ? 0.f : o0 * inv);
    if (lane + kWave < hd) put(out + lane + kWave, l == 0.f ? 0.f : o1 * inv);
  }
}

// The rows among a wave's 16 of which some lane says so (lanes fr, fr + 16, .. hold row fr).
__device__ __forceinline__ uint32_t rows_of(bool odd) {
  const uint64_t hit = __ballot(odd);
  return (uint32_t)(hit | hit >> 16 | hit >> 32 | hit >> 48) & 0xffffu;
}

// A sequence outside its table, or a page outside the pool: NaN for its rows r0 .. r1 - 1 of this head (r1 may be
// beyond what an int holds: a sequence may have more tokens than the call was made for).
template <typename TQ>
__device__ __forceinline__ void not_a_number(const Args& a, const Unit& u, int kvh, long r0, long r1, int R) {
  const int tid = threadIdx.x;
  if (u.count > 1) {
    for (long r = r0 + tid; r < r1; r += kThreads) {
      const size_t row = ((size_t)(u.slot + u.part) * a.Hkv + kvh) * R + r;
      a.pm[row] = 0.f;
      a.pl[row] = __builtin_nanf("");
    }
    return;
  }
  for (long e = tid; e < (r1 - r0) * a.hd; e += kThreads) {
    const long r = r0 + e / a.hd, i = r / a.G, h = kvh * a.G + (r - i * a.G);
    put(static_cast<TQ*>(a.out) + ((u.first + i) * a.H + h) * a.hd + e % a.hd, __builtin_nanf(""));
  }
}

// A query row's operand: 8 columns of each 32-wide step, whole or in three pieces.
template <typename TQ, int KS, int NQ>
__device__ __forceinline__ void load_query(const TQ* src, bool there, int g, int hd8, bf16x8_t (&qf)[KS][NQ]) {
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int c = 4 * s + g;
    const bool on = there && c < hd8;
    if constexpr (NQ == 3) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (on) {
        const float4 x = *reinterpret_cast<const float4*>(src + 8 * c), y = *reinterpret_cast<const float4*>(src + 8 * c + 4);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      }
#pragma unroll
      for (int pc = 0; pc < 3; ++pc) {
        qf[s][pc] = __builtin_bit_cast(bf16x8_t, make_uint4(high_halves(v[0], v[1]), high_halves(v[2], v[3]),
                                                             high_halves(v[4], v[5]), high_halves(v[6], v[7])));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = rest(v[e]);
      }
    } else {
      qf[s][0] = __builtin_bit_cast(bf16x8_t, on ? *reinterpret_cast<const uint4*>(src + 8 * c) : make_uint4(0u, 0u, 0u, 0u));
    }
  }
}

// Probabilities as NP bf16 pieces, the last one cut off (three hold every bit), a single one rounded.
template <int NP>
__device__ __forceinline__ void pieces(float (&x)[8], bf16x8_t (&pf)[NP]) {
  if constexpr (NP == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) pf[0][e] = (__bf16)x[e];
  } else {
#pragma unroll
    for (int pc = 0; pc < NP; ++pc) {
      pf[pc] = __builtin_bit_cast(bf16x8_t, make_uint4(high_halves(x[0], x[1]), high_halves(x[2], x[3]),
                                                       high_halves(x[4], x[5]), high_halves(x[6], x[7])));
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = rest_finite(x[e]);
    }
  }
}

// Products to scores: scale, cap and bias of N values at positions t0 + 32 (j / 8) + 8 g + j % 8. (Without
// MOD bf16 products stay as they are: the scale goes into the exponent.)
template <bool MOD, bool F32, int N>
__device__ __forceinline__ void modify(const Args& a, float* x, const RowLimits& lim, float slope, float inv_cap, int t0, int g) {
  if constexpr (MOD || F32) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] *= a.scale;
  }
  if constexpr (MOD) {
    if (a.cap > 0.f) {
      float most = fabsf(x[0]);
#pragma unroll
      for (int e = 1; e < N; ++e) most = __builtin_elementwise_maximum(most, fabsf(x[e]));
      if (__ballot(!(most * inv_cap <= 0.35f)) != 0) {  // rare: scores are small beside a cap
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = capped(x[e], a.cap, inv_cap);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = cap_near(x[e], inv_cap);
      }
    }
    if (a.slopes != nullptr) {
      const float away = (float)(lim.last - t0 - 8 * g);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = fmaf(-slope, away - (float)(32 * (e / 8) + e % 8), x[e]);
    }
  }
}

// KS: 32-wide steps of the head size. MOD: any of cap, slopes, window, mask.
template <typename TQ, int KS, bool MOD>
__global__ __launch_bounds__(kThreads, 2) void attn_rows_kernel(Args a) {
  constexpr bool kF32 = sizeof(TQ) == 4;
  constexpr int NQ = kF32 ? 3 : 1, NP = kF32 ? 3 : 2;  // pieces of queries and probabilities
  constexpr int kHd = KS * 32, DT = KS * 2;
  __shared__ uint2 s_page[kGroups];  // page, offset of an 8-position group
  // the queries' pieces stay in LDS: they would take 48 of the 256 registers
  __shared__ uint4 s_q[kF32 ? KS * NQ * kWave : 1];
  __shared__ int s_bad, s_odd;  // a page outside the pool; a row whose sums are infinite or NaN
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][16][kHd + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int fr = lane & 15, g = lane >> 4, hd8 = a.hd >> 3, ps = a.pg.page_size;
  // heads fastest: workgroups of one head run on one XCD where there are 8 of them
  const int kvh = blockIdx.x % a.Hkv, rg = blockIdx.x / a.Hkv % a.rgroups;
  const Unit u = unit_at(a, make_plan(a), blockIdx.x / (a.Hkv * a.rgroups));
  if (u.b < 0) return;
  const int R = a.G * a.pg.n, r0 = rg * 16;
  if (tid == 0 && kvh == 0 && rg == 0) a.info[u.b] = make_int2(u.slot, u.count);
  if (u.c1 <= u.c0 && !valid(a, u.p, u.n)) {
    // every row, also those behind the row groups that the call was launched for
    if (rg == 0) not_a_number<TQ>(a, u, kvh, 0, (long)u.n * a.G, R);
    return;
  }
  const int nrows = u.n * a.G;
  if (r0 >= nrows) return;
  const int nr = min(16, nrows - r0);
  const size_t prow = ((size_t)(u.slot + u.part) * a.Hkv + kvh) * R + r0;  // this unit's partial rows
  // positions that the group's rows see at all
  const int last = u.p + (r0 + nr - 1) / a.G;
  const int c1 = min(u.c1, last + 1);
  // ---- queries: the B operand, lane (row, 8 columns of each step)
  bf16x8_t qf[KS][NQ];
  const int row = r0 + fr, qi = row / a.G, qh = kvh * a.G + (row - qi * a.G);
  const bool there = row < nrows;
  const RowLimits lim = limits<MOD>(a, u, row, nrows);
  const float slope = MOD && a.slopes != nullptr && there ? a.slopes[qh] : 0.f;
  if (!kF32 || wave == 0) {
    load_query<TQ, KS, NQ>(static_cast<const TQ*>(a.q) + (long)(u.first + (there ? qi : 0)) * a.ldq + (long)(there ? qh : 0) * a.hd,
                           there, g, hd8, qf);
    if constexpr (kF32) {
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int pc = 0; pc < NQ; ++pc) s_q[(s * NQ + pc) * kWave + lane] = __builtin_bit_cast(uint4, qf[s][pc]);
    }
  }
  float m = -FLT_MAX, l = 0.f;
  floatx4_t o[DT];  // columns 16 d + 4 g + e of row fr
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  const float to_exp2 = a.scale * 1.44269504088896341f, inv_cap = MOD && a.cap > 0.f ? 1.f / a.cap : 0.f;
  const int low_last = MOD && a.window > 0 ? max(0, last + 1 - a.window) : 0;  // below it some row sees nothing
  const float slack = kF32 || MOD ? 4.f : 4.f / a.scale;
  if (tid == 0) s_bad = s_odd = 0;

  struct Frag {
    uint4 k[2][KS];
    uint4 v[DT];
  };
  auto load = [&](Frag& f, int t0, int seg) {  // the tile at t0; groups are staged from position seg
    const int gk = (lane >> 2) & 3;
    const uint2 pk = s_page[((t0 - seg) >> 3) + gk], pv = s_page[((t0 - seg) >> 3) + g];
    const uint4* kp = reinterpret_cast<const uint4*>(a.pg.k_pages) +
                      (((size_t)pk.x * a.Hkv + kvh) * ps + pk.y + (lane & 3)) * hd8 + g;
    const uint4* vp = reinterpret_cast<const uint4*>(a.pg.v_pages + (((size_t)pv.x * a.Hkv + kvh) * a.hd + fr) * ps + pv.y);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s)
        f.k[t][s] = 4 * s + g < hd8 ? kp[4 * t * hd8 + 4 * s] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      f.v[d] = 16 * d + fr < a.hd ? vp[(size_t)16 * d * (ps >> 3)] : make_uint4(0u, 0u, 0u, 0u);
  };
  auto query = [&](int s, int pc) {
    if constexpr (kF32) return __builtin_bit_cast(bf16x8_t, s_q[(s * NQ + pc) * kWave + lane]);
    else return qf[s][pc];
  };
  auto compute = [&](Frag& f, int t0) {
    if (kF32) asm volatile("" ::: "memory");  // the queries are read again for each tile, not held
    if (t0 + kTile > c1) {  // uniform: nothing of the rows behind reaches the sums
      uint32_t keep[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = t0 + 8 * g + 2 * e;
        keep[e] = (pos < c1 ? 0xffffu : 0u) | (pos + 1 < c1 ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
        f.v[d] = make_uint4(f.v[d].x & keep[0], f.v[d].y & keep[1], f.v[d].z & keep[2], f.v[d].w & keep[3]);
    }
    {
      float x[8];  // positions t0 + 8 g + e
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        floatx4_t hi = floatx4_t{0.f, 0.f, 0.f, 0.f}, low = hi;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, f.k[h][s]);
#pragma unroll
          for (int pc = NQ - 1; pc > 0; --pc) low = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, query(s, pc), low, 0, 0, 0);
          hi = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, query(s, 0), hi, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = kF32 ? hi[e] + low[e] : hi[e];
      }
      modify<MOD, kF32, 8>(a, x, lim, slope, inv_cap, t0, g);
      // uniform: some row does not see all of it (a mask may hide row p from its own token)
      if (t0 + kTile > min(c1, MOD ? u.p : u.p + 1) || (MOD && t0 < low_last)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int pos = t0 + 8 * g + e;
          const bool seen = MOD ? lim.sees(pos) : pos <= lim.last;
          x[e] = (seen & (pos < c1)) ? x[e] : -INFINITY;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = __builtin_elementwise_maximum(mx, x[e]);
      const float c = MOD ? 1.44269504088896341f : to_exp2;
      // sums stay on their maximum until some score is e^4 above it (or a NaN)
      if (__ballot(!(mx <= m + slack)) != 0) {
        mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 16, kWave));
        mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 32, kWave));
        const float m_new = __builtin_elementwise_maximum(m, mx);
        const float alpha = kF32 ? exp_neg(m - m_new) : __builtin_amdgcn_exp2f((m - m_new) * c);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= alpha;
      }
      float pr[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pr[e] = kF32 ? exp_neg(x[e] - m) : __builtin_amdgcn_exp2f((x[e] - m) * c);
        sum += pr[e];
      }
      l += sum;
      bf16x8_t pf[NP];
      pieces<NP>(pr, pf);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int pc = NP - 1; pc >= 0; --pc)
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f.v[d]), pf[pc], o[d], 0, 0, 0);
    }
  };
  for (int seg = u.c0; seg < c1; seg += kGroups * 8) {
    const int end = min(c1, seg + kGroups * 8);
    __syncthreads();  // the pages staged before are read
    for (int e = tid; e < kGroups && seg + 8 * e < end + kStep; e += kThreads) {
      const int pos = seg + 8 * e;
      uint2 w = make_uint2(0u, 0u);
      if (pos < c1) {
        const int pg = page_of(a.pg, pos), id = a.pg.table[(size_t)u.b * a.pg.max_pages + pg];
        if (id >= 0 && id < a.pg.n_pages) w = make_uint2((uint32_t)id, (uint32_t)(pos - pg * ps));
        else if (pos + 8 > u.lo) s_bad = 1;
      }
      s_page[e] = w;
    }
    __syncthreads();
    Frag fa, fb;
    int t0 = seg + kTile * wave;
    if (t0 < end) load(fa, t0, seg);
    for (; t0 < end; t0 += 2 * kStep) {
      if (t0 + kStep < end) load(fb, t0 + kStep, seg);
      compute(fa, t0);
      if (t0 + kStep >= end) break;
      if (t0 + 2 * kStep < end) load(fa, t0 + 2 * kStep, seg);
      compute(fb, t0 + kStep);
    }
  }
  // ---- the waves' shares joined in order, one query tile at a time
  {
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    floatx4_t chk = floatx4_t{l, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) chk += o[d];
    const float c = (chk[0] + chk[1]) + (chk[2] + chk[3]);
    // infinite sums count: they may be an overflow's, or an infinite value's, which the pieces turned
    if ((rows_of(!(fabsf(c) < INFINITY)) & ((1u << nr) - 1)) != 0 && lane == 0) s_odd = 1;
  }
  __syncthreads();
  if (s_bad) {
    not_a_number<TQ>(a, u, kvh, r0, r0 + nr, R);
    return;
  }
  if (s_odd) {  // uniform
    Unit w = u;
    w.c1 = c1;
    for (int r = wave; r < nr; r += kWaves)
      whole_row<TQ>(a, w, r0 + r, kvh, u.count > 1 ? a.po + (prow + r) * a.hd : nullptr, a.pm + prow + r, a.pl + prow + r);
    return;
  }
  {
    if (g == 0) {
      s_m[wave][fr] = l > 0.f ? m : -INFINITY;
      s_l[wave][fr] = l;
    }
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][fr]);
    const float unit = kF32 || MOD ? 1.f : a.scale;  // m counts unscaled scores there
    const float f = l > 0.f ? expf((m - M) * unit) : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<float4*>(&s_o[wave][fr][16 * d + 4 * g]) =
          make_float4(o[d][0] * f, o[d][1] * f, o[d][2] * f, o[d][3] * f);
    __syncthreads();
    const int rows = nr;
    for (int e = tid; e < rows * (kHd / 4); e += kThreads) {
      const int rr = e / (kHd / 4), c = 4 * (e % (kHd / 4));
      if (c >= a.hd) continue;
      float Mr = -INFINITY, lt = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) Mr = fmaxf(Mr, s_m[w][rr]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(&s_o[w][rr][c]);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        const float mw = s_m[w][rr];
        lt += mw > -INFINITY ? s_l[w][rr] * expf((mw - Mr) * unit) : 0.f;
      }
      const int r = r0 + rr;
      if (u.count > 1) {
        const size_t row = prow + rr;
        *reinterpret_cast<float4*>(a.po + row * a.hd + c) = v;
        if (c == 0) {
          a.pm[row] = Mr * (Mr > -INFINITY ? unit : 1.f);
          a.pl[row] = lt;
        }
      } else {
        const int i = r / a.G, h = kvh * a.G + (r - i * a.G);
        if (lt == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
        else v = make_float4(v.x / lt, v.y / lt, v.z / lt, v.w / lt);
        put4(static_cast<TQ*>(a.out) + ((long)(u.first + i) * a.H + h) * a.hd + c, v);
      }
    }
  }
}

// Query rows by the 64 QT: each wave keeps 16 QT of them for itself, and the four share tiles of 64 positions
// in LDS (keys row by row, values column by column, 16-byte chunks swizzled so that the 16 rows of
// an operand read hit all banks). The tile after the next is on its way to registers while one is
// worked on, and goes to the other LDS buffer behind it: one barrier a tile.
constexpr int kTileP = 64;
constexpr int kRing = 256;  // page entries per half of the ring: 2048 positions

template <typename TQ, int KS, int QT, bool MOD>
__global__ __launch_bounds__(kThreads, 2) void attn_tiles_kernel(Args a) {
  constexpr bool kF32 = sizeof(TQ) == 4;
  constexpr int NQ = kF32 ? 3 : 1;
  // Pieces of the probabilities. bf16 ones of a sequence with more than 64 rows go in one, rounded: their output is rounded
  // to 8 bits too, and two cost a quarter more (prompts of 4500 and 1124 tokens: 213 us with an error of 2.07e-3 of
  // the output's root mean square, 269 us with 1.64e-3, what the output's own rounding makes). Up to 64 rows, drafted chunks
  // and single tokens, they keep 16 bits whatever the call's longest sequence is, and the waves share the rows by 16 (48 tokens over up to
  // 30000 rows in a call for long prompts: 432 us, 438 by one piece, 570 by rows of 32).
  constexpr bool kByRows = !kF32 && QT == 2;
  constexpr int kRowsOfTwo = 64;
  // bf16 scores without anything on top: x c - m c in one step, where m starts at a number whose product
  // is finite (a row with scores below it alone goes the long way)
  constexpr bool kFused = !kF32 && !MOD;
  constexpr float kFusedMin = -1e30f;
  constexpr int DT = KS * 2, kC = KS == 2 ? 8 : 16;  // 16-byte chunks of a key row in LDS
  constexpr int kKLoads = kTileP * kC / kThreads, kVLoads = KS * 32 * 8 / kThreads;
  constexpr int kKChunks = kTileP * kC, kVChunks = KS * 32 * 8;
  __shared__ uint4 s_kv[2][kKChunks + kVChunks];
  __shared__ ulonglong2 s_page[2 * kRing];  // where an 8-position group's keys and values start, in 16-byte units
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 15, g = lane >> 4, hd8 = a.hd >> 3, ps = a.pg.page_size;
  // the longest rows of a prompt first; heads fastest, so that with 8 of them a head stays on one XCD
  const int kvh = blockIdx.x % a.Hkv, rg = a.rgroups - 1 - blockIdx.x / a.Hkv % a.rgroups;
  const Unit u = unit_at(a, make_plan(a), blockIdx.x / (a.Hkv * a.rgroups));
  if (u.b < 0) return;
  const int R = a.G * a.pg.n, r0 = rg * 64 * QT;
  if (tid == 0 && kvh == 0 && rg == 0) a.info[u.b] = make_int2(u.slot, u.count);
  if (u.c1 <= u.c0 && !valid(a, u.p, u.n)) {
    if (rg == 0) not_a_number<TQ>(a, u, kvh, 0, (long)u.n * a.G, R);
    return;
  }
  const int nrows = u.n * a.G;
  if (r0 >= nrows) return;
  const int nr = min(64 * QT, nrows - r0);
  const size_t prow = ((size_t)(u.slot + u.part) * a.Hkv + kvh) * R;
  const int last = u.p + (r0 + nr - 1) / a.G;
  // positions that some row of the group sees
  const int c1 = min(u.c1, last + 1);
  int c0 = u.c0;
  if (MOD && a.window > 0) c0 = max(c0, (u.p + r0 / a.G + 1 - a.window) & ~(kTile - 1));
  const bool few = kByRows && nrows <= kRowsOfTwo;  // uniform
  const int tiles = few ? 1 : QT;                   // of 16 rows, this wave's
  const int w0 = r0 + 16 * tiles * wave;
  bf16x8_t qf[QT][KS][NQ];
  RowLimits lim[QT];
  float slope[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = w0 + 16 * t + fr, i = r / a.G, h = kvh * a.G + (r - i * a.G);
    const bool there = r < nrows && t < tiles;
    lim[t] = limits<MOD>(a, u, r, there ? nrows : 0);
    slope[t] = MOD && a.slopes != nullptr && there ? a.slopes[h] : 0.f;
    load_query<TQ, KS, NQ>(static_cast<const TQ*>(a.q) + (long)(u.first + (there ? i : 0)) * a.ldq + (long)(there ? h : 0) * a.hd,
                           there, g, hd8, qf[t]);
  }
  float m[QT], l[QT];
  floatx4_t o[QT][DT], ls[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = kFused ? kFusedMin : -FLT_MAX;
    l[t] = 0.f;
    ls[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float to_exp2 = a.scale * 1.44269504088896341f, inv_cap = MOD && a.cap > 0.f ? 1.f / a.cap : 0.f;
  const float slack = kF32 || MOD ? 4.f : 4.f / a.scale;
  const int wlast = w0 < nrows ? u.p + (min(w0 + 16 * tiles, nrows) - 1) / a.G : -1;  // the last row this wave sees
  const int low_last = MOD && a.window > 0 ? max(0, wlast + 1 - a.window) : 0;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  auto stage = [&](int seg) {  // the pages of positions c0 + 2048 seg ..
    const int pos = c0 + (seg * kRing + tid) * 8;
    int id = 0, off = 0;
    if (pos < c1) {
      const int pg = page_of(a.pg, pos);
      id = a.pg.table[(size_t)u.b * a.pg.max_pages + pg];
      off = pos - pg * ps;
      if (id < 0 || id >= a.pg.n_pages) {
        id = off = 0;
        if (pos + 8 > u.lo) s_bad = 1;
      }
    }
    const u64 head = (u64)id * a.Hkv + kvh;
    s_page[(seg & 1) * kRing + tid] = make_ulonglong2((head * ps + off) * hd8, head * a.hd * (ps >> 3) + (off >> 3));
  };
  static_assert(kRing == kThreads, "one entry a thread");
  uint4 kw[kKLoads], vw[kVLoads];
  const int kc = tid % kC, kr = tid / kC, vc = tid & 7, vr = tid >> 3;
  static_assert(kThreads / kC % 8 == 0, "a thread's key rows are one row of their groups");
  // Every load is made by every thread: a load under a condition waits for the ones before it. Columns
  // behind the head's read its last ones and are zeroed on the way into LDS.
  const uint4* kbase = reinterpret_cast<const uint4*>(a.pg.k_pages) + (kr & 7) * hd8 + min(kc, hd8 - 1);
  const uint4* vbase[kVLoads];
#pragma unroll
  for (int j = 0; j < kVLoads; ++j)
    vbase[j] = reinterpret_cast<const uint4*>(a.pg.v_pages) + min(vr + j * (kThreads / 8), a.hd - 1) * (ps >> 3);
  auto load = [&](int t0) {
    const int e0 = (t0 - c0) >> 3;
#pragma unroll
    for (int j = 0; j < kKLoads; ++j) kw[j] = kbase[s_page[(e0 + (kr >> 3) + j * (kThreads / kC / 8)) & (2 * kRing - 1)].x];
    const u64 vo = s_page[(e0 + vc) & (2 * kRing - 1)].y;
#pragma unroll
    for (int j = 0; j < kVLoads; ++j) vw[j] = vbase[j][vo];
  };
  auto k_at = [&](int pos, int c) {  // chunk of a key row
    return kC == 16 ? pos * 16 + (c ^ ((pos & 3) | ((pos >> 1) & 12)))
                    : pos * 8 + (c ^ (((pos >> 1) & 1) | ((pos >> 2) & 6)));
  };
  auto v_at = [&](int d, int c) { return kKChunks + d * 8 + (c ^ ((d >> 1) & 7)); };
  auto store = [&](uint4* buf, int t0) {
    if (t0 + kTileP > c1) {  // uniform: nothing behind the last row reaches the sums
      uint32_t keep[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = t0 + 8 * vc + 2 * e;
        keep[e] = (pos < c1 ? 0xffffu : 0u) | (pos + 1 < c1 ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int j = 0; j < kVLoads; ++j)
        vw[j] = make_uint4(vw[j].x & keep[0], vw[j].y & keep[1], vw[j].z & keep[2], vw[j].w & keep[3]);
    }
    if (a.hd < 32 * KS || kC > 4 * KS) {  // uniform
#pragma unroll
      for (int j = 0; j < kKLoads; ++j)
        if (kc >= hd8) kw[j] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int j = 0; j < kVLoads; ++j)
        if (vr + j * (kThreads / 8) >= a.hd) vw[j] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int j = 0; j < kKLoads; ++j) buf[k_at(kr + j * (kThreads / kC), kc)] = kw[j];
#pragma unroll
    for (int j = 0; j < kVLoads; ++j) buf[v_at(vr + j * (kThreads / 8), vc)] = vw[j];
  };
  auto compute = [&](auto np, auto qt, const uint4* buf, int t0) {
    constexpr int NP = decltype(np)::value, QN = decltype(qt)::value;
    constexpr bool kOnes = NP == 1;  // one rounded piece: the sum is of the rounded probabilities, by a product with ones
    if (t0 > wlast) return;  // uniform over the wave
    const bf16x8_t* frag = reinterpret_cast<const bf16x8_t*>(buf);
    float x[QN][2][8];  // positions t0 + 32 nb + 8 g + e
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        floatx4_t hi[QN], low[QN];
#pragma unroll
        for (int t = 0; t < QN; ++t) hi[t] = low[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const bf16x8_t kf = frag[k_at(32 * nb + 8 * (fr >> 2) + 4 * h + (fr & 3), 4 * s + g)];
#pragma unroll
          for (int t = 0; t < QN; ++t) {
#pragma unroll
            for (int pc = NQ - 1; pc > 0; --pc) low[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][s][pc], low[t], 0, 0, 0);
            hi[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][s][0], hi[t], 0, 0, 0);
          }
        }
#pragma unroll
        for (int t = 0; t < QN; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[t][nb][4 * h + e] = kF32 ? hi[t][e] + low[t][e] : hi[t][e];
      }
    // some row of the wave does not see all of it (a mask may hide row p from its own token)
    const bool part = t0 + kTileP > min(c1, MOD && a.mask != nullptr ? u.p : u.p + w0 / a.G + 1);
#pragma unroll
    for (int t = 0; t < QN; ++t) {
      modify<MOD, kF32, 16>(a, &x[t][0][0], lim[t], slope[t], inv_cap, t0, g);
      if (part || (MOD && t0 < low_last)) {  // uniform over the wave
        asm volatile("");  // a branch, not 48 instructions of every tile
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int pos = t0 + 32 * nb + 8 * g + e;
            const bool seen = MOD ? lim[t].sees(pos) : pos <= lim[t].last;
            x[t][nb][e] = (seen & (pos < c1)) ? x[t][nb][e] : -INFINITY;
          }
      }
      float mx = x[t][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = __builtin_elementwise_maximum(mx, x[t][e >> 3][e & 7]);
      const float c = MOD ? 1.44269504088896341f : to_exp2;
      // Sums stay on their maximum until some score is e^4 above it (or a NaN): rare behind a row's
      // first tiles, so the lanes of a row seldom have to agree on a new one
      if (__ballot(!(mx <= m[t] + slack)) != 0) {
        mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 16, kWave));
        mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 32, kWave));
        const float m_new = __builtin_elementwise_maximum(m[t], mx);
        const float alpha = kF32 ? exp_neg(m[t] - m_new) : __builtin_amdgcn_exp2f((m[t] - m_new) * c);
        m[t] = m_new;
        if constexpr (kOnes) ls[t] *= alpha;
        else l[t] *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
      }
      float sum = 0.f;
      const float mc = m[t] * c;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float& y = x[t][nb][e];
          y = kF32 ? exp_neg(y - m[t]) : __builtin_amdgcn_exp2f(kFused ? fmaf(y, c, -mc) : (y - m[t]) * c);
          if (!kOnes) sum += y;
        }
      if (!kOnes) l[t] += sum;
    }
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      bf16x8_t pf[QN][NP];
#pragma unroll
      for (int t = 0; t < QN; ++t) pieces<NP>(x[t][nb], pf[t]);
      if constexpr (kOnes) {
        const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
#pragma unroll
        for (int t = 0; t < QN; ++t) ls[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t][0], ls[t], 0, 0, 0);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8_t vf = frag[v_at(16 * d + fr, 4 * nb + g)];
#pragma unroll
        for (int t = 0; t < QN; ++t)
#pragma unroll
          for (int pc = NP - 1; pc >= 0; --pc) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][pc], o[t][d], 0, 0, 0);
      }
    }
  };
  auto walk = [&](auto np, auto qt) {
    stage(0);
    __syncthreads();
    load(c0);
    store(s_kv[0], c0);
    int seg = 0;
    for (int t0 = c0, i = 0; t0 < c1; t0 += kTileP, ++i) {
      if (i % (kRing * 8 / kTileP) == 0) stage(++seg);  // read from the last tile of this half on
      __syncthreads();
      if (t0 + kTileP < c1) load(t0 + kTileP);
      compute(np, qt, s_kv[i & 1], t0);
      if (t0 + kTileP < c1) store(s_kv[(i + 1) & 1], t0 + kTileP);
    }
  };
  if (c0 < c1) {
    using std::integral_constant;
    if constexpr (kByRows) {
      if (few) walk(integral_constant<int, 2>{}, integral_constant<int, 1>{});
      else walk(integral_constant<int, 1>{}, integral_constant<int, QT>{});
    } else {
      walk(integral_constant<int, kF32 ? 3 : 2>{}, integral_constant<int, QT>{});
    }
  }
  __syncthreads();
  if (s_bad) {
    not_a_number<TQ>(a, u, kvh, r0, r0 + nr, R);
    return;
  }
  uint32_t odd[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, kWave);
    l[t] += __shfl_xor(l[t], 32, kWave);
    if (kByRows) l[t] += ls[t][0];  // one of them is 0
    floatx4_t chk = floatx4_t{l[t], 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) chk += o[t][d];
    odd[t] = rows_of(!(fabsf((chk[0] + chk[1]) + (chk[2] + chk[3])) < INFINITY) || (kFused && !(l[t] > 0.f) && lim[t].last >= c0));
  }
  if ((odd[0] | odd[QT - 1]) != 0) {
    Unit w = u;
    w.c0 = c0;
    w.c1 = c1;
    for (int r = w0; r < min(w0 + 16 * tiles, nrows); ++r)
      whole_row<TQ>(a, w, r, kvh, u.count > 1 ? a.po + (prow + r) * a.hd : nullptr, a.pm + prow + r, a.pl + prow + r);
    return;
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = w0 + 16 * t + fr;
    if (r >= nrows || t >= tiles) continue;
    const float unit = kF32 || MOD ? 1.f : a.scale;
    if (u.count > 1) {
      if (g == 0) {
        a.pm[prow + r] = l[t] > 0.f ? m[t] * unit : -INFINITY;
        a.pl[prow + r] = l[t];
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
        if (16 * d + 4 * g < a.hd)
          *reinterpret_cast<float4*>(a.po + (prow + r) * a.hd + 16 * d + 4 * g) = make_float4(o[t][d][0], o[t][d][1], o[t][d][2], o[t][d][3]);
    } else {
      const int i = r / a.G, h = kvh * a.G + (r - i * a.G);
      TQ* out = static_cast<TQ*>(a.out) + ((long)(u.first + i) * a.H + h) * a.hd;
      const float inv = l[t] > 0.f ? 1.f / l[t] : 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        if (16 * d + 4 * g < a.hd)
          put4(out + 16 * d + 4 * g, make_float4(o[t][d][0] * inv, o[t][d][1] * inv, o[t][d][2] * inv, o[t][d][3] * inv));
    }
  }
}

// The units of a sequence joined in order: one wave per token and head, a lane per two columns, eight units' outputs
// on their way at once. Bound by latency: 5 us for the 17 units of one token, 9 for the two of each of 320 tokens.
template <typename TQ>
__global__ __launch_bounds__(kThreads) void attn_paged_merge_kernel(Args a) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const int t = blockIdx.x, h = blockIdx.y * kWaves + wave;
  if (h >= a.H) return;
  const int b = sequence_of_wave(a.pg, t);
  if (b < 0) return;
  const int2 tk = tokens_of(a.pg, b);
  if (t < tk.x || t >= tk.x + min(tk.y, a.pg.n)) return;
  const int2 info = a.info[b];
  if (info.y <= 1) return;
  const int R = a.G * a.pg.n, kvh = h / a.G, r = (t - tk.x) * a.G + (h - kvh * a.G);
  const size_t row0 = ((size_t)info.x * a.Hkv + kvh) * R + r, stride = (size_t)a.Hkv * R;
  float M = -INFINITY;
  for (int s = lane; s < info.y; s += kWave) M = fmaxf(M, a.pm[row0 + s * stride]);
  for (int k = 1; k < kWave; k <<= 1) M = fmaxf(M, __shfl_xor(M, k, kWave));
  const int c = 2 * lane;
  float den = 0.f;
  float2 num = make_float2(0.f, 0.f);
  for (int s0 = 0; s0 < info.y; s0 += kWave) {
    const int ns = min(kWave, info.y - s0);
    float w = 0.f;
    if (lane < ns) {
      const size_t row = row0 + (s0 + lane) * stride;
      const float ms = a.pm[row];
      w = ms > -INFINITY ? expf(ms - M) : 0.f;
      den += w > 0.f || a.pl[row] != a.pl[row] ? a.pl[row] * w : 0.f;
    }
    for (int s = 0; s < ns; s += kAhead) {
      float2 x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        x[k] = s + k < ns && c < a.hd ? *reinterpret_cast<const float2*>(a.po + (row0 + (s0 + s + k) * stride) * a.hd + c)
                                      : make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float wk = __shfl(w, (s + k) & (kWave - 1), kWave);
        if (s + k < ns && wk > 0.f) {  // an empty unit's outputs were not written
          num.x = fmaf(wk, x[k].x, num.x);
          num.y = fmaf(wk, x[k].y, num.y);
        }
      }
    }
  }
  den = wave_sum(den);
  if (c < a.hd) {
    TQ* out = static_cast<TQ*>(a.out) + ((long)t * a.H + h) * a.hd + c;
    put(out, den == 0.f ? 0.f : num.x / den);
    put(out + 1, den == 0.f ? 0.f : num.y / den);
  }
}

// Query rows of a workgroup: up to 16 on the kernel without LDS, more by 64, and bf16 ones by 128 where
// there are more than 64. (24 bf16 rows over 48 sequences of up to 30000 rows: 300 us in tiles, 426 as twice
// 16 rows; 12 rows 305 us there.)
constexpr int kFewRows = 16;
int group_rows(int rows, bool bf16) { return rows <= kFewRows ? 16 : !bf16 || rows <= 64 ? 64 : 128; }

}  // namespace

// Where the partials of `rows` (unit, query row)s lie.
static void place_partials(PagedAttnLayout& L, int B, size_t rows, int hd) {
  Carve c;
  L.info = c.take((size_t)std::max(B, 1) * sizeof(int2));
  L.pm = c.take(rows * sizeof(float));
  L.pl = c.take(rows * sizeof(float));
  L.po = c.take(rows * hd * sizeof(float));
  L.total = c.off;
}
static int units_per_round(long wgs, int rounds) {
  return (int)std::min<long>(std::max((kTargetWgs + (rounds == 1 ? wgs - 1 : 0)) / wgs, 1l), kMaxUnits);
}

PagedAttnLayout paged_attn_layout(int B, int n, int H, int Hkv, int hd, bool bf16) {
  PagedAttnLayout L{};
  const int R = H / Hkv * n;
  L.rgroups = ceil_div(std::max(R, 1), group_rows(R, bf16));
  // Few rows are bound by memory, which one round and what is over keeps busy; tiles by the matrix units, so
  // a second round that is not full costs as much as a full one.
  L.rounds = R <= kFewRows ? 1 : 2;
  L.units = units_per_round((long)Hkv * L.rgroups, L.rounds);
  // A unit is at least the total row count over rounds * units: sequences of more than one unit make fewer
  // than twice as many of them.
  place_partials(L, B, L.units > 1 ? (size_t)2 * L.rounds * L.units * Hkv * R : 0, hd);
  return L;
}

// What every call of at most B sequences and n tokens of each needs, of either type. The partials of one layout do
// not grow with n: 32 tokens of 32 / 8 heads of 128 take 136 MB, 33 take 70, a long prompt none. Above few rows units *
// Hkv * rgroups <= kTargetWgs and a group has at most 128 rows, which bounds them all.
size_t paged_attn_workspace(int B, int n, int H, int Hkv, int hd) {
  const long R = (long)(H / Hkv) * n;
  const int units = units_per_round(Hkv, 1);
  size_t rows = units > 1 ? (size_t)2 * units * Hkv * std::min<long>(R, kFewRows) : 0;
  if (R > kFewRows && units_per_round(Hkv, 2) > 1) rows = std::max(rows, (size_t)4 * kTargetWgs * std::min(R, 128l));
  PagedAttnLayout L{};
  place_partials(L, B, rows, hd);
  return L.total;
}

long paged_attn_grid(const PagedView& pg, int Hkv, const PagedAttnLayout& L) {
  // every sequence has a unit, and the cuts add fewer than rounds * units
  const long most = (long)pg.B * ceil_div(pg.max_pages * pg.page_size + kTile, kStep);
  return (long)Hkv * L.rgroups * (L.units > 1 ? std::min<long>(pg.B + L.rounds * L.units, most) : pg.B);
}

hipError_t launch_attn_paged(const PagedAttnCall& c, const PagedView& pg, char* ws, const PagedAttnLayout& L,
                             hipStream_t stream) {
  Args a{};
  a.pg = pg;
  a.q = c.q; a.ldq = c.ldq;
  a.H = c.H; a.Hkv = c.Hkv; a.hd = c.hd; a.G = c.H / c.Hkv;
  a.rgroups = L.rgroups; a.units = L.units; a.rounds = L.rounds;
  a.scale = c.scale; a.cap = c.cap; a.slopes = c.slopes; a.window = c.window; a.mask = c.mask;
  a.out = c.out;
  a.info = reinterpret_cast<int2*>(ws + L.info);
  a.pm = reinterpret_cast<float*>(ws + L.pm);
  a.pl = reinterpret_cast<float*>(ws + L.pl);
  a.po = reinterpret_cast<float*>(ws + L.po);
  const bool mod = c.cap > 0.f || c.slopes != nullptr || c.window > 0 || c.mask != nullptr;
  const int R = a.G * pg.n, rows = group_rows(R, c.q_bf16), ks = ceil_div(c.hd, 32);
  const long grid = paged_attn_grid(pg, c.Hkv, L);
  {
    ProfScope prof("attn_paged", stream);
    auto launch = [&](auto tq, auto kss, auto mods) {
      using TQ = decltype(tq);
      constexpr int KS = decltype(kss)::value;
      constexpr bool MOD = decltype(mods)::value;
      if (rows == 16) klaunch(attn_rows_kernel<TQ, KS, MOD>, (int)grid, kThreads, 0, stream, a);
      else if (rows == 64) klaunch(attn_tiles_kernel<TQ, KS, 1, MOD>, (int)grid, kThreads, 0, stream, a);
      else if constexpr (sizeof(TQ) == 2) klaunch(attn_tiles_kernel<TQ, KS, 2, MOD>, (int)grid, kThreads, 0, stream, a);
    };
    auto by_size = [&](auto tq, auto mods) {
      if (ks <= 2) launch(tq, std::integral_constant<int, 2>{}, mods);
      else if (ks == 3) launch(tq, std::integral_constant<int, 3>{}, mods);
      else launch(tq, std::integral_constant<int, 4>{}, mods);
    };
    auto by_mods = [&](auto tq) {
      if (mod) by_size(tq, std::true_type{});
      else by_size(tq, std::false_type{});
    };
    if (c.q_bf16) by_mods(uint16_t{});
    else by_mods(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // a table that holds one unit's rows at most is never cut
  if (L.units <= 1 || (long)pg.max_pages * pg.page_size <= kStep) return hipSuccess;
  ProfScope prof("attn_paged_merge", stream);
  const dim3 mgrid(pg.T, ceil_div(c.H, kWaves));
  if (c.q_bf16) klaunch(attn_paged_merge_kernel<uint16_t>, mgrid, kThreads, 0, stream, a);
  else klaunch(attn_paged_merge_kernel<float>, mgrid, kThreads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace sirius
