// Rotary positions with per-head norms, and the append of rotated keys and of values to the paged cache.
//
// A head's row x (hd columns) is normalised (optional), x^ = x / sqrt(mean(x^2) + eps) * w, and its first
// rot columns are turned pair by pair: with angle a = position * freq_j,
//   (u, v) -> mscale (u cos a - v sin a, u sin a + v cos a),
// pair j being columns (j, j + rot/2) or, interleaved, (2j, 2j + 1). The angle is formed in fp64 and
// reduced to a fraction of a quarter turn there (a position of 10^6 times a frequency of 1 would lose
// 0.06 rad in fp32); sine and cosine of the rest are fp32 polynomials. The norm's sum, the products and
// the one rounding at the end are fp32.
//
// rope_kernel: a thread owns four pairs of a head (two vectors of four columns), 2^lph threads a head,
// and keeps its sines and cosines over all the head rows that it takes (32 + 8 rows share them at
// Llama-3-8B heads). Workgroups take one token each; at few tokens a token's rows are cut over more
// of them. Behind the rotating workgroups, append launches add workgroups that move values: a tile of
// 16 tokens of one head goes through LDS, because the cache holds values transposed (a column's
// positions adjacent, as the attention's matrix operands want them): 16 lanes then store the adjacent
// positions of a column. (Tiles of 64 tokens gave a decode batch of 64 sequences 8 workgroups, 9.5 us
// against 4.8; a prompt of 8192 tokens goes from 57.4 to 58.2 us a call.)
//
// Bound: HBM for prompts. 8192 tokens of 32 + 8 heads of 128, bf16, norms: rotation 36.7 us for 168 MB
// (4.6 TB/s, a large copy's 4.88), append 44.5 us for 201 MB. One token: 3.0 and 4.6 us, a launch.
// A decode batch's values are single 2-byte stores a column (2048 sequences: 46 us, five times its bytes'
// time); that is what the transposed layout costs, and the attention reads each of them hundreds of times.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "paged.h"
#include "profile.h"

namespace sirius {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kValueTokens = 16;  // tokens per value tile

struct RopeArgs {
  const void* q;
  const void* k;
  const void* v;
  long ldq, ldk, ldv;  // elements between tokens
  const int32_t* positions;
  const double* freqs;
  const uint16_t* qw;
  const uint16_t* kw;
  void* q_out;
  uint16_t* k_out;
  int T, H, Hkv, hd, rot, inter;
  float mscale, eps;
  int lph;         // log2 of the threads per head
  int rows;        // head rows per workgroup
  int parts;       // workgroups per token
  PagedView pg;    // append only
};

__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

template <int VEC>
__device__ __forceinline__ void load_vec(const float* p, float* x) {
  if constexpr (VEC == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else {
    x[0] = *p;
  }
}
template <int VEC>
__device__ __forceinline__ void load_vec(const uint16_t* p, float* x) {
  if constexpr (VEC == 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
  } else {
    x[0] = bf16_lo(*p);
  }
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float* x) {
  if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  else *p = x[0];
}
template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t* p, const float* x) {
  if constexpr (VEC == 4)
    *reinterpret_cast<uint2*>(p) = make_uint2(to_bf16(x[0]) | (uint32_t)to_bf16(x[1]) << 16,
                                              to_bf16(x[2]) | (uint32_t)to_bf16(x[3]) << 16);
  else *p = to_bf16(x[0]);
}

// Sine and cosine of `turns` whole turns: the turns and quarter turns come off in fp64, the rest is
// at most an eighth of a turn and goes through the series of sin and cos, cut where the next term is
// below 2e-9 (about one ulp in all).
__device__ __forceinline__ void sincos_turns(double turns, float& s, float& c) {
  const double y = 4.0 * (turns - rint(turns)), k = rint(y);
  const float a = (float)(y - k) * 1.57079632679489662f, z = a * a;
  const float sn = fmaf(a * z, fmaf(z, fmaf(z, fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), a);
  const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
  const int quarter = (int)k & 3;
  const float p = quarter & 1 ? cs : sn, r = quarter & 1 ? sn : cs;
  s = quarter & 2 ? -p : p;
  c = (quarter == 1 || quarter == 2) ? -r : r;
}

// One head row by 2^lph threads, this one with the vectors at columns ca and cb, whose first `live` pairs
// turn (without `inter`: all or none).
template <int VEC, typename TI, typename TO>
__device__ __forceinline__ void turn_row(const RopeArgs& a, const TI* src, const uint16_t* w, TO* dst, bool mine,
                                         int ca, int cb, int live, const float* cs, const float* sn) {
  float x[VEC], y[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = y[e] = 0.f;
  if (mine) {
    load_vec<VEC>(src + ca, x);
    load_vec<VEC>(src + cb, y);
  }
  if (a.eps >= 0.f) {  // uniform
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
    for (int m = 1; m < 1 << a.lph; m <<= 1) ss += __shfl_xor(ss, m, kWave);
    const float inv = 1.0f / sqrtf(ss / (float)a.hd + a.eps);
    float wx[VEC], wy[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) wx[e] = wy[e] = 1.f;
    if (w != nullptr && mine) {
      load_vec<VEC>(w + ca, wx);
      load_vec<VEC>(w + cb, wy);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      x[e] = x[e] * inv * wx[e];
      y[e] = y[e] * inv * wy[e];
    }
  }
  if (!mine || dst == nullptr) return;
  if (VEC == 4 && a.inter) {  // pairs (x0, x1), (x2, x3), (y0, y1), (y2, y3)
    float* const v[2] = {x, y};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float& p = v[j >> 1][(2 * j & 3) & (VEC - 1)];
      float& r = v[j >> 1][((2 * j & 3) + 1) & (VEC - 1)];
      if (j < live) {
        const float t = p * cs[j & (VEC - 1)] - r * sn[j & (VEC - 1)];
        r = fmaf(p, sn[j & (VEC - 1)], r * cs[j & (VEC - 1)]);
        p = t;
      }
    }
  } else if (live > 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float t = x[e] * cs[e] - y[e] * sn[e];
      y[e] = fmaf(x[e], sn[e], y[e] * cs[e]);
      x[e] = t;
    }
  }
  store_vec<VEC>(dst + ca, x);
  store_vec<VEC>(dst + cb, y);
}

// Values of a tile of tokens of one head into the cache.
template <typename TK>
__device__ __forceinline__ void move_values(const RopeArgs& a, int tile, int kvh) {
  __shared__ uint16_t s_v[kValueTokens][128 + 2];  // an odd number of banks between tokens
  __shared__ long s_at[kValueTokens];
  const int tid = threadIdx.x;
  const int t0 = tile * kValueTokens, nt = min(kValueTokens, a.T - t0), ps = a.pg.page_size;
  if (tid < nt) {
    long at = -1;
    const int t = t0 + tid, b = sequence_of_lane(a.pg, t);
    if (b >= 0) {
      const int2 tk = tokens_of(a.pg, b);
      const int p = a.pg.pos[b], row = p + (t - tk.x);
      if (t >= tk.x && t < tk.x + tk.y && rows_fit(a.pg, p, tk.y)) {
        const int pg = page_of(a.pg, row), id = a.pg.table[(size_t)b * a.pg.max_pages + pg];
        if (id >= 0 && id < a.pg.n_pages) at = ((long)id * a.Hkv + kvh) * a.hd * ps + (row - pg * ps);
      }
    }
    s_at[tid] = at;
  }
  const int h4 = a.hd >> 2;
  for (int e = tid; e < nt * h4; e += kRopeThreads) {
    const int t = e / h4, c = 4 * (e - t * h4);
    float x[4];
    load_vec<4>(static_cast<const TK*>(a.v) + (t0 + t) * a.ldv + (long)kvh * a.hd + c, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) s_v[t][c + i] = to_bf16(x[i]);
  }
  __syncthreads();
  if (nt > 8) {
    const int t = tid % kValueTokens;
    const long at = t < nt ? s_at[t] : -1;
    if (at >= 0)
      for (int c = tid / kValueTokens; c < a.hd; c += kRopeThreads / kValueTokens) a.pg.v_pages[at + (long)c * ps] = s_v[t][c];
  } else {  // few tokens: the lanes go over the columns
    for (int e = tid; e < nt * a.hd; e += kRopeThreads) {
      const int t = e / a.hd, c = e - t * a.hd;
      const long at = s_at[t];
      if (at >= 0) a.pg.v_pages[at + (long)c * ps] = s_v[t][c];
    }
  }
}

template <typename TQ, typename TK, int VEC, bool PAGED>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  const int nrot = a.T * a.parts;
  if constexpr (PAGED) {
    if ((int)blockIdx.x >= nrot) {
      const int e = blockIdx.x - nrot;
      move_values<TK>(a, e / a.Hkv, e % a.Hkv);
      return;
    }
  }
  const int t = blockIdx.x / a.parts, part = blockIdx.x - t * a.parts;
  const int tid = threadIdx.x;
  const int u = tid & ((1 << a.lph) - 1), slot = tid >> a.lph, slots = kRopeThreads >> a.lph;
  const int half = a.rot >> 1;
  // this token's position, and with a cache its key row's place
  int position;
  long at = -1;
  if constexpr (PAGED) {
    const int b = sequence_of_wave(a.pg, t);
    if (b < 0) return;  // behind the last sequence: left as it is
    const int2 tk = tokens_of(a.pg, b);
    const int p = a.pg.pos[b];
    if (t < tk.x || t >= tk.x + tk.y) return;  // offsets that do not ascend
    const int row = p + (t - tk.x);
    position = a.positions != nullptr ? a.positions[t] : row;
    if (rows_fit(a.pg, p, tk.y)) {
      const int pg = page_of(a.pg, row), id = a.pg.table[(size_t)b * a.pg.max_pages + pg];
      if (id >= 0 && id < a.pg.n_pages)
        at = (long)id * a.Hkv * a.pg.page_size * a.hd + (long)(row - pg * a.pg.page_size) * a.hd;
    }
  } else {
    position = a.positions[t];
  }
  // columns of this thread and the sines of its pairs
  const int j0 = VEC * u;  // its first pair
  const bool mine = 2 * j0 < a.hd, inter = a.inter != 0;
  int ca, cb;
  if (inter) {
    ca = 2 * j0;
    cb = ca + VEC;
  } else if (j0 < half) {
    ca = j0;
    cb = j0 + half;
  } else {
    ca = a.rot + 2 * (j0 - half);
    cb = ca + VEC;
  }
  const int live = min(max(half - j0, 0), VEC);
  float cs[VEC], sn[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
    if (e < live) {
      constexpr double kInvTurn = 0.159154943091895335769;
      sincos_turns(position * a.freqs[j0 + e] * kInvTurn, sn[e], cs[e]);
      sn[e] *= a.mscale;
      cs[e] *= a.mscale;
    }
  }
  const int end = min((part + 1) * a.rows, a.H + a.Hkv);
  for (int r0 = part * a.rows; r0 < end; r0 += slots) {
    const int r = r0 + slot;
    if (r >= end) break;  // whole heads leave: the norm's lanes are one head's
    if (r < a.H) {
      turn_row<VEC>(a, static_cast<const TQ*>(a.q) + t * a.ldq + (long)r * a.hd, a.qw,
                    static_cast<TQ*>(a.q_out) + ((long)t * a.H + r) * a.hd, mine, ca, cb, live, cs, sn);
    } else {
      const int kvh = r - a.H;
      uint16_t* dst = PAGED ? (at >= 0 ? a.pg.k_pages + at + (long)kvh * a.pg.page_size * a.hd : nullptr)
                            : a.k_out + ((long)t * a.Hkv + kvh) * a.hd;
      turn_row<VEC>(a, static_cast<const TK*>(a.k) + t * a.ldk + (long)kvh * a.hd, a.kw, dst, mine, ca, cb, live, cs, sn);
    }
  }
}

template <bool PAGED>
hipError_t launch(const RopeCall& c, const PagedView* pg, hipStream_t stream) {
  RopeArgs a{};
  a.q = c.q; a.k = c.k; a.v = c.v;
  a.ldq = c.ldq; a.ldk = c.ldk; a.ldv = c.ldv;
  a.positions = c.positions; a.freqs = c.freqs; a.qw = c.qw; a.kw = c.kw;
  a.q_out = c.q_out; a.k_out = c.k_out;
  a.T = c.T; a.H = c.q != nullptr ? c.H : 0; a.Hkv = c.k != nullptr ? c.Hkv : 0; a.hd = c.hd; a.rot = c.rot; a.inter = c.inter;
  a.mscale = c.mscale; a.eps = c.eps;
  if (PAGED) a.pg = *pg;
  // vectors of four columns wherever both halves of a pair start on one
  const bool vec = c.inter || c.rot % 8 == 0;
  const int units = vec ? c.hd / 8 : c.hd / 2;
  while ((1 << a.lph) < units) ++a.lph;
  const int slots = kRopeThreads >> a.lph, heads = a.H + a.Hkv;
  // One workgroup per token forms its sines once; below 1024 tokens a token's heads go to more of them (256 tokens:
  // 4.9 us, 6.5 by one each; 1024: 9.7 by one each, 11.9 where they are cut).
  a.parts = std::max(1, std::min(ceil_div(heads, slots), 1024 / std::max(1, c.T)));
  a.rows = ceil_div(ceil_div(heads, a.parts), slots) * slots;
  a.parts = ceil_div(heads, a.rows);
  const int grid = c.T * a.parts + (PAGED ? ceil_div(c.T, kValueTokens) * c.Hkv : 0);
  ProfScope prof(PAGED ? "kv_append" : "rope", stream);
#define SIRIUS_ROPE(TQ, TK)                                                                  \
  (vec ? klaunch(rope_kernel<TQ, TK, 4, PAGED>, grid, kRopeThreads, 0, stream, a)            \
       : klaunch(rope_kernel<TQ, TK, 1, PAGED>, grid, kRopeThreads, 0, stream, a))
  if (c.q_bf16 && c.k_bf16) SIRIUS_ROPE(uint16_t, uint16_t);
  else if (c.q_bf16) SIRIUS_ROPE(uint16_t, float);
  else if (c.k_bf16) SIRIUS_ROPE(float, uint16_t);
  else SIRIUS_ROPE(float, float);
#undef SIRIUS_ROPE
  return hipGetLastError();
}

}  // namespace

long kv_append_grid(int T, int Hkv) { return T + (long)ceil_div(T, kValueTokens) * Hkv; }

hipError_t launch_rope(const RopeCall& c, hipStream_t stream) { return launch<false>(c, nullptr, stream); }
hipError_t launch_kv_append(const RopeCall& c, const PagedView& pg, hipStream_t stream) {
  return launch<true>(c, &pg, stream);
}

}  // namespace sirius
