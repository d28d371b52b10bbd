// Sampling from rows of logits with temperature, top-k, top-p and min-p, on gfx950.
//
// With best logit M, a token's weight is w = exp((x - M) / T). Every filter keeps a prefix of the
// tokens ordered by (logit descending, index ascending): the first k; of these the ones in front of
// which less than p of their mass lies; of these the ones with w >= m. So a row's kept set is one cut,
// a logit and how many of the tokens that equal it stay. The token drawn is the first in index order
// whose running kept mass exceeds u times the kept mass.
//
// Weights are formed in fp64 and added as whole numbers of 2^-s (s = 62 - log2 V bits), so sums do not
// depend on their order: the histograms below are filled by atomics and every call gives the same
// token. A row's sums carry an error of about 2^-s sqrt(V) of the best token's weight.
//
// sample_row_kernel: one workgroup per row. The cut is found digit by digit (11, 11, 10 bits of the
// logit's ordered bits): counts and masses per digit, the digit that holds the cut, the next one
// within it. A last pass adds the kept mass per tile of the row and the tile that holds the draw is
// looked through token by token.
#include <float.h>
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "profile.h"

namespace sirius {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kTiles = 4096;      // tiles of a row at most
constexpr int kTile = kThreads;   // tokens per tile, a multiple of this where the row has more tiles

typedef unsigned long long u64;

struct Args {
  const float* logits;
  long ld;
  int V, shift;  // weights are counted in units of 2^-shift
  int tile;      // tokens per tile of the last pass
  const float* u;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  int32_t* kept;
  float* prob;
};

// Ordered bits: larger logits have larger keys; a NaN counts as -infinity.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x : -INFINITY);
  return b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xffffffffu));
}

// exp(z) for -700 <= z <= 0: the powers of two come off, the rest (at most ln 2 / 2) goes through the
// series of exp, whose next term is 6e-15.
__device__ __forceinline__ double exp_nonpos(double z) {
  const double n = rint(z * 1.44269504088896340736);
  const double r = fma(-n, 2.3190468138462996e-17, fma(-n, 0.69314718055994530942, z));  // ln 2 and its rest
  double p = 1.0 / 39916800.0;
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

// A row's weights.
struct Weigh {
  double best, inv_t;
  int shift;
  // 0 for what weighs nothing: more than 700 temperatures below the best
  __device__ __forceinline__ double weight(float x) const {
    if (best == INFINITY) return x == INFINITY ? 1.0 : 0.0;
    const double z = ((double)x - best) * inv_t;
    return z >= -700.0 ? exp_nonpos(z) : 0.0;  // NaN too
  }
  __device__ __forceinline__ u64 units(double w) const { return (u64)rint(ldexp(w, shift)); }
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int o) {
  return (u64)__shfl_up((unsigned)(v >> 32), o, kWave) << 32 | __shfl_up((unsigned)v, o, kWave);
}

// Inclusive sums of (count, mass) over the workgroup's threads, and the totals.
struct Scan {
  int c, ct;
  u64 m, mt;
};
__device__ __forceinline__ Scan block_scan(int c, u64 m, int* s_c, u64* s_m) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  for (int o = 1; o < kWave; o <<= 1) {
    const int oc = __shfl_up(c, o, kWave);
    const u64 om = shfl_up64(m, o);
    if (lane >= o) {
      c += oc;
      m += om;
    }
  }
  __syncthreads();  // s_c, s_m of the call before are read
  if (lane == kWave - 1) {
    s_c[wave] = c;
    s_m[wave] = m;
  }
  __syncthreads();
  Scan r{c, 0, m, 0};
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) {
      r.c += s_c[w];
      r.m += s_m[w];
    }
    r.ct += s_c[w];
    r.mt += s_m[w];
  }
  return r;
}

// Four tokens from v0 on; -infinity behind the row.
template <bool ALIGNED>
__device__ __forceinline__ void load4(const float* row, int V, int v0, float* x) {
  if (ALIGNED && v0 + 4 <= V) {
    const float4 t = *reinterpret_cast<const float4*>(row + v0);
    x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = v0 + e < V ? row[v0 + e] : -INFINITY;
  }
}

// A cut: tokens with keys above `key` stay, and the first `ties` of those that equal it.
struct Cut {
  uint32_t key;
  int ties;
  int count;  // tokens that stay
  u64 mass;
};

template <bool ALIGNED>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(Args a) {
  __shared__ u64 s_mass[kTiles];       // histogram or tiles
  __shared__ uint32_t s_count[kTiles];
  __shared__ int s_c[kWaves];
  __shared__ u64 s_m[kWaves];
  __shared__ float s_x[kWaves];
  __shared__ int s_i[kWaves];
  __shared__ int s_bin, s_bc;
  __shared__ u64 s_bm;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int b = blockIdx.x, V = a.V;
  const float* row = a.logits + (long)b * a.ld;
  const float temp = a.temperature != nullptr ? a.temperature[b] : 1.f;
  const float top_p = a.top_p != nullptr ? a.top_p[b] : 1.f, min_p = a.min_p != nullptr ? a.min_p[b] : 0.f;
  const int top_k = a.top_k != nullptr ? a.top_k[b] : 0;
  const float uu = a.u[b];
  // ---- the best token: the lowest index of the largest logit
  float best = -INFINITY;
  int bi = INT32_MAX;
  for (int v0 = 4 * tid; v0 < V; v0 += 4 * kThreads) {
    float x[4];
    load4<ALIGNED>(row, V, v0, x);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (x[e] > best) {
        best = x[e];
        bi = v0 + e;
      }
  }
  auto better = [](float& v, int& i, float ov, int oi) {
    if (ov > v || (ov == v && oi < i)) {
      v = ov;
      i = oi;
    }
  };
  for (int o = 1; o < kWave; o <<= 1) {
    const float ov = __shfl_xor(best, o, kWave);
    const int oi = __shfl_xor(bi, o, kWave);
    better(best, bi, ov, oi);
  }
  if (lane == 0) {
    s_x[wave] = best;
    s_i[wave] = bi;
  }
  __syncthreads();
  best = s_x[0];
  bi = s_i[0];
  for (int w = 1; w < kWaves; ++w) better(best, bi, s_x[w], s_i[w]);
  const bool ok = temp >= 0.f && temp < INFINITY && top_p == top_p && min_p == min_p && uu == uu && best > -INFINITY;
  const bool greedy = temp == 0.f || top_k == 1 || top_p <= 0.f || min_p > 1.f;
  if (!ok || greedy) {  // uniform
    if (tid == 0) {
      a.token[b] = ok ? bi : -1;
      if (a.kept != nullptr) a.kept[b] = ok ? 1 : 0;
      if (a.prob != nullptr) a.prob[b] = ok ? 1.f : 0.f;
    }
    return;
  }
  const Weigh wg{(double)best, 1.0 / (double)temp, a.shift};
  Cut cut{0, INT32_MAX, 0, 0};  // everything
  // ---- one cut: the first `want` tokens, or (want < 0) the tokens in front of which less than `share`
  // units lie; of the tokens that `cut` leaves
  auto refine = [&](int want, double share) {
    uint32_t prefix = 0;
    int above_c = 0;
    u64 above_m = 0;
    int shift = 32;
    for (int level = 0; level < 3; ++level) {
      const int bits = level < 2 ? 11 : 10, low = shift - bits;
      for (int i = tid; i < kBins; i += kThreads) {
        s_mass[i] = 0;
        s_count[i] = 0;
      }
      __syncthreads();
      for (int v0 = 4 * tid; v0 < V; v0 += 4 * kThreads) {
        float x[4];
        load4<ALIGNED>(row, V, v0, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t key = key_of(x[e]);
          if ((level > 0 && key >> shift != prefix) || key <= cut.key) continue;
          const double w = wg.weight(x[e]);
          if (w == 0.0) continue;
          const int bin = key >> low & ((1u << bits) - 1);
          atomicAdd(&s_count[bin], 1u);
          atomicAdd(&s_mass[bin], wg.units(w));
        }
      }
      __syncthreads();
      if (tid == 0 && cut.key != 0 && (level == 0 || cut.key >> shift == prefix)) {  // the ties that the cut before left
        const int bin = cut.key >> low & ((1u << bits) - 1);
        s_count[bin] += cut.ties;
        s_mass[bin] += cut.ties * wg.units(wg.weight(logit_of(cut.key)));
      }
      __syncthreads();
      const int hi = kBins - 1 - 2 * tid;  // two bins a thread, the largest logits first
      const int c0 = s_count[hi], c1 = s_count[hi - 1];
      const u64 m0 = s_mass[hi], m1 = s_mass[hi - 1];
      const Scan sc = block_scan(c0 + c1, m0 + m1, s_c, s_m);
      if (level == 0 && (want >= 0 ? sc.ct <= want : !((double)sc.mt >= share))) {  // uniform: everything stays
        cut.count = sc.ct;
        cut.mass = sc.mt;
        return;
      }
      if (tid == 0) s_bin = -1;
      __syncthreads();
      int bc = above_c + sc.c - c0 - c1;
      u64 bm = above_m + sc.m - m0 - m1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = k == 0 ? c0 : c1;
        const u64 m = k == 0 ? m0 : m1;
        // the cut's bin: the first whose end reaches it
        const bool before = want >= 0 ? bc < want : (double)bm < share, after = want >= 0 ? bc + c >= want : (double)(bm + m) >= share;
        if (c > 0 && before && after) {
          s_bin = hi - k;
          s_bc = bc;
          s_bm = bm;
        }
        bc += c;
        bm += m;
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)s_bin;
      above_c = s_bc;
      above_m = s_bm;
      shift = low;
      __syncthreads();
    }
    const u64 each = wg.units(wg.weight(logit_of(prefix)));
    const int there = (int)s_count[prefix & 1023];
    int ties;
    if (want >= 0) ties = want - above_c;
    else ties = each > 0 ? (int)min(ceil((share - (double)above_m) / (double)each), 2147483647.0) : there;
    ties = min(max(ties, 1), there);
    cut = Cut{prefix, ties, above_c + ties, above_m + ties * each};
    __syncthreads();
  };
  const bool by_k = top_k > 0 && top_k < V, by_p = top_p < 1.f;
  if (by_k) refine(top_k, 0.0);
  if (by_p) {
    if (!by_k) {  // the whole mass first
      u64 m = 0;
      for (int v0 = 4 * tid; v0 < V; v0 += 4 * kThreads) {
        float x[4];
        load4<ALIGNED>(row, V, v0, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) m += wg.units(wg.weight(x[e]));
      }
      cut.mass = block_scan(0, m, s_c, s_m).mt;
      __syncthreads();
    }
    refine(-1, (double)top_p * (double)cut.mass);
  }
  // ---- kept mass per tile, ties apart
  const int tile = a.tile, ntiles = (V + tile - 1) / tile;
  const double floor_w = (double)min_p;
  const u64 tie_mass = cut.key != 0 ? wg.units(wg.weight(logit_of(cut.key))) : 0;
  const bool ties_stay = cut.key != 0 && wg.weight(logit_of(cut.key)) >= floor_w;
  int kept = 0;
  for (int t = wave; t < ntiles; t += kWaves) {
    u64 m = 0;
    int ties = 0;
    const int end = min(V, (t + 1) * tile);
    for (int v0 = t * tile + 4 * lane; v0 < end; v0 += 4 * kWave) {
      float x[4];
      load4<ALIGNED>(row, V, v0, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t key = key_of(x[e]);
        if (key == cut.key) ++ties;
        if (key <= cut.key) continue;
        const double w = wg.weight(x[e]);
        if (w == 0.0 || w < floor_w) continue;
        m += wg.units(w);
        ++kept;
      }
    }
    for (int o = 1; o < kWave; o <<= 1) {
      ties += __shfl_xor(ties, o, kWave);
      m += (u64)__shfl_xor((unsigned)(m >> 32), o, kWave) << 32 | __shfl_xor((unsigned)m, o, kWave);
    }
    if (lane == 0) {
      s_mass[t] = m;
      s_count[t] = ties_stay ? ties : 0;
    }
  }
  for (int i = ntiles + tid; i < kTiles; i += kThreads) {
    s_mass[i] = 0;
    s_count[i] = 0;
  }
  __syncthreads();
  // four tiles a thread: ties first, then the tiles' masses with the ties that stay
  constexpr int kPer = kTiles / kThreads;
  int tie[kPer], tsum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) tsum += tie[k] = s_count[kPer * tid + k];
  const Scan st = block_scan(tsum, 0, s_c, s_m);
  int before = st.c - tsum;
  u64 mass[kPer], msum = 0;
  int tkept = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int stay = min(max(cut.ties - before, 0), tie[k]);
    s_count[kPer * tid + k] = min(cut.ties - min(before, cut.ties), INT32_MAX);  // ties that may still stay here
    before += tie[k];
    tkept += stay;
    mass[k] = s_mass[kPer * tid + k] + stay * tie_mass;
    msum += mass[k];
  }
  const Scan sm = block_scan(kept + tkept, msum, s_c, s_m);
  const double target = (double)fminf(fmaxf(uu, 0.f), 1.f) * (double)sm.mt;
  if (tid == 0) s_bin = -1;
  __syncthreads();
  // the last tile with mass takes what u = 1 asks for
  u64 run = sm.m - msum;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (mass[k] > 0 && (double)run <= target && ((double)(run + mass[k]) > target || run + mass[k] == sm.mt)) {
      s_bin = kPer * tid + k;
      s_bm = run;
    }
    run += mass[k];
  }
  __syncthreads();
  // ---- the tile, one token a thread
  const int t = s_bin;
  u64 ahead = s_bm;
  int may = (int)s_count[t];
  if (tid == 0) s_bc = -1;
  for (int v0 = t * tile; v0 < min(V, (t + 1) * tile); v0 += kThreads) {
    const int v = v0 + tid;
    const float x = v < V ? row[v] : -INFINITY;
    const uint32_t key = key_of(x);
    const bool tied = v < V && ties_stay && key == cut.key;
    const Scan tr = block_scan(tied ? 1 : 0, 0, s_c, s_m);
    double w = 0.0;
    if (tied ? tr.c <= may : v < V && key > cut.key) w = wg.weight(x);
    if (w < floor_w) w = 0.0;
    const u64 m = wg.units(w);
    const Scan ts = block_scan(0, m, s_c, s_m);
    const u64 end = ahead + ts.m;
    if (m > 0 && (double)(end - m) <= target && ((double)end > target || end == sm.mt)) {
      s_bc = v;
      a.token[b] = v;
      if (a.prob != nullptr) a.prob[b] = (float)((double)m / (double)sm.mt);
    }
    __syncthreads();
    if (s_bc >= 0) break;
    ahead += ts.mt;
    may -= min(may, tr.ct);
  }
  if (tid == 0 && a.kept != nullptr) a.kept[b] = sm.ct;
}

}  // namespace

SampleLayout sample_layout(int B, int V) {
  SampleLayout L{};
  L.total = 256;
  return L;
}

hipError_t launch_sample(const SampleCall& c, char* ws, const SampleLayout& L, hipStream_t stream) {
  Args a{};
  a.logits = c.logits; a.ld = c.ld; a.V = c.V;
  a.u = c.u; a.temperature = c.temperature; a.top_k = c.top_k; a.top_p = c.top_p; a.min_p = c.min_p;
  a.token = c.token; a.kept = c.kept; a.prob = c.prob;
  int bits = 0;
  while ((1 << bits) < c.V) ++bits;
  a.shift = 62 - bits;
  a.tile = kTile * ceil_div(ceil_div(c.V, kTile), kTiles);
  const bool aligned = c.ld % 4 == 0 || c.B == 1;
  ProfScope prof("sample_row", stream);
  if (aligned) klaunch(sample_row_kernel<true>, c.B, kThreads, 0, stream, a);
  else klaunch(sample_row_kernel<false>, c.B, kThreads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace sirius
