// Sampling from rows of logits with temperature, top-k, top-p and min-p, on gfx950.
//
// With best logit M, a token's weight is w = exp((x - M) / T). Every filter keeps a prefix of the
// tokens ordered by (logit descending, index ascending): the first k; of these the ones in front of
// which less than p of their mass lies; of these the ones with w >= m. So a row's kept set is one cut,
// a logit and how many of the tokens that equal it stay. The token drawn is the first in index order
// whose running kept mass exceeds u times the kept mass.
//
// Weights are formed in fp64 and added as whole numbers of 2^-s (s = min(50, 62 - log2 V)), so sums do not
// depend on their order: the histograms below are filled by atomics and every call gives the same
// token. A row's sums are off by about 2^-s sqrt(V) of the best token's weight, by V / 2 2^-s at most (a tail of equal
// weights just beside half a unit).
//
// sample_chunk_kernel: one workgroup per chunk of a row, its logits in registers, one reading of HBM: the
// chunk's best token, and what the row's filters need,
//   few (1 < k <= 256)   the tokens that may be among the row's first k: those above a bound that at
//                        least k of the chunk reach (the k-th of the maxima of 512 groups);
//   other filters        the chunk's mass, and counts and masses by bins of an eighth of a temperature,
//                        down to the lightest token that a cut can fall on;
//   none                 the chunk's mass.
// sample_finish_kernel: one workgroup per row. Few: the chunks' tokens above the best bound, sorted in
// LDS; everything is decided on them. Otherwise the bins give the cut's bin, whose tokens are
// gathered from the row (256 MB of cache hold it) and the cut found among them by steps of their keys; the
// chunks' kept masses give the chunk of the draw, and its tokens the draw. Rows that none of this fits (lists
// and bins that overflow, a cut below 32 temperatures, infinite logits) take the long way, row_cut: the cut
// digit by digit (11, 11, 10 bits of the logit's ordered bits), each by a pass over the row. Flat rows are among them: a
// bin's tokens overflow from a temperature of about 1.5 on at 128256 tokens of normal logits (deviation 2.5), and from 1.2
// on at 262144 (top-p of one row 62 us by bins, 324 the long way, 624 at 262144; 192 rows 109 and 403).
//
// Bound: the chunk kernel by HBM and its fp64 weights together (192 rows of 128256 tokens, 98 MB: greedy 16 us,
// the rate of a read; top_k 29; sums alone 34; bins too 40-44), the finishing kernel by the chain of barriers
// and LDS sums of its slowest row (greedy 4 us, top_k 50 11, none 17, min_p 37, top_p 51 of which the gathering 15-20). One row of
// 32000 tokens: 5.8 + 10.4 us. Twice the finishing threads measured the same or slower (top_p 52.9 us).
#include <float.h>
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "profile.h"

namespace sirius {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kTiles = 4096;      // tiles of a row at most
constexpr int kTile = 1024;       // tokens per tile, a multiple of this where the row has more tiles
constexpr int kMaximaAll = 512;   // groups of a chunk whose maxima bound its k-th token
constexpr int kFew = 256;         // the largest k that goes by lists (192 rows of 128256: k = 250 62 us, 2000 by bins 109)
constexpr int kList = 512;        // entries of a chunk's list
constexpr int kSort = 4096;       // tokens that are sorted in LDS at most
constexpr int kFine = 256;        // bins of an eighth of a temperature; the last one is never counted
constexpr int kMaxChunks = 2048;  // 2^24 tokens by 8192
constexpr int kTable = 512;       // powers of two
constexpr int kMarks = 4;         // bounds of a chunk

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
  int chunk, chunks;  // tokens per chunk, chunks per row
  struct ChunkStat* stat;  // [B][chunks]
  u64* list;               // [B][chunks][kList]: key << 32 | ~index, or kFine masses and counts up to each bin's end
};

// What a chunk says of itself.
struct ChunkStat {
  float best, least;  // least: of its finite logits
  int best_at, finite;
  int listed;         // few: tokens on its list (more than kList: it overflowed)
  uint32_t bound[kMarks];  // few: at least mark_of(k, i) tokens reach this key, 0: unknown
  u64 mass;           // in units of its own best
};

// How many tokens reach a chunk's i-th bound: k, a third of it, a ninth, a 27th.
__device__ __forceinline__ int mark_of(int k, int i) {
  for (; i > 0; --i) k = (k + 2) / 3;
  return k;
}

constexpr int kNone = 0, kByList = 1, kByBins = 2, kWhole = 3;  // kNone: bad parameters, or greedy

// A row's parameters and what they ask for.
struct Ask {
  float temp, top_p, min_p, u;
  int top_k, mode;
  bool bad, greedy;
};
__device__ __forceinline__ Ask ask_of(const Args& a, int b) {
  Ask q;
  q.temp = a.temperature != nullptr ? a.temperature[b] : 1.f;
  q.top_p = a.top_p != nullptr ? a.top_p[b] : 1.f;
  q.min_p = a.min_p != nullptr ? a.min_p[b] : 0.f;
  q.top_k = a.top_k != nullptr ? a.top_k[b] : 0;
  q.u = a.u[b];
  q.bad = !(q.temp >= 0.f && q.temp < INFINITY && q.top_p == q.top_p && q.min_p == q.min_p && q.u == q.u);
  q.greedy = q.temp == 0.f || q.top_k == 1 || q.top_p <= 0.f || q.min_p > 1.f;
  if (q.top_k >= a.V) q.top_k = 0;
  q.mode = q.bad || q.greedy ? kNone
           : q.top_k > 0 && q.top_k <= kFew ? kByList
           : q.top_k > 0 || q.top_p < 1.f || q.min_p > 0.f ? kByBins
                                                           : kWhole;
  return q;
}
// Bins per unit of logit. The bin of x counts down from the bin of the best: floor(best s) - floor(x s), the same
// in every kernel; exact while the floors stay below 2^23.
__device__ __forceinline__ float bin_scale(const Ask& q) { return 8.f / q.temp; }
__device__ __forceinline__ float bin_of(float x, float s) { return floorf(x * s); }
// The last bin that a cut can lie in: tokens lighter than (1 - p) / V of the best weigh less than
// (1 - p) of the row together, and those below min_p of it are out. Some more for the roundings.
__device__ __forceinline__ int last_bin(const Ask& q, int V) {
  if (q.top_k > 0) return kFine - 2;
  float z = -1e30f;
  if (q.top_p < 1.f) z = logf((1.f - q.top_p) / (float)V);
  if (q.min_p > 0.f) z = fmaxf(z, logf(q.min_p));
  return (int)fminf(kFine - 2.f, 8.f * -z + 4.f);
}

// Ordered bits: larger logits have larger keys, equal ones (0 and -0) the same; a NaN counts as -infinity.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x + 0.f : -INFINITY);
  return b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xffffffffu));
}

// The first key of a finite logit for which `reached` holds, as it does for all behind it; 64 keys at a time, one per
// lane. Infinity's key: none.
template <typename F>
__device__ __forceinline__ uint32_t first_key(F reached) {
  constexpr uint32_t kLast = 0xff7fffffu;
  const uint32_t lane = threadIdx.x & (kWave - 1);
  uint32_t base = 0x00800000u;  // the lowest logit's; later one that is not reached
  for (int bits = 26; bits >= 0; bits = bits > 6 ? bits - 6 : bits - 2) {  // 26, 20, 14, 8, 2, 0
    const uint32_t away = lane << bits, key = away > kLast - base ? kLast : base + away;
    const int n = __popcll(__ballot(!reached(logit_of(key))));  // of lanes in order
    if (bits == 0) return min(base + n, kLast + 1);
    const uint32_t on = (uint32_t)max(n - 1, 0) << bits;
    if (on > kLast - base) break;
    base += on;
  }
  return kLast + 1;
}

// Lighter than exp(-`least`) beside the best (NaN too). What lies kNothing temperatures below it weighs nothing; up to
// kClear nobody has to look.
constexpr double kNothing = 700.0, kClear = 690.0;
__device__ __forceinline__ bool far_below(float x, double best, double inv_t, double least) {
  return !(((double)x - best) * inv_t >= -least);
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
  __device__ __forceinline__ double weight(float x) const {
    if (best == INFINITY) return x == INFINITY ? 1.0 : 0.0;
    return far_below(x, best, inv_t, kNothing) ? 0.0 : exp_nonpos(((double)x - best) * inv_t);
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

__device__ __forceinline__ void load4_whole(const float* p, float* x) {
  const float4 t = *reinterpret_cast<const float4*>(p);
  x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
}

// A cut: tokens with keys above `key` stay, and the first `ties` of those that equal it.
struct Cut {
  uint32_t key;
  int ties;
  int count;  // tokens that stay
  u64 mass;
};

struct Shared {
  union {
    u64 mass[kTiles];    // the long way: a histogram, or the tiles' masses
    u64 sorted[kSort];
  };
  union {
    uint32_t count[kTiles];
    struct {
      u64 few_mass[kFew];
      uint32_t few_at[kFew];
    };
    struct {
      double scale[kMaxChunks];  // a chunk's units in the row's
      float off[kMaxChunks];     // its bins count from here; infinity: it has nothing
    };
  };
  u64 chunk_mass[kMaxChunks];
  u64 cum_mass[kFine + 1];       // of the bins up to here; entry 0 is 0
  int cum_count[kFine + 1];
  int scan_c[kWaves];
  u64 scan_m[kWaves];
  float x[kWaves];
  int i[kWaves];
  int bin, bc;
  u64 bm;
  int n;
  uint32_t bound;
};

// The long way, over the whole row.
template <bool ALIGNED>
__device__ __forceinline__ void row_cut(const Args& a, const Ask& q, const Weigh& wg, int b, Shared& sh) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, V = a.V;
  const float* row = a.logits + (long)b * a.ld;
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
        sh.mass[i] = 0;
        sh.count[i] = 0;
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
          atomicAdd(&sh.count[bin], 1u);
          atomicAdd(&sh.mass[bin], wg.units(w));
        }
      }
      __syncthreads();
      if (tid == 0 && cut.key != 0 && (level == 0 || cut.key >> shift == prefix)) {  // the ties that the cut before left
        const int bin = cut.key >> low & ((1u << bits) - 1);
        sh.count[bin] += cut.ties;
        sh.mass[bin] += cut.ties * wg.units(wg.weight(logit_of(cut.key)));
      }
      __syncthreads();
      constexpr int kB = kBins / kThreads;
      const int hi = kBins - 1 - kB * tid;  // some bins a thread, the largest logits first
      int c0 = 0;
      u64 m0 = 0;
#pragma unroll
      for (int k = 0; k < kB; ++k) {
        c0 += sh.count[hi - k];
        m0 += sh.mass[hi - k];
      }
      const Scan sc = block_scan(c0, m0, sh.scan_c, sh.scan_m);
      if (level == 0 && (want >= 0 ? sc.ct <= want : !((double)sc.mt >= share))) {  // uniform: everything stays
        cut.count = sc.ct;
        cut.mass = sc.mt;
        return;
      }
      if (tid == 0) sh.bin = -1;
      __syncthreads();
      int bc = above_c + sc.c - c0;
      u64 bm = above_m + sc.m - m0;
#pragma unroll
      for (int k = 0; k < kB; ++k) {
        const int c = sh.count[hi - k];
        const u64 m = sh.mass[hi - k];
        // the cut's bin: the first whose end reaches it
        const bool before = want >= 0 ? bc < want : (double)bm < share, after = want >= 0 ? bc + c >= want : (double)(bm + m) >= share;
        if (c > 0 && before && after) {
          sh.bin = hi - k;
          sh.bc = bc;
          sh.bm = bm;
        }
        bc += c;
        bm += m;
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)sh.bin;
      above_c = sh.bc;
      above_m = sh.bm;
      shift = low;
      __syncthreads();
    }
    const u64 each = wg.units(wg.weight(logit_of(prefix)));
    const int there = (int)sh.count[prefix & 1023];
    int ties;
    if (want >= 0) ties = want - above_c;
    else ties = each > 0 ? (int)min(ceil((share - (double)above_m) / (double)each), 2147483647.0) : there;
    ties = min(max(ties, 1), there);
    cut = Cut{prefix, ties, above_c + ties, above_m + ties * each};
    __syncthreads();
  };
  const bool by_k = q.top_k > 0, by_p = q.top_p < 1.f;
  if (by_k) refine(q.top_k, 0.0);
  if (by_p) {
    if (!by_k) {  // the whole mass first
      u64 m = 0;
      for (int v0 = 4 * tid; v0 < V; v0 += 4 * kThreads) {
        float x[4];
        load4<ALIGNED>(row, V, v0, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) m += wg.units(wg.weight(x[e]));
      }
      cut.mass = block_scan(0, m, sh.scan_c, sh.scan_m).mt;
      __syncthreads();
    }
    refine(-1, (double)q.top_p * (double)cut.mass);
  }
  // ---- kept mass per tile, ties apart
  const int tile = a.tile, ntiles = (V + tile - 1) / tile;
  const double floor_w = (double)q.min_p;
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
      sh.mass[t] = m;
      sh.count[t] = ties_stay ? ties : 0;
    }
  }
  for (int i = ntiles + tid; i < kTiles; i += kThreads) {
    sh.mass[i] = 0;
    sh.count[i] = 0;
  }
  __syncthreads();
  // eight tiles a thread: ties first, then the tiles' masses with the ties that stay
  constexpr int kPer = kTiles / kThreads;
  int tie[kPer], tsum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) tsum += tie[k] = sh.count[kPer * tid + k];
  const Scan st = block_scan(tsum, 0, sh.scan_c, sh.scan_m);
  int before = st.c - tsum;
  u64 mass[kPer], msum = 0;
  int tkept = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int stay = min(max(cut.ties - before, 0), tie[k]);
    sh.count[kPer * tid + k] = min(cut.ties - min(before, cut.ties), INT32_MAX);  // ties that may still stay here
    before += tie[k];
    tkept += stay;
    mass[k] = sh.mass[kPer * tid + k] + stay * tie_mass;
    msum += mass[k];
  }
  const Scan sm = block_scan(kept + tkept, msum, sh.scan_c, sh.scan_m);
  const double target = (double)fminf(fmaxf(q.u, 0.f), 1.f) * (double)sm.mt;
  if (tid == 0) sh.bin = -1;
  __syncthreads();
  // the last tile with mass takes what u = 1 asks for
  u64 run = sm.m - msum;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (mass[k] > 0 && (double)run <= target && ((double)(run + mass[k]) > target || run + mass[k] == sm.mt)) {
      sh.bin = kPer * tid + k;
      sh.bm = run;
    }
    run += mass[k];
  }
  __syncthreads();
  // ---- the tile, one token a thread
  const int t = sh.bin;
  u64 ahead = sh.bm;
  int may = (int)sh.count[t];
  if (tid == 0) sh.bc = -1;
  for (int v0 = t * tile; v0 < min(V, (t + 1) * tile); v0 += kThreads) {
    const int v = v0 + tid;
    const float x = v < V ? row[v] : -INFINITY;
    const uint32_t key = key_of(x);
    const bool tied = v < V && ties_stay && key == cut.key;
    const Scan tr = block_scan(tied ? 1 : 0, 0, sh.scan_c, sh.scan_m);
    double w = 0.0;
    if (tied ? tr.c <= may : v < V && key > cut.key) w = wg.weight(x);
    if (w < floor_w) w = 0.0;
    const u64 m = wg.units(w);
    const Scan ts = block_scan(0, m, sh.scan_c, sh.scan_m);
    const u64 end = ahead + ts.m;
    if (m > 0 && (double)(end - m) <= target && ((double)end > target || end == sm.mt)) {
      sh.bc = v;
      a.token[b] = v;
      if (a.prob != nullptr) a.prob[b] = (float)((double)m / (double)sm.mt);
    }
    __syncthreads();
    if (sh.bc >= 0) break;
    ahead += ts.mt;
    may -= min(may, tr.ct);
  }
  if (tid == 0 && a.kept != nullptr) a.kept[b] = sm.ct;
}


// 2^(j / 512) for the powers below.
__device__ __forceinline__ void fill_table(double* table) {
  for (int i = threadIdx.x; i < kTable; i += blockDim.x) table[i] = 2.0 * exp_nonpos((i - kTable) * (0.69314718055994530942 / kTable));
}
// Units of 2^-shift (shift <= 50) of exp((x - best) / T), y = (x - best) 512 log2(e) / T <= 0: a power of two
// from the table times the series of 2^(r / 512), |r| <= 1/2, whose next term is 1e-14. Rounding to whole
// numbers is done by adding numbers whose last bit is 1. What is far below one unit comes out 0.
__device__ __forceinline__ u64 fast_units(double y, int shift, const double* table) {
  constexpr double kL = 0.69314718055994530942 / kTable, kWhole = 6755399441055744.0;  // 1.5 * 2^52
  y = fmax(y, -64.0 * kTable);
  const double z = y + kWhole;
  const double r = y - (z - kWhole);
  const int n = (int)(uint32_t)__double_as_longlong(z);
  const double g = r * fma(r, fma(r, kL * kL * kL / 6.0, kL * kL / 2.0), kL);
  const double t = __longlong_as_double(__double_as_longlong(table[n & (kTable - 1)]) + ((long long)((n >> 9) + shift) << 52));
  return (u64)__double_as_longlong(fma(t, g, t) + 4503599627370496.0) & 0xfffffffffffffull;
}

// THREADS * PER * 4 tokens; 256 threads with 8 float4s each stream a large call faster than 512 with 4 (18 against
// 24 us for 98 MB), 512 with one each finish a small one sooner.
template <bool ALIGNED, int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void sample_chunk_kernel(Args a) {
  constexpr int kW = THREADS / kWave, kSub = kMaximaAll / THREADS, kMaxima = kMaximaAll / kWave;
  static_assert(kW >= kMarks && THREADS >= kFine, "a wave for each bound, a thread for each bin");
  __shared__ float s_x[kW], s_y[kW];
  __shared__ int s_i[kW], s_f[kW], s_n;
  __shared__ u64 s_m[kW];
  __shared__ uint32_t s_bound[kMarks];
  __shared__ int s_c[kW];
  __shared__ union {
    uint32_t sub[kMaximaAll];
    struct {
      double table[kTable];
      u64 mass[kFine];
      uint32_t count[kFine];
    };
  } sh;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int c = blockIdx.x % a.chunks, b = blockIdx.x / a.chunks;
  const Ask q = ask_of(a, b);
  if (q.bad) return;
  const float* row = a.logits + (long)b * a.ld;
  const int v0 = c * a.chunk;
  float x[PER][4];
  if (ALIGNED && v0 + a.chunk <= a.V) {  // uniform: loads under no condition, all on their way together
#pragma unroll
    for (int j = 0; j < PER; ++j) load4_whole(row + v0 + 4 * (tid + j * THREADS), x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j) load4<ALIGNED>(row, a.V, v0 + 4 * (tid + j * THREADS), x[j]);
  }
  const bool sums = q.mode == kByBins || q.mode == kWhole;  // uniform
  float best = -INFINITY, least = INFINITY;
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[j][e] = fmaxf(x[j][e], -INFINITY);  // a NaN too
      best = fmaxf(best, x[j][e]);
      least = fminf(least, x[j][e]);
    }
  for (int o = 1; o < kWave; o <<= 1) {
    best = fmaxf(best, __shfl_xor(best, o, kWave));
    least = fminf(least, __shfl_xor(least, o, kWave));
  }
  if (lane == 0) {
    s_x[wave] = best;
    s_y[wave] = least;
  }
  if (tid == 0) s_n = 0;
  if (sums) fill_table(sh.table);
  if (q.mode == kByBins && tid < kFine) {
    sh.mass[tid] = 0;
    sh.count[tid] = 0;
  }
  if (q.mode == kByList) {
#pragma unroll
    for (int k = 0; k < kSub; ++k) {  // of the thread's tokens, in kSub groups
      float m = -INFINITY;
#pragma unroll
      for (int e = k * 4 * PER / kSub; e < (k + 1) * 4 * PER / kSub; ++e) m = fmaxf(m, x[e / 4][e % 4]);
      sh.sub[k * THREADS + tid] = key_of(m);
    }
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kW; ++w) {
    best = fmaxf(best, s_x[w]);
    least = fminf(least, s_y[w]);
  }
  if (q.mode == kNone) {  // greedy: the best's first index
    int at = INT32_MAX;
#pragma unroll
    for (int j = PER - 1; j >= 0; --j)
#pragma unroll
      for (int e = 3; e >= 0; --e) at = x[j][e] == best ? 4 * j * THREADS + e : at;
    if (at != INT32_MAX) at += v0 + 4 * tid;
    for (int o = 1; o < kWave; o <<= 1) at = min(at, __shfl_xor(at, o, kWave));
    if (lane == 0) s_i[wave] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kW; ++w) at = min(at, s_i[w]);
      a.stat[(size_t)b * a.chunks + c] = ChunkStat{best, best, at, 0, 0, {}, 0};
    }
    return;
  }
  int finite = min(a.V, v0 + a.chunk) - v0;
  if (const double inv_t = 1.0 / (double)q.temp; sums && far_below(least, (double)best, inv_t, kClear)) {
    // uniform: what weighs something beside the chunk's best, and the least of it; a mask's lowest numbers are not counted
    const float weighs = logit_of(first_key([&](float y) { return !far_below(y, (double)best, inv_t, kNothing); }));
    float low = INFINITY;
    finite = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (x[j][e] >= weighs) {
          ++finite;
          low = fminf(low, x[j][e]);
        }
      }
    for (int o = 1; o < kWave; o <<= 1) {
      low = fminf(low, __shfl_xor(low, o, kWave));
      finite += __shfl_xor(finite, o, kWave);
    }
    __syncthreads();
    if (lane == 0) {
      s_y[wave] = low;
      s_f[wave] = finite;
    }
    __syncthreads();
    least = s_y[0];
    finite = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      least = fminf(least, s_y[w]);
      finite += s_f[w];
    }
  }
  ChunkStat st{best, least, INT32_MAX, finite, 0, {}, 0};
  u64* list = a.list + ((size_t)b * a.chunks + c) * kList;
  if (q.mode == kByList) {
    if (wave < kMarks) {  // the largest key of 16 bits that so many of the threads' maxima reach
      const int want = mark_of(q.top_k, wave);
      uint32_t sub[kMaxima];
#pragma unroll
      for (int k = 0; k < kMaxima; ++k) sub[k] = sh.sub[k * kWave + lane];
      uint32_t bound = 0;
      for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        int n = 0;
#pragma unroll
        for (int k = 0; k < kMaxima; ++k) n += __popcll(__ballot(sub[k] >= (bound | bit)));
        if (n >= want) bound |= bit;
      }
      if (lane == 0) s_bound[wave] = bound;
    }
    __syncthreads();
    const uint32_t bound = s_bound[0];
    float reach = bound > key_of(-INFINITY) ? logit_of(bound) : -INFINITY;
    // tokens that weigh nothing stay off the list: few may be left where a mask's lowest numbers are many
    reach = fmaxf(reach, (float)((double)best - (kNothing + 1.0) * (double)q.temp));
    int from = v0 + 4 * tid;
    asm volatile("" : "+v"(from));  // or all indices are formed, and held, from the kernel's start on
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (x[j][e] >= reach && x[j][e] > -INFINITY) {
          const int n = atomicAdd(&s_n, 1);
          if (n < kList) list[n] = (u64)key_of(x[j][e]) << 32 | ~(uint32_t)(from + 4 * j * THREADS + e);
        }
      }
    __syncthreads();
    st.listed = s_n;
#pragma unroll
    for (int i = 0; i < kMarks; ++i) st.bound[i] = s_bound[i] > key_of(-INFINITY) ? s_bound[i] : 0;
  } else if (sums && best > -INFINITY) {
    const double to = kTable * 1.44269504088896340736 / (double)q.temp, from = (double)best;
    const float s = bin_scale(q), top = bin_of(best, s);
    const float last = q.mode == kByBins ? (float)last_bin(q, a.V) : -1.f;
    u64 m = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u64 w = fast_units(((double)x[j][e] - from) * to, a.shift, sh.table);
        m += w;
        if (q.mode == kByBins) {  // uniform
          const float bin = top - bin_of(x[j][e], s);
          if (bin <= last) {
            atomicAdd(&sh.mass[(int)bin], w);
            atomicAdd(&sh.count[(int)bin], 1u);
          }
        }
      }
    auto add_up = [&](u64 v) {
      for (int o = 1; o < kWave; o <<= 1) v += (u64)__shfl_xor((unsigned)(v >> 32), o, kWave) << 32 | __shfl_xor((unsigned)v, o, kWave);
      return v;
    };
    m = add_up(m);
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
    for (int w = 0; w < kW; ++w) st.mass += s_m[w];
    if (q.mode == kByBins) {  // sums up to each bin's end
      u64 cm = tid < kFine ? sh.mass[tid] : 0;
      int cc = tid < kFine ? (int)sh.count[tid] : 0;
      for (int o = 1; o < kWave; o <<= 1) {
        const u64 om = shfl_up64(cm, o);
        const int oc = __shfl_up(cc, o, kWave);
        if (lane >= o) {
          cm += om;
          cc += oc;
        }
      }
      __syncthreads();
      if (lane == kWave - 1) {
        s_m[wave] = cm;
        s_c[wave] = cc;
      }
      __syncthreads();
      for (int w = 0; w < wave; ++w) {
        cm += s_m[w];
        cc += s_c[w];
      }
      if (tid < kFine) {
        list[tid] = cm;
        reinterpret_cast<uint32_t*>(list + kFine)[tid] = cc;
      }
    }
  }
  if (tid == 0) a.stat[(size_t)b * a.chunks + c] = st;
}

// Sorts v[0 .. n), the largest first (bitonic; zeros behind them up to a power of two of at least 64).
// Partners less than 64 apart are a wave's own: they are exchanged between its lanes.
__device__ __forceinline__ void sort_down(u64* v, int n) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  int n2 = kWave;
  while (n2 < n) n2 <<= 1;
  for (int i = n + tid; i < n2; i += kThreads) v[i] = 0;
  __syncthreads();
  auto in_wave = [&](int s0, int s1) {  // the steps within a wave of sizes s0 .. s1
    for (int i0 = tid & ~(kWave - 1); i0 < n2; i0 += kThreads) {
      const int i = i0 + lane;
      u64 x = v[i];
      for (int size = s0; size <= s1; size <<= 1)
        for (int step = min(size, kWave) >> 1; step > 0; step >>= 1) {
          const u64 y = (u64)__shfl_xor((unsigned)(x >> 32), step, kWave) << 32 | __shfl_xor((unsigned)x, step, kWave);
          const bool larger = ((i & size) == 0) == ((i & step) == 0);  // keeps the larger one
          x = (x > y) == larger ? x : y;
        }
      v[i] = x;
    }
  };
  in_wave(2, kWave);
  for (int size = 2 * kWave; size <= n2; size <<= 1) {
    for (int step = size >> 1; step >= kWave; step >>= 1) {
      __syncthreads();
      for (int i = tid; i < n2 >> 1; i += kThreads) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const u64 p = v[lo], r = v[hi];
        if ((p < r) == ((lo & size) == 0)) {
          v[lo] = r;
          v[hi] = p;
        }
      }
    }
    __syncthreads();
    in_wave(size, size);
  }
  __syncthreads();
}

template <bool ALIGNED>
__global__ __launch_bounds__(kThreads) void sample_finish_kernel(Args a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int b = blockIdx.x, V = a.V;
  const float* row = a.logits + (long)b * a.ld;
  const Ask q = ask_of(a, b);
  const ChunkStat* stat = a.stat + (size_t)b * a.chunks;
  auto answer = [&](int token, int kept, float prob) {
    a.token[b] = token;
    if (a.kept != nullptr) a.kept[b] = kept;
    if (a.prob != nullptr) a.prob[b] = prob;
  };
  if (q.bad) {
    if (tid == 0) answer(-1, 0, 0.f);
    return;
  }
  // ---- the row's best, the least logit that its chunks count and how many those are
  float best = -INFINITY, least = INFINITY;
  int at = INT32_MAX, finite = 0;
  for (int c = tid; c < a.chunks; c += kThreads) {
    const ChunkStat st = stat[c];
    if (st.best > best || (st.best == best && st.best_at < at)) {
      best = st.best;
      at = st.best_at;
    }
    least = fminf(least, st.least);
    finite += st.finite;
  }
  if (a.chunks > 1) {  // uniform
    for (int o = 1; o < kWave; o <<= 1) {
      const float ov = __shfl_xor(best, o, kWave);
      const int oi = __shfl_xor(at, o, kWave);
      if (ov > best || (ov == best && oi < at)) {
        best = ov;
        at = oi;
      }
      least = fminf(least, __shfl_xor(least, o, kWave));
      finite += __shfl_xor(finite, o, kWave);
    }
  }
  if (lane == 0) {
    sh.x[wave] = best;
    sh.i[wave] = at;
    sh.scan_c[wave] = finite;
    sh.scan_m[wave] = __float_as_uint(least);
  }
  if (tid == 0) {
    sh.n = 0;
    sh.bin = sh.bc = -1;
  }
  __syncthreads();
  const int nw = a.chunks > kThreads - kWave ? kWaves : (a.chunks + kWave - 1) / kWave;  // waves that saw chunks
  best = sh.x[0];
  at = sh.i[0];
  finite = sh.scan_c[0];
  least = __uint_as_float((uint32_t)sh.scan_m[0]);
  for (int w = 1; w < nw; ++w) {
    if (sh.x[w] > best || (sh.x[w] == best && sh.i[w] < at)) {
      best = sh.x[w];
      at = sh.i[w];
    }
    finite += sh.scan_c[w];
    least = fminf(least, __uint_as_float((uint32_t)sh.scan_m[w]));
  }
  if (best == -INFINITY || q.greedy) {
    if (tid == 0) {
      if (best == -INFINITY) answer(-1, 0, 0.f);
      else answer(at, 1, 1.f);
    }
    return;
  }
  const Weigh wg{(double)best, 1.0 / (double)q.temp, a.shift};
  const double share_u = (double)fminf(fmaxf(q.u, 0.f), 1.f);
  const float s = bin_scale(q), top = bin_of(best, s);
  bool longway = best == INFINITY;
  if (q.mode == kByList && !longway) {
    if (wave == 0) {
      // The largest key that k tokens of the row are known to reach: the chunks' bounds say how many of
      // theirs do
      uint32_t bound = 0;
      int weight[kMarks];
#pragma unroll
      for (int i = 0; i < kMarks; ++i) weight[i] = mark_of(q.top_k, i) - (i + 1 < kMarks ? mark_of(q.top_k, i + 1) : 0);
      const bool one = a.chunks <= kWave;
      uint32_t mine[kMarks] = {0, 0, 0, 0};
      if (one && lane < a.chunks)
#pragma unroll
        for (int i = 0; i < kMarks; ++i) mine[i] = stat[lane].bound[i];
      for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        int n = 0;
        for (int c0 = 0; c0 < a.chunks; c0 += kWave) {
          if (!one) {
#pragma unroll
            for (int i = 0; i < kMarks; ++i) mine[i] = c0 + lane < a.chunks ? stat[c0 + lane].bound[i] : 0;
          }
#pragma unroll
          for (int i = 0; i < kMarks; ++i) n += weight[i] * __popcll(__ballot(mine[i] >= (bound | bit)));
        }
        if (n >= q.top_k) bound |= bit;
      }
      if (lane == 0) sh.bound = bound;
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    for (int c0 = wave; c0 < a.chunks; c0 += 4 * kWaves) {  // four lists' first entries at once
      u64 e[4];
      int n[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = min(c0 + k * kWaves, a.chunks - 1);
        // a list without a token that reaches the bound is passed over, also one that overflowed
        const int listed = stat[c].listed;
        n[k] = ((c0 + k * kWaves < a.chunks) & (key_of(stat[c].best) >= bound)) ? listed : 0;
        if (n[k] > kList) {
          if (lane == 0) atomicAdd(&sh.n, kSort + 1);  // the long way
          n[k] = 0;
        }
        e[k] = a.list[((size_t)b * a.chunks + c) * kList + lane];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        for (int i = lane; i < n[k]; i += kWave) {
          const u64 x = i == lane ? e[k] : a.list[((size_t)b * a.chunks + c0 + k * kWaves) * kList + i];
          if ((uint32_t)(x >> 32) >= bound) {
            const int to = atomicAdd(&sh.n, 1);
            if (to < kSort) sh.sorted[to] = x;
          }
        }
    }
    __syncthreads();
    const int n = sh.n;
    longway = n > kSort;
    if (!longway) {
      sort_down(sh.sorted, n);
      // the first k, their masses in order, and how many of them stay
      double w = 0.0;
      const u64 mine = tid < min(n, q.top_k) ? sh.sorted[tid] : 0;
      if (mine != 0) w = wg.weight(logit_of((uint32_t)(mine >> 32)));
      const u64 m = wg.units(w);
      const Scan all = block_scan(0, m, sh.scan_c, sh.scan_m);
      const bool stays = w > 0.0 && (tid == 0 || ((q.top_p >= 1.f || (double)(all.m - m) < (double)q.top_p * (double)all.mt) && w >= (double)q.min_p));
      const Scan kept = block_scan(stays ? 1 : 0, stays ? m : 0, sh.scan_c, sh.scan_m);
      if (stays) {
        sh.few_mass[tid] = m;
        sh.few_at[tid] = ~(uint32_t)mine;
      }
      if (tid < kFew) sh.chunk_mass[tid] = 0;
      __syncthreads();
      // each one's mass up to its index, by as many threads as there are for it (50 tokens: 10.6 us, 12.6 by one each)
      int lp = 6;
      while (1 << lp < kept.ct) ++lp;
      if (const int at = tid & ((1 << lp) - 1); at < kept.ct) {
        const uint32_t here = sh.few_at[at];
        u64 run = 0;
        for (int i = tid >> lp; i < kept.ct; i += kThreads >> lp) run += sh.few_at[i] <= here ? sh.few_mass[i] : 0;
        atomicAdd(&sh.chunk_mass[at], run);
      }
      __syncthreads();
      if (stays && m > 0) {
        const uint32_t here = sh.few_at[tid];
        const u64 run = sh.chunk_mass[tid];
        const double target = share_u * (double)kept.mt;
        if ((double)(run - m) <= target && ((double)run > target || run == kept.mt))
          answer((int)here, kept.ct, (float)((double)m / (double)kept.mt));
      }
      return;
    }
  }
  if (!(fabsf(top) < 8388608.f)) longway = true;  // the bins beside it have to be exact
  if (!longway && far_below(least, wg.best, wg.inv_t, kClear)) {
    // Beside the row's best a token may weigh nothing although its chunk counted it. Whole chunks leave first, then the
    // row is counted (8 cold rows of 128256 tokens: 21 us, against 8 at a temperature where no token is so far below).
    auto add_up = [&]() {
      const int n = block_scan(finite, 0, sh.scan_c, sh.scan_m).ct;
      __syncthreads();
      for (int o = 1; o < kWave; o <<= 1) least = fminf(least, __shfl_xor(least, o, kWave));
      if (lane == 0) sh.x[wave] = least;
      __syncthreads();
      for (int w = 0; w < kWaves; ++w) least = fminf(least, sh.x[w]);
      finite = n;
    };
    least = INFINITY;
    finite = 0;
    for (int c = tid; c < a.chunks; c += kThreads) {
      const ChunkStat st = stat[c];
      if (far_below(st.best, wg.best, wg.inv_t, kNothing)) continue;
      least = fminf(least, st.least);
      finite += st.finite;
    }
    add_up();
    if (far_below(least, wg.best, wg.inv_t, kClear)) {
      finite = 0;
      for (int v0 = 4 * tid; v0 < V; v0 += 4 * kThreads) {
        float x[4];
        load4<ALIGNED>(row, V, v0, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) finite += far_below(x[e], wg.best, wg.inv_t, kNothing) ? 0 : 1;
      }
      add_up();
    }
  }
  // a mass in units of a chunk's best, in the row's
  auto scaled = [&](u64 m, int c) { return (u64)rint((double)m * sh.scale[c]); };
  if (!longway && q.mode != kByList) {
    __syncthreads();
    for (int c = tid; c < a.chunks; c += kThreads) {
      const float from = stat[c].best;
      const bool has = !far_below(from, wg.best, wg.inv_t, kNothing);
      sh.off[c] = has ? top - bin_of(from, s) : INFINITY;
      sh.scale[c] = has ? exp_nonpos(((double)from - (double)best) * wg.inv_t) : 0.0;
    }
    __syncthreads();
  }
  const u64* sums = a.list + (size_t)b * a.chunks * kList;
  // the mass of chunk c up to the end of its bin j
  auto mass_to = [&](int c, float j) { return j >= 0.f ? scaled(sums[(size_t)c * kList + (int)j], c) : 0; };
  u64 cutoff = 0;        // tokens whose (key, ~index) reaches this stay
  int kept = finite;
  int lo = 0, hi = -1;   // the bins whose tokens are in sh.sorted; the bins in front of them stay whole
  if (q.mode == kByBins && !longway) {
    const int last = last_bin(q, V);
    u64 total = 0;
    for (int c = tid; c < a.chunks; c += kThreads) total += scaled(stat[c].mass, c);
    total = block_scan(0, total, sh.scan_c, sh.scan_m).mt;
    {  // half of the threads each take every second chunk of a bin
      static_assert(kThreads == 2 * kFine, "two threads a bin");
      constexpr int kAhead = 16;
      const int bin = tid & (kFine - 1);
      u64 m = 0;
      int n = 0;
      for (int c0 = tid / kFine; c0 < a.chunks; c0 += 2 * kAhead) {
        u64 pm[kAhead];
        int pn[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = min(c0 + 2 * k, a.chunks - 1), j = max((int)fmaxf((float)bin - sh.off[c], -1.f), 0);
          pm[k] = sums[(size_t)c * kList + j];
          pn[k] = (int)reinterpret_cast<const uint32_t*>(sums + (size_t)c * kList + kFine)[j];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = c0 + 2 * k;
          if (c < a.chunks && (float)bin - sh.off[c] >= 0.f) {
            m += scaled(pm[k], c);
            n += pn[k];
          }
        }
      }
      if (tid == 0) {
        sh.cum_mass[0] = 0;
        sh.cum_count[0] = 0;
      }
      if (tid < kFine) {
        sh.cum_mass[bin + 1] = m;
        sh.cum_count[bin + 1] = n;
      }
      __syncthreads();
      if (tid >= kFine) {
        sh.cum_mass[bin + 1] += m;
        sh.cum_count[bin + 1] += n;
      }
      __syncthreads();
    }
    int above_c = 0;  // tokens and mass in front of bin lo
    u64 above = 0;
    // The first bin whose end reaches `want` tokens (want > 0) or `share` units; -1: none.
    auto find = [&](int want, double share) {
      if (tid == 0) sh.bin = -1;
      __syncthreads();
      if (tid <= last && (want > 0 ? sh.cum_count[tid] < want && sh.cum_count[tid + 1] >= want
                                   : (double)sh.cum_mass[tid] < share && (double)sh.cum_mass[tid + 1] >= share))
        sh.bin = tid;
      __syncthreads();
      const int bin = sh.bin;
      __syncthreads();
      return bin;
    };
    // Bins b0 .. b1 into sh.sorted. false: too many tokens.
    auto gather = [&](int b0, int b1) {
      if (b0 == lo && b1 == hi) return true;
      lo = b0;
      hi = b1;
      __syncthreads();
      if (tid == 0) sh.n = 0;
      __syncthreads();
      above_c = sh.cum_count[b0];
      above = sh.cum_mass[b0];
      // Pieces of 2048 tokens, one wave each; the next piece is on its way while one is looked through. Chunks
      // whose best lies behind the bins are passed over.
      constexpr int kAhead = 8, kPiece = 4 * kAhead * kWave;
      const int pieces = (V + kPiece - 1) / kPiece;
      auto next = [&](int p) {
        while (p < pieces && !(sh.off[p * kPiece / a.chunk] <= (float)b1)) p += kWaves;
        return p;
      };
      auto fetch = [&](int p, float (&x)[kAhead][4]) {
        if (ALIGNED && (p + 1) * kPiece <= V) {  // uniform: loads under no condition, all on their way together
#pragma unroll
          for (int k = 0; k < kAhead; ++k) load4_whole(row + p * kPiece + 4 * (lane + k * kWave), x[k]);
        } else {
#pragma unroll
          for (int k = 0; k < kAhead; ++k) load4<ALIGNED>(row, p < pieces ? V : 0, p * kPiece + 4 * (lane + k * kWave), x[k]);
        }
      };
      // The bins as a range of logits: the outermost ones that floor(x s) puts there
      const float low = logit_of(first_key([&](float x) { return top - bin_of(x, s) <= (float)b1; }));
      const float high = logit_of(first_key([&](float x) { return top - bin_of(x, s) < (float)b0; }) - 1);
      // each wave lists what it finds in its own part of the room; one that runs over sends the row the long way
      constexpr int kRoom = kSort / kWaves;
      int found = 0;
      auto look = [&](int p, const float (&x)[kAhead][4]) {
#pragma unroll
        for (int k = 0; k < 4 * kAhead; ++k) {
          const float y = x[k >> 2][k & 3];
          const bool in = (y >= low) & (y <= high);  // no NaN, no infinity
          const uint64_t hit = __ballot(in);
          if (hit == 0) continue;  // uniform
          const int at = found + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
          if (in && at < kRoom)
            sh.sorted[wave * kRoom + at] = (u64)key_of(y) << 32 | ~(uint32_t)(p * kPiece + 4 * (lane + (k >> 2) * kWave) + (k & 3));
          found += __popcll(hit);
        }
      };
      float xa[kAhead][4], xb[kAhead][4];
      int p = next(wave);
      fetch(p, xa);
      while (p < pieces) {
        const int p2 = next(p + kWaves);
        fetch(p2, xb);
        look(p, xa);
        if (p2 >= pieces) break;
        p = next(p2 + kWaves);
        fetch(p, xa);
        look(p2, xb);
      }
      if (lane == 0) sh.i[wave] = found;
      __syncthreads();
      u64 mine[kRoom / kWave];  // the parts moved together
#pragma unroll
      for (int k = 0; k < kRoom / kWave; ++k) mine[k] = sh.sorted[wave * kRoom + k * kWave + lane];
      int from = 0, n = 0;
      bool over = false;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) from += sh.i[w];
        n += sh.i[w];
        over |= sh.i[w] > kRoom;
      }
      __syncthreads();
      if (over) return false;
#pragma unroll
      for (int k = 0; k < kRoom / kWave; ++k)
        if (k * kWave + lane < found) sh.sorted[from + k * kWave + lane] = mine[k];
      if (tid == 0) sh.n = n;
      __syncthreads();
      return true;
    };
    // The last of the gathered tokens (in order) that stays and how many do, by count (want > 0: of them) or by
    // the mass in front (share): counts and masses by 256 steps of the keys, then the tokens of the step
    // that holds the cut, sorted.
    auto select = [&](int want, double share, u64& at) {
      u64* const mass = sh.chunk_mass;  // not in use yet
      uint32_t* const count = reinterpret_cast<uint32_t*>(sh.chunk_mass + kFine);
      u64* const small = sh.chunk_mass + 2 * kFine;
      constexpr int kSmall = kMaxChunks - 2 * kFine;
      const int n = sh.n;
      uint32_t least = 0xffffffffu, most = 0;
      for (int i = tid; i < n; i += kThreads) {
        const uint32_t key = (uint32_t)(sh.sorted[i] >> 32);
        least = min(least, key);
        most = max(most, key);
      }
      for (int o = 1; o < kWave; o <<= 1) {
        least = min(least, (uint32_t)__shfl_xor((int)least, o, kWave));
        most = max(most, (uint32_t)__shfl_xor((int)most, o, kWave));
      }
      if (lane == 0) sh.scan_m[wave] = (u64)most << 32 | least;
      if (tid < kFine) {
        mass[tid] = 0;
        count[tid] = 0;
      }
      if (tid == 0) sh.bc = -1;
      __syncthreads();
      for (int w = 0; w < kWaves; ++w) {
        least = min(least, (uint32_t)sh.scan_m[w]);
        most = max(most, (uint32_t)(sh.scan_m[w] >> 32));
      }
      const int bits = max(32 - __clz((int)(most - least)), 8) - 8;  // the keys' range in 256 steps
      for (int i = tid; i < n; i += kThreads) {
        const uint32_t key = (uint32_t)(sh.sorted[i] >> 32);
        atomicAdd(&count[(most - key) >> bits], 1u);
        if (want == 0) atomicAdd(&mass[(most - key) >> bits], wg.units(wg.weight(logit_of(key))));
      }
      __syncthreads();
      const int c = tid < kFine ? (int)count[tid] : 0;
      const u64 m = tid < kFine ? mass[tid] : 0;
      const Scan sc = block_scan(c, m, sh.scan_c, sh.scan_m);
      const bool holds = want > 0 ? sc.c - c < want && sc.c >= want : (double)(above + sc.m - m) < share && ((double)(above + sc.m) >= share || sc.c == n);
      if (c > 0 && holds) {
        sh.bc = tid;
        sh.bin = sc.c - c;
        sh.bm = above + sc.m - m;
      }
      __syncthreads();
      const int step = sh.bc, front = sh.bin, here = step < 0 ? 0 : (int)count[step];
      const u64 ahead = sh.bm;
      if (step < 0) return 0;
      __syncthreads();
      u64* list = small;
      if (here <= kSmall / 2) {  // the sort wants a power of two
        if (tid == 0) sh.bin = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
          if ((int)((most - (uint32_t)(sh.sorted[i] >> 32)) >> bits) == step) small[atomicAdd(&sh.bin, 1)] = sh.sorted[i];
        __syncthreads();
        sort_down(small, here);
      } else {  // crowded (ties): all of them in order, those of the step behind the ones in front
        sort_down(sh.sorted, n);
        list = sh.sorted + front;
      }
      int stay = 0;
      if (want > 0) {
        stay = want - front;
      } else {
        u64 run = ahead;
        for (int i0 = 0; i0 < here; i0 += kThreads) {
          const int i = i0 + tid;
          const u64 w = i < here ? wg.units(wg.weight(logit_of((uint32_t)(list[i] >> 32)))) : 0;
          const Scan t = block_scan(0, w, sh.scan_c, sh.scan_m);
          stay += block_scan(i < here && (double)(run + t.m - w) < share ? 1 : 0, 0, sh.scan_c, sh.scan_m).ct;
          run += t.mt;
        }
        stay = max(stay, 1);
      }
      at = list[stay - 1];
      __syncthreads();
      return front + stay;
    };
    if (q.top_k > 0 && finite > q.top_k) {
      const int bin = find(q.top_k, 0.0);
      if (bin < 0 || !gather(bin, bin)) {
        longway = true;
      } else {
        kept = q.top_k;
        select(kept - above_c, 0.0, cutoff);
        u64 m = 0;
        for (int i = tid; i < sh.n; i += kThreads)
          if (sh.sorted[i] >= cutoff) m += wg.units(wg.weight(logit_of((uint32_t)(sh.sorted[i] >> 32))));
        total = above + block_scan(0, m, sh.scan_c, sh.scan_m).mt;
      }
    }
    // the lightest logit that min_p leaves lies in bin `edge` or, for its rounding, beside it
    const float xm = q.min_p > 0.f ? (float)((double)best + (double)q.temp * log((double)q.min_p)) : -INFINITY;
    const float edge = fmaxf(top - bin_of(xm, s), 0.f);
    const bool by_m = edge < (float)last;  // else behind the bins: it cuts nothing that another cut leaves
    const int m0 = max((int)fminf(edge, (float)last) - 1, 0), m1 = min((int)fminf(edge, (float)last) + 1, last);
    const int pbin = q.top_p < 1.f && !longway ? find(0, (double)q.top_p * (double)total) : -1;
    // p cuts in front of all that m may cut, m in front of p's bin, or both in one range of bins
    const bool only_p = pbin >= 0 && (!by_m || pbin < m0), only_m = by_m && (pbin < 0 || m1 < pbin);
    // a cut that lies behind the bins, and none in front of it
    if (cutoff == 0 && (q.top_p < 1.f || q.min_p > 0.f) && pbin < 0 && !by_m) longway = true;
    if (!longway && (pbin >= 0 || by_m)) {
      const int g0 = only_p ? pbin : only_m ? m0 : min(pbin, m0), g1 = only_p ? pbin : only_m ? m1 : max(pbin, m1);
      if (!gather(g0, g1)) {
        longway = true;
      } else {
        if (!only_m) {
          u64 at = 0;
          const int n = select(0, (double)q.top_p * (double)total, at);
          if (n > 0 && above_c + n < kept) {
            kept = above_c + n;
            cutoff = at;
          }
        }
        if (!only_p) {  // the tokens that weigh enough, and the last of them
          int n = 0;
          u64 at = ~0ull;
          for (int i = tid; i < sh.n; i += kThreads) {
            const u64 e = sh.sorted[i];
            if (wg.weight(logit_of((uint32_t)(e >> 32))) >= (double)q.min_p) {
              ++n;
              at = min(at, e);
            }
          }
          for (int o = 1; o < kWave; o <<= 1) at = min(at, (u64)__shfl_xor((unsigned)(at >> 32), o, kWave) << 32 | __shfl_xor((unsigned)at, o, kWave));
          n = block_scan(n, 0, sh.scan_c, sh.scan_m).ct;
          __syncthreads();
          if (lane == 0) sh.scan_m[wave] = at;
          __syncthreads();
          for (int w = 0; w < kWaves; ++w) at = min(at, sh.scan_m[w]);
          __syncthreads();
          if (above_c + n < kept) {
            kept = above_c + n;
            if (n > 0) {
              cutoff = at;
            } else {  // none: everything above the gathered bins stays
              u64 most = 0;
              for (int i = 0; i < sh.n; ++i) most = max(most, sh.sorted[i]);
              cutoff = sh.n > 0 ? most + 1 : (u64)key_of(xm) << 32;
            }
          }
        }
      }
    }
    if (!longway && cutoff != 0) {  // the cut's bin among the gathered ones
      const int bin = (int)(top - bin_of(logit_of((uint32_t)(cutoff >> 32)), s));
      if ((bin < lo || bin > hi) && (bin < 0 || bin > last || !gather(bin, bin))) longway = true;
    }
  }
  if (longway || q.mode == kByList) {
    __syncthreads();
    row_cut<ALIGNED>(a, q, wg, b, sh);
    return;
  }
  // ---- the chunks' kept masses, the chunk of the draw
  for (int c = tid; c < a.chunks; c += kThreads)
    sh.chunk_mass[c] = cutoff == 0 ? scaled(stat[c].mass, c) : mass_to(c, (float)(lo - 1) - sh.off[c]);
  __syncthreads();
  if (cutoff != 0)
    for (int i = tid; i < sh.n; i += kThreads) {
      const u64 e = sh.sorted[i];
      if (e >= cutoff) atomicAdd(&sh.chunk_mass[~(uint32_t)e / (uint32_t)a.chunk], wg.units(wg.weight(logit_of((uint32_t)(e >> 32)))));
    }
  __syncthreads();
  constexpr int kPer = kMaxChunks / kThreads;
  u64 cm[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) sum += cm[k] = kPer * tid + k < a.chunks ? sh.chunk_mass[kPer * tid + k] : 0;
  const Scan cs = block_scan(0, sum, sh.scan_c, sh.scan_m);
  const double target = share_u * (double)cs.mt;
  u64 run = cs.m - sum;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (cm[k] > 0 && (double)run <= target && ((double)(run + cm[k]) > target || run + cm[k] == cs.mt)) {
      sh.bin = kPer * tid + k;
      sh.bm = run;
    }
    run += cm[k];
  }
  __syncthreads();
  // ---- its tokens, the same number to each thread
  const int c = sh.bin, each = a.chunk / kThreads, first = c * a.chunk + tid * each;
  const double share = (target - (double)sh.bm) / (double)sh.chunk_mass[c];  // of its kept mass
  u64 m = 0;
  for (int e = 0; e < each; ++e) {
    const int v = first + e;
    const float x = v < V ? row[v] : -INFINITY;
    if (x > -INFINITY && ((u64)key_of(x) << 32 | ~(uint32_t)v) >= cutoff) m += wg.units(wg.weight(x));
  }
  const Scan ts = block_scan(0, m, sh.scan_c, sh.scan_m);
  if (ts.mt == 0) {  // uniform: tokens that make up units together, none alone (u at 1, a tail far down)
    __syncthreads();
    row_cut<ALIGNED>(a, q, wg, b, sh);
    return;
  }
  // The chunk's own sum may be off its mass in the row's units (tokens of half a unit count as one each here): the same
  // share of it, and at u = 1, whatever these quotients round to, the last token of positive mass.
  const double rest = share_u < 1.0 ? share * (double)ts.mt : INFINITY;
  if (m > 0 && (double)(ts.m - m) <= rest && ((double)ts.m > rest || ts.m == ts.mt)) {
    u64 before = ts.m - m;
    for (int e = 0; e < each; ++e) {
      const int v = first + e;
      const float x = v < V ? row[v] : -INFINITY;
      if (!(x > -INFINITY) || ((u64)key_of(x) << 32 | ~(uint32_t)v) < cutoff) continue;
      const u64 w = wg.units(wg.weight(x));
      before += w;
      if (w > 0 && ((double)before > rest || before == ts.mt)) {
        answer(v, kept, (float)((double)w / (double)cs.mt));
        break;
      }
    }
  }
}

}  // namespace

// Tokens per chunk: 8192, or 2048 where a call has fewer chunks than CUs of them (both kernels, filters without a
// top_k: one row of 128256 tokens 28.6 us by 2048, 32.5 by 8192; 16 rows 58.7 and 58.3; 64 rows 82 and 72).
static int chunk_of(int B, int V) { return (long)B * ceil_div(V, 8192) < 256 && ceil_div(V, 2048) <= kMaxChunks ? 2048 : 8192; }

static SampleLayout layout_of(size_t chunks) {
  SampleLayout L{};
  Carve c;
  L.stat = c.take(chunks * sizeof(ChunkStat));
  L.list = c.take(chunks * kList * sizeof(u64));
  L.total = c.off;
  return L;
}

SampleLayout sample_layout(int B, int V) { return layout_of((size_t)B * ceil_div(V, chunk_of(B, V))); }

// What every call of at most B rows of at most V tokens needs. A call has chunks of 2048 only where it has at most 255
// of 8192, so at most four times as many of them: sizes grow with both arguments, over the border of the rule too.
size_t sample_workspace(int B, int V) {
  const size_t large = (size_t)B * ceil_div(V, 8192), small = (size_t)B * ceil_div(V, 2048);
  return layout_of(std::max(large, std::min<size_t>(small, 4 * 255))).total;
}

long sample_grid(int B, int V) { return (long)B * ceil_div(V, chunk_of(B, V)); }

hipError_t launch_sample(const SampleCall& c, char* ws, const SampleLayout& L, hipStream_t stream) {
  Args a{};
  a.logits = c.logits; a.ld = c.ld; a.V = c.V;
  a.u = c.u; a.temperature = c.temperature; a.top_k = c.top_k; a.top_p = c.top_p; a.min_p = c.min_p;
  a.token = c.token; a.kept = c.kept; a.prob = c.prob;
  int bits = 0;
  while ((1 << bits) < c.V) ++bits;
  a.shift = std::min(62 - bits, 50);
  a.tile = kTile * ceil_div(ceil_div(c.V, kTile), kTiles);
  a.chunk = chunk_of(c.B, c.V);
  a.chunks = ceil_div(c.V, a.chunk);
  a.stat = reinterpret_cast<ChunkStat*>(ws + L.stat);
  a.list = reinterpret_cast<u64*>(ws + L.list);
  const bool aligned = c.ld % 4 == 0 || c.B == 1;
  {
    ProfScope prof("sample_chunk", stream);
    const int grid = c.B * a.chunks;
    if (a.chunk == 2048) {
      if (aligned) klaunch(sample_chunk_kernel<true, 512, 1>, grid, 512, 0, stream, a);
      else klaunch(sample_chunk_kernel<false, 512, 1>, grid, 512, 0, stream, a);
    } else {
      if (aligned) klaunch(sample_chunk_kernel<true, 256, 8>, grid, 256, 0, stream, a);
      else klaunch(sample_chunk_kernel<false, 256, 8>, grid, 256, 0, stream, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope prof("sample_finish", stream);
  if (aligned) klaunch(sample_finish_kernel<true>, c.B, kThreads, 0, stream, a);
  else klaunch(sample_finish_kernel<false>, c.B, kThreads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace sirius
