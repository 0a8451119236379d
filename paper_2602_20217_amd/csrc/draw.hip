// Draw of one token per logits row from a given uniform, every row with its own
// temperature, top-k, min-p and top-p, any k up to the vocabulary.
//
// Order a row's entries by decreasing logit, equal ones by id.  Every filter keeps
// a prefix of that order (top-k a length, min-p a value, top-p a probability mass),
// and the draw is the first entry whose cumulative mass exceeds u times the mass
// kept.  So nothing has to be sorted: each step is the search for a place in the
// order by its rank or by its mass.
//
// The mass of an entry is e^x, x = (logit - largest) / temperature, computed in 64
// bits and held as an integer in units of 2^-44: sums of integers do not depend on
// the order of the atomics that add them, and what neighbours of the draw differ by
// is kept (float32 sums lose it).  Entries below e^-31 of the largest have mass 0.
//
//  k_draw_max     largest logit of every chunk of a row; clears the row's histogram
//  k_draw_hist    count and mass of every bin of width 1/64 in x, over the row
//  k_draw_gather  the bins that hold the places searched for follow from the
//                 histogram (a few when one search depends on the one before);
//                 their entries are gathered
//  k_draw_pick    sorts the gathered entries and finds the places; a row whose bins
//                 hold too many (equal logits, high temperature) finds each place
//                 digit by digit over the whole row instead
#include "ks_internal.h"

#include <algorithm>
#include <cfloat>

namespace ks {

namespace {

constexpr int BINS = 2048;
constexpr double BIN_W = 64.0;  // bins per unit of x; the last one has no lower end
constexpr double X_MIN = -32.0;
constexpr int FRAC = 44;        // fraction bits of a mass: 2^19 entries of mass 1 fit 63 bits
constexpr int CAP = 4096;       // gathered entries of a row
constexpr int SCAN_T = 256;     // threads of a chunk workgroup
constexpr int PICK_T = 1024;    // threads of a row's last workgroup
constexpr int NB_MAX = 128;     // chunks of a row

typedef unsigned long long u64;

// One row's scratch.
struct RowWs {
  u64 mass[BINS];
  u64 cand[CAP];
  uint32_t cnt[BINS];
  float cmax[NB_MAX];
  uint32_t n_cand;
  uint32_t pad[3];
};

__device__ inline float ld_logit(const float* p) { return *p; }
__device__ inline float ld_logit(const bf16_t* p) { return bf2f(*p); }

// Unsigned order of float32 (-0 as +0).
__device__ inline uint32_t order_key(float f) {
  uint32_t u = __float_as_uint(f);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ inline float key_logit(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
// An entry as one integer, larger first in the order.
__device__ inline u64 entry_of(float l, int id) {
  return ((u64)order_key(l) << 32) | (uint32_t)~id;
}

// f(logit, id) for the ids [n0, n1) of a row, by NT threads.
template <int NT, typename T, typename F>
__device__ inline void each_logit(const T* row, int n0, int n1, F f) {
  constexpr int E = 16 / sizeof(T);
  if (((uintptr_t)(row + n0) & 15) == 0) {
    const int nv = (n1 - n0) / E;
#pragma unroll 2
    for (int i = threadIdx.x; i < nv; i += NT) {
      T x[E];
      *(uint4*)x = *(const uint4*)(row + n0 + E * i);
#pragma unroll
      for (int e = 0; e < E; ++e) f(ld_logit(&x[e]), n0 + E * i + e);
    }
    n0 += nv * E;
  }
  for (int i = n0 + threadIdx.x; i < n1; i += NT) f(ld_logit(row + i), i);
}

// A row's settings, with what switches a filter off put as what never cuts.
struct Setting {
  double inv_t, min_p, top_p, u;
  uint32_t k;
  float lmax;
  __device__ bool entry(float l) const { return l > -INFINITY; }  // not barred, not NaN
  __device__ double x_of(float l) const {
    return l == lmax ? 0.0 : ((double)l - (double)lmax) * inv_t;
  }
  __device__ int bin_of(double x) const {
    return x > X_MIN ? min((int)(-x * BIN_W), BINS - 1) : BINS - 1;
  }
  // mass of an entry; keep: min-p keeps it
  __device__ u64 mass_of(double x, bool& keep) const {
    keep = true;
    double w = 0.0;
    if (x > X_MIN || min_p > 0.0) {
      w = exp(x);
      keep = w >= min_p;
    }
    // adding 2^52 rounds to an integer in the low mantissa bits
    return (u64)__double_as_longlong(fma(w, (double)(1ull << FRAC), 4503599627370496.0)) &
           ((1ull << 52) - 1);
  }
};
__device__ inline Setting setting(const DrawArgs& a, int r, float lmax) {
  Setting s;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(t > 0.f);
  const int k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
  const float mp = greedy || !a.min_p ? 0.f : a.min_p[r];
  const float tp = greedy || !a.top_p ? 1.f : a.top_p[r];
  const float u = a.u[r];
  s.inv_t = greedy ? 1.0 : 1.0 / (double)t;
  s.k = k > 0 ? (uint32_t)k : 0xFFFFFFFFu;
  s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
  s.top_p = tp < 1.f ? fmax((double)tp, 0.0) : 1.0;
  s.u = u > 0.f ? (double)u : 0.0;
  s.lmax = lmax;
  return s;
}
// masses are in [0, 2^63]: the first cumulative mass that reaches p z, and the first
// that exceeds u z, as the least integer that does
__device__ inline u64 reach(double p, u64 z) {
  return max((u64)ceil(p * (double)z), (u64)1);
}
__device__ inline u64 exceed(double u, u64 z) {
  const u64 t = (u64)(u * (double)z);
  return min(t + 1, z);
}

template <typename V>
__device__ inline V wave_incl(V v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V y = __shfl_up(v, o);
    if ((int)(threadIdx.x & 63) >= o) v += y;
  }
  return v;
}
// Inclusive prefix over the NT threads of a workgroup.
template <int NT, typename V>
__device__ inline V block_incl(V v, V* sh) {
  v = wave_incl(v);
  const int w = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sh[w] = v;
  __syncthreads();
  for (int i = 0; i < w; ++i) v += sh[i];
  return v;
}

// The histogram of a row as inclusive sums, BINS / NT bins a thread.
template <int NT>
struct Sums {
  static constexpr int E = BINS / NT;
  u64 m[E];
  uint32_t c[E];
};
// The first bin whose inclusive sum reaches thr, and the sum before it.
template <int NT, typename V>
__device__ inline int first_bin(const V (&incl)[BINS / NT], V thr, V* s_before, int* s_bin) {
  constexpr int E = BINS / NT;
  __syncthreads();
  if (threadIdx.x == 0) *s_bin = BINS - 1;
  __syncthreads();
  V before = 0;
  {
    // the inclusive sum of the thread before
    __shared__ V s_last[NT];
    s_last[threadIdx.x] = incl[E - 1];
    __syncthreads();
    if (threadIdx.x > 0) before = s_last[threadIdx.x - 1];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (before < thr && thr <= incl[e]) {
      *s_bin = threadIdx.x * E + e;
      *s_before = before;
    }
    before = incl[e];
  }
  __syncthreads();
  return *s_bin;
}

// What the histogram says of the places: the bins that hold the k-th entry, the end
// of top-p's prefix and the draw, as ranges where one depends on another's exact
// place inside its bin.
struct Plan {
  uint32_t total;  // entries that min-p keeps
  u64 z;           // their mass
  int k_bin;       // bin of the k-th entry; -1: it cuts no mass
  int p_lo, p_hi, d_lo, d_hi;
  __device__ bool wants(int b) const {
    return b == k_bin || (b >= p_lo && b <= p_hi) || (b >= d_lo && b <= d_hi);
  }
};
template <int NT>
__device__ inline Plan plan(const RowWs& w, const Setting& s, Sums<NT>& h) {
  constexpr int E = BINS / NT;
  __shared__ u64 s_m[NT / 64];
  __shared__ uint32_t s_c[NT / 64];
  __shared__ u64 s_bm, s_z;
  __shared__ uint32_t s_bc, s_n;
  __shared__ int s_bin;
  u64 m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    m += w.mass[threadIdx.x * E + e];
    c += w.cnt[threadIdx.x * E + e];
    h.m[e] = m;
    h.c[e] = c;
  }
  const u64 mi = block_incl<NT>(m, s_m) - m;
  const uint32_t ci = block_incl<NT>(c, s_c) - c;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    h.m[e] += mi;
    h.c[e] += ci;
  }
  if (threadIdx.x == NT - 1) {
    s_z = h.m[E - 1];
    s_n = h.c[E - 1];
  }
  __syncthreads();
  Plan p;
  p.total = s_n;
  p.z = s_z;
  // inclusive and exclusive mass of a bin, to every thread
  auto mass_at = [&](int b, u64& before) {
    __syncthreads();
    if ((int)threadIdx.x == b / E) {
      u64 x = 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e == b % E) x = h.m[e];
      s_bm = x;
    }
    __syncthreads();
    const u64 incl = s_bm;
    before = incl - w.mass[b];
    return incl;
  };
  u64 zlo = p.z, zhi = p.z;  // mass that top-k keeps
  p.k_bin = -1;
  if (s.k < p.total) {
    const int b = first_bin<NT>(h.c, s.k, &s_bc, &s_bin);
    zhi = mass_at(b, zlo);
    if (zhi > zlo) p.k_bin = b;
  }
  p.p_lo = p.d_lo = BINS;
  p.p_hi = p.d_hi = -1;
  if (s.top_p < 1.0) {
    u64 before;
    p.p_lo = first_bin<NT>(h.m, reach(s.top_p, zlo), &s_bm, &s_bin);
    p.p_hi = first_bin<NT>(h.m, reach(s.top_p, zhi), &s_bm, &s_bin);
    const u64 top = mass_at(p.p_hi, before);
    mass_at(p.p_lo, before);
    zlo = before + 1;
    zhi = min(zhi, top);
  }
  p.d_lo = first_bin<NT>(h.m, exceed(s.u, max(zlo, (u64)1)), &s_bm, &s_bin);
  p.d_hi = first_bin<NT>(h.m, exceed(s.u, zhi), &s_bm, &s_bin);
  return p;
}

// grid (chunks, rows)
template <typename T>
__global__ __launch_bounds__(SCAN_T) void k_draw_max(DrawArgs a, int chunk) {
  __shared__ float s_m[SCAN_T / 64];
  const int b = blockIdx.x, NB = gridDim.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  for (int i = b * SCAN_T + threadIdx.x; i < BINS; i += NB * SCAN_T) {
    w.mass[i] = 0;
    w.cnt[i] = 0;
  }
  if (b == 0 && threadIdx.x == 0) w.n_cand = 0;
  float m = -INFINITY;
  each_logit<SCAN_T>((const T*)a.logits + (size_t)r * a.ld, b * chunk,
                     min(a.vocab, (b + 1) * chunk), [&](float l, int) { m = fmaxf(m, l); });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) s_m[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < SCAN_T / 64; ++i) m = fmaxf(m, s_m[i]);
    w.cmax[b] = m;
  }
}

// largest logit of the row, to every lane
__device__ inline float row_max(const RowWs& w, int NB) {
  float m = -INFINITY;
  for (int i = threadIdx.x & 63; i < NB; i += 64) m = fmaxf(m, w.cmax[i]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  return m;
}

template <typename T>
__global__ __launch_bounds__(SCAN_T) void k_draw_hist(DrawArgs a, int chunk) {
  __shared__ u64 s_mass[BINS];
  __shared__ uint32_t s_cnt[BINS];
  const int b = blockIdx.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  const Setting s = setting(a, r, row_max(w, gridDim.x));
  if (!s.entry(s.lmax)) return;
  for (int i = threadIdx.x; i < BINS; i += SCAN_T) {
    s_mass[i] = 0;
    s_cnt[i] = 0;
  }
  __syncthreads();
  each_logit<SCAN_T>((const T*)a.logits + (size_t)r * a.ld, b * chunk,
                     min(a.vocab, (b + 1) * chunk), [&](float l, int) {
                       if (!s.entry(l)) return;
                       const double x = s.x_of(l);
                       bool keep;
                       const u64 m = s.mass_of(x, keep);
                       if (!keep) return;
                       const int bin = s.bin_of(x);
                       atomicAdd(&s_cnt[bin], 1u);
                       if (m) atomicAdd(&s_mass[bin], m);
                     });
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += SCAN_T) {
    if (!s_cnt[i]) continue;
    atomicAdd(&w.cnt[i], s_cnt[i]);
    if (s_mass[i]) atomicAdd(&w.mass[i], s_mass[i]);
  }
}

template <typename T>
__global__ __launch_bounds__(SCAN_T) void k_draw_gather(DrawArgs a, int chunk) {
  const int b = blockIdx.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  const Setting s = setting(a, r, row_max(w, gridDim.x));
  if (!s.entry(s.lmax)) return;
  Sums<SCAN_T> h;
  const Plan p = plan<SCAN_T>(w, s, h);
  each_logit<SCAN_T>((const T*)a.logits + (size_t)r * a.ld, b * chunk,
                     min(a.vocab, (b + 1) * chunk), [&](float l, int id) {
                       if (!s.entry(l)) return;
                       const double x = s.x_of(l);
                       if (!p.wants(s.bin_of(x))) return;
                       bool keep;
                       s.mass_of(x, keep);
                       if (!keep) return;
                       const uint32_t at = atomicAdd(&w.n_cand, 1u);
                       if (at < CAP) w.cand[at] = entry_of(l, id);
                     });
}

// The place searched for: the entry, and rank and cumulative mass up to it.
struct Place {
  u64 entry, cum;
  uint32_t rank;
};

// First entry, in order, of bin `bin` whose rank (by_mass: cumulative mass) reaches
// thr, with rank0 and cum0 before the bin: radix search over the row, 11 bits of
// the entry a pass (the id has at most 20 bits, so the order key's 32 bits and they
// take 5 passes).
template <typename T>
__device__ Place search(const T* row, int V, const Setting& s, int bin, bool by_mass, u64 thr,
                        uint32_t rank0, u64 cum0, u64* s_mass, uint32_t* s_cnt) {
  __shared__ u64 s_m[PICK_T / 64], s_bm;
  __shared__ uint32_t s_c[PICK_T / 64], s_bc;
  __shared__ int s_bin;
  constexpr int E = BINS / PICK_T;
  // the entry's bits from the top: key 31..21, 20..10, 9..0 with the id's complement
  // above bit 20 fixed, then 20..11 and 10..0 of the complement
  const int lo[5] = {53, 42, 32, 11, 0}, nb[5] = {11, 11, 10, 10, 11};
  u64 prefix = 0, fixed = 0;
  for (int d = 0; d < 5; ++d) {
    for (int i = threadIdx.x; i < BINS; i += PICK_T) {
      s_mass[i] = 0;
      s_cnt[i] = 0;
    }
    __syncthreads();
    const u64 mask = ((1ull << nb[d]) - 1) << lo[d];
    each_logit<PICK_T>(row, 0, V, [&](float l, int id) {
      if (!s.entry(l)) return;
      const double x = s.x_of(l);
      if (s.bin_of(x) != bin) return;
      const u64 e = entry_of(l, id);
      if ((e & fixed) != prefix) return;
      bool keep;
      const u64 m = s.mass_of(x, keep);
      if (!keep) return;
      // digits in decreasing order
      const int at = (int)((mask - (e & mask)) >> lo[d]);
      atomicAdd(&s_cnt[at], 1u);
      if (m) atomicAdd(&s_mass[at], m);
    });
    __syncthreads();
    u64 hm[E], m = 0;
    uint32_t hc[E], c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      m += s_mass[threadIdx.x * E + e];
      c += s_cnt[threadIdx.x * E + e];
      hm[e] = m;
      hc[e] = c;
    }
    const u64 mi = block_incl<PICK_T>(m, s_m) - m + cum0;
    const uint32_t ci = block_incl<PICK_T>(c, s_c) - c + rank0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      hm[e] += mi;
      hc[e] += ci;
    }
    const int at = by_mass ? first_bin<PICK_T>(hm, thr, &s_bm, &s_bin)
                           : first_bin<PICK_T>(hc, (uint32_t)thr, &s_bc, &s_bin);
    // rank and mass before the digit, and up to it
    __syncthreads();
    if ((int)threadIdx.x == at / E) {
      u64 x = 0;
      uint32_t y = 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e == at % E) {
          x = hm[e];
          y = hc[e];
        }
      s_bm = x - s_mass[at];
      s_bc = y - s_cnt[at];
    }
    __syncthreads();
    cum0 = s_bm;
    rank0 = s_bc;
    prefix |= mask - ((u64)at << lo[d]);
    fixed |= mask;
    if (d == 2) {  // ids lie below 2^20: the complement's other bits are ones
      const u64 ones = 0xFFFFFFFFull & ~((1ull << 21) - 1);
      prefix |= ones;
      fixed |= ones;
    }
    __syncthreads();
  }
  // one entry is left
  bool keep;
  const double x = s.x_of(key_logit((uint32_t)(prefix >> 32)));
  return Place{prefix, cum0 + s.mass_of(x, keep), rank0 + 1};
}

// one workgroup a row
template <typename T>
__global__ __launch_bounds__(PICK_T) void k_draw_pick(DrawArgs a, int NB) {
  __shared__ u64 s_e[CAP];  // entries in order; the radix search's masses
  __shared__ uint32_t s_x[BINS];
  __shared__ u64 s_gap[BINS];
  __shared__ u64 s_m[PICK_T / 64];
  __shared__ uint32_t s_c[PICK_T / 64];
  __shared__ int s_at;
  __shared__ u64 s_cum, s_ent;
  __shared__ uint32_t s_rank;
  const int r = blockIdx.x;
  RowWs& w = ((RowWs*)a.ws)[r];
  const Setting s = setting(a, r, row_max(w, NB));
  if (!s.entry(s.lmax)) {  // every token is barred
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = -INFINITY;
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  Sums<PICK_T> h;
  const Plan p = plan<PICK_T>(w, s, h);
  const uint32_t n = w.n_cand;
  u64 z = p.z;
  uint32_t kept = min(s.k, p.total);
  u64 ent = 0;
  if (n <= CAP) {
    // sort (decreasing), padded with zeros to a power of two
    int N = 64;
    while (N < (int)n) N <<= 1;
    for (int i = threadIdx.x; i < N; i += PICK_T) s_e[i] = i < (int)n ? w.cand[i] : 0;
    for (int k = 2; k <= N; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < N / 2; i += PICK_T) {
          const int x = 2 * i - (i & (j - 1)), y = x + j;
          const u64 ex = s_e[x], ey = s_e[y];
          if ((ex < ey) == ((x & k) == 0)) {
            s_e[x] = ey;
            s_e[y] = ex;
          }
        }
      }
    // counts and masses of the bins not gathered, up to each bin
    {
      constexpr int E = BINS / PICK_T;
      u64 m = 0, mm[E];
      uint32_t c = 0, cc[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int b = threadIdx.x * E + e;
        if (!p.wants(b)) {
          m += w.mass[b];
          c += w.cnt[b];
        }
        mm[e] = m;
        cc[e] = c;
      }
      const u64 mi = block_incl<PICK_T>(m, s_m) - m;
      const uint32_t ci = block_incl<PICK_T>(c, s_c) - c;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s_gap[threadIdx.x * E + e] = mm[e] + mi;
        s_x[threadIdx.x * E + e] = cc[e] + ci;
      }
    }
    __syncthreads();
    // rank and cumulative mass of each entry, CAP / PICK_T a thread
    constexpr int E = CAP / PICK_T;
    u64 cum[E], m = 0;
    uint32_t rank[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = threadIdx.x * E + e;
      if (i < (int)n) {
        bool keep;
        m += s.mass_of(s.x_of(key_logit((uint32_t)(s_e[i] >> 32))), keep);
      }
      cum[e] = m;
    }
    const u64 mi = block_incl<PICK_T>(m, s_m) - m;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = threadIdx.x * E + e;
      cum[e] += mi;
      rank[e] = i + 1;
      if (i < (int)n) {
        const int b = s.bin_of(s.x_of(key_logit((uint32_t)(s_e[i] >> 32))));
        cum[e] += s_gap[b];
        rank[e] += s_x[b];
      }
    }
    // first entry that reaches a rank or a mass
    auto find = [&](bool by_mass, u64 thr) {
      __syncthreads();
      if (threadIdx.x == 0) s_at = INT32_MAX;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = threadIdx.x * E + e;
        if (i < (int)n && (by_mass ? cum[e] >= thr : rank[e] >= (uint32_t)thr)) {
          atomicMin(&s_at, i);
          break;
        }
      }
      __syncthreads();
      const int at = min(s_at, (int)n - 1);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((int)threadIdx.x * E + e == at) {
          s_cum = cum[e];
          s_rank = rank[e];
          s_ent = s_e[at];
        }
      __syncthreads();
      return Place{s_ent, s_cum, s_rank};
    };
    if (p.k_bin >= 0) z = find(false, s.k).cum;
    if (s.top_p < 1.0) {
      const Place q = find(true, reach(s.top_p, z));
      z = q.cum;
      kept = q.rank;
    }
    ent = find(true, exceed(s.u, z)).entry;
  } else {
    const T* row = (const T*)a.logits + (size_t)r * a.ld;
    __shared__ u64 s_bm;
    __shared__ uint32_t s_bc;
    __shared__ int s_bin;
    constexpr int E = BINS / PICK_T;
    auto find = [&](bool by_mass, u64 thr) {
      const int b = by_mass ? first_bin<PICK_T>(h.m, thr, &s_bm, &s_bin)
                            : first_bin<PICK_T>(h.c, (uint32_t)thr, &s_bc, &s_bin);
      __syncthreads();
      if ((int)threadIdx.x == b / E) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e == b % E) {
            s_bm = h.m[e] - w.mass[b];
            s_bc = h.c[e] - w.cnt[b];
          }
      }
      __syncthreads();
      return search<T>(row, a.vocab, s, b, by_mass, thr, s_bc, s_bm, s_e, s_x);
    };
    if (p.k_bin >= 0) z = find(false, s.k).cum;
    if (s.top_p < 1.0) {
      const Place q = find(true, reach(s.top_p, z));
      z = q.cum;
      kept = q.rank;
    }
    ent = find(true, exceed(s.u, z)).entry;
  }
  if (threadIdx.x == 0) {
    a.tokens[r] = (int32_t)~(uint32_t)ent;
    const double x = s.x_of(key_logit((uint32_t)(ent >> 32)));
    if (a.logprob) a.logprob[r] = (float)(x - log((double)z * (1.0 / (double)(1ull << FRAC))));
    if (a.kept) a.kept[r] = (int32_t)kept;
  }
}

}  // namespace

size_t draw_ws_bytes(int rows) { return (size_t)rows * sizeof(RowWs); }

void draw_rows(const DrawArgs& a, hipStream_t st) {
  // chunks: about 1024 workgroups over the rows, of at least 1024 logits
  int NB = std::min(std::min(NB_MAX, (1024 + a.rows - 1) / a.rows), (a.vocab + 1023) / 1024);
  const int chunk = ((a.vocab + NB - 1) / NB + 7) / 8 * 8;
  NB = (a.vocab + chunk - 1) / chunk;
  const dim3 grid(NB, a.rows);
#define KS_DRAW(T_)                                                        \
  do {                                                                     \
    KS_LAUNCH(k_draw_max<T_>, grid, dim3(SCAN_T), 0, st, a, chunk);        \
    KS_LAUNCH(k_draw_hist<T_>, grid, dim3(SCAN_T), 0, st, a, chunk);       \
    KS_LAUNCH(k_draw_gather<T_>, grid, dim3(SCAN_T), 0, st, a, chunk);     \
    KS_LAUNCH(k_draw_pick<T_>, dim3(a.rows), dim3(PICK_T), 0, st, a, NB);  \
  } while (0)
  if (a.dtype == KS_BF16) KS_DRAW(bf16_t);
  else KS_DRAW(float);
#undef KS_DRAW
}

}  // namespace ks
