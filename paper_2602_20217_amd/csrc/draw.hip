// Draw of one token per logits row from a given uniform, every row with its own
// temperature, top-k, min-p and top-p, any k up to the vocabulary.
//
// Order a row's entries by decreasing logit, equal ones by id.  Every filter keeps
// a prefix of that order (top-k a length, min-p a value, top-p a probability mass),
// and the draw is the first entry whose cumulative mass exceeds u times the mass
// kept.  So nothing has to be sorted: each step is the search for a place in the
// order by its rank or by its mass.
//
// Entries fall into bins of width 1/64 in x = (logit - largest) / temperature, whose
// places 64 (largest - logit) / temperature are computed in 64 bits.  An entry's mass
// is e^-bin/64 times (1 - s), s = 1 - e^-r of its remainder r < 1/64, held in units of
// 2^-31.  A bin keeps its entries' number and the sum of s in one 64-bit word, so an
// entry costs one atomic, and sums of integers do not depend on the order of the
// atomics that make them.  Masses are known to about 2^-30 (sums of float32 would lose
// what neighbours of the draw differ by); bin masses and their sums are integers in
// units of 2^-44 of the largest entry's.  Entries below e^-31.98 have mass 0.
//
//  k_draw_max     largest logit of every chunk of a row; clears the row's bins
//  k_draw_hist    number and mass of every bin, over the row
//  k_draw_gather  the bins that hold the places searched for follow from these (a few
//                 when one search depends on the one before); their entries are
//                 gathered
//  k_draw_pick    orders the gathered entries and finds the places: up to 64 in one
//                 wave, up to CAP in a sort; a row whose bins hold more (equal logits,
//                 high temperature) finds each place digit by digit over the whole row
//
// 256 rows of 128256 logits (131 MB): 20 + 26 + 33 + 13 us, three readings
// at 3.9 to 6.7 TB/s that share the time with the bins' arithmetic, and the ordering of
// the densest row.  One such row: 3 + 5 + 7 + 4, the latency of four launches and their
// barriers.
#include "ks_internal.h"

#include <algorithm>
#include <cfloat>

namespace ks {

namespace {

constexpr int BINS = 2048;   // the last one has no lower end and no mass
constexpr double BIN_W = 64.0;
constexpr int FRAC = 44;     // fraction bits of a mass: 2^19 entries of mass 1 fit 63 bits
constexpr int UNIT = 31;     // fraction bits of s
constexpr int CNT_AT = 44;   // bits of a sum of s, below its number of entries
constexpr int CAP = 4096;    // gathered entries of a row
constexpr int SCAN_T = 256;  // threads of a chunk workgroup
constexpr int PICK_T = 1024; // threads of a row's last workgroup
constexpr int NB_MAX = 128;  // chunks of a row

typedef unsigned long long u64;

// What the bins say of the places: the bins that hold the k-th entry, the end of
// top-p's prefix and the draw, as ranges where one depends on another's exact place
// inside its bin.
struct Plan {
  u64 z;           // mass that min-p keeps
  uint32_t total;  // its entries
  int k_bin;       // bin of the k-th entry; -1: it cuts no mass
  int p_lo, p_hi, d_lo, d_hi;
  __device__ bool wants(int b) const {
    return b == k_bin || (b >= p_lo && b <= p_hi) || (b >= d_lo && b <= d_hi);
  }
};

// One row's scratch.
struct RowWs {
  u64 bin[BINS];       // entries << CNT_AT | sum of s
  u64 mass[BINS];      // up to and with each bin
  u64 cand[CAP];
  uint32_t cnt[BINS];  // up to and with each bin
  float cmax[NB_MAX];
  Plan plan;
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

// f(logit, id) for the ids [n0, n1) of a row, by NT threads; the next load is under
// way while one's logits are dealt with.  (Four at a time: 256 rows of 128256 22 us in
// k_draw_max for 20, 40 in k_draw_gather for 33, and 27 in k_draw_hist for 29.)
template <int NT, typename T, typename F>
__device__ inline void each_logit(const T* row, int n0, int n1, F f) {
  constexpr int E = 16 / sizeof(T);
  if (((uintptr_t)(row + n0) & 15) == 0) {
    const int nv = (n1 - n0) / E;
    const uint4* v = (const uint4*)(row + n0);
    uint4 q, next;
    if ((int)threadIdx.x < nv) next = v[threadIdx.x];
    for (int i = threadIdx.x; i < nv; i += NT) {
      q = next;
      if (i + NT < nv) next = v[i + NT];
      T x[E];
      *(uint4*)x = q;
#pragma unroll
      for (int e = 0; e < E; ++e) f(ld_logit(&x[e]), n0 + E * i + e);
    }
    n0 += nv * E;
  }
  for (int i = n0 + threadIdx.x; i < n1; i += NT) f(ld_logit(row + i), i);
}

// A row's settings, with what switches a filter off put as what never cuts.
struct Setting {
  double scale;   // 64 / temperature
  double y_max;   // min-p keeps entries up to it
  double top_p, u;
  uint32_t k;
  float lmax;
  __device__ static bool entry(float l) { return l > -INFINITY; }  // not barred, not NaN
  // 64 (largest - logit) / temperature
  __device__ double y_of(float l) const {
    return l == lmax ? 0.0 : ((double)lmax - (double)l) * scale;
  }
  // Bin of an entry and its remainder in units of 2^-31 of a bin, the last bin's 0; false
  // for what is no entry or falls to min-p.  Added to 2^21, a place has its bin and
  // remainder as the low bits of the sum.  (inf - inf is 0 here.)
  __device__ bool place(float l, int& bin, uint32_t& rem) const {
    const double y = ((double)lmax - (double)l) * scale;
    if (!entry(l) || y > y_max) return false;
    const double t = fmin(fmax(y, 0.0), (double)(BINS - 1)) + (double)(1 << (52 - UNIT));
    const u64 u = __double_as_longlong(t);
    bin = (int)(u >> UNIT) & (BINS - 1);
    rem = (uint32_t)u & ((1u << UNIT) - 1);
    return true;
  }
  __device__ int bin_of(float l) const {
    int b;
    uint32_t rem;
    return place(l, b, rem) ? b : BINS - 1;
  }
  // s of a remainder: 1 - e^-r = r (1 - r/2 (1 - r/3 (1 - r/4))) to 2^-31
  __device__ static uint32_t s_of(uint32_t rem) {
    const float x = (float)rem * (float)(1.0 / BIN_W);
    const float r = x * (1.0f / (1u << UNIT));
    return (uint32_t)fmaf(x, fmaf(r * -0.5f, fmaf(r * (-1.0f / 3), fmaf(r, -0.25f, 1.0f), 1.0f), 1.0f), 0.5f);
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
  s.scale = greedy ? BIN_W : BIN_W / (double)t;
  s.k = k > 0 ? (uint32_t)k : 0xFFFFFFFFu;
  s.y_max = mp > 0.f ? -BIN_W * log(fmin((double)mp, 1.0)) : (double)INFINITY;
  s.top_p = tp < 1.f ? fmax((double)tp, 0.0) : 1.0;
  s.u = u > 0.f ? fmin((double)u, 1.0) : 0.0;
  s.lmax = lmax;
  return s;
}
// units of mass that one unit of 1 - s has in a bin: e^-8i/64 e^-j/64, whose second
// factors are constants where a thread has bins in a row
__device__ inline double unit_of(int bin) {
  constexpr double W[8] = {1.0, 0.98449643700540845, 0.96923323447634413, 0.95420666596918835, 0.93941306281347581, 0.92484881321620482, 0.91051036138003416, 0.89639420663515046};
  return bin == BINS - 1 ? 0.0 : exp((bin >> 3) * (-8 / BIN_W)) * W[bin & 7] * (double)(1ull << (FRAC - UNIT));
}
// units of 1 - s of a bin's word, and their mass
__device__ inline u64 units_of(u64 w) {
  return ((w >> CNT_AT) << UNIT) - (w & ((1ull << CNT_AT) - 1));
}
__device__ inline u64 mass_of(double unit, u64 units) { return (u64)(unit * (double)units); }
// masses are in [0, 2^63]: the first cumulative mass that reaches p z, and the first
// that exceeds u z, as the least integer that does
__device__ inline u64 reach(double p, u64 z) { return max((u64)ceil(p * (double)z), (u64)1); }
__device__ inline u64 exceed(double u, u64 z) { return min((u64)(u * (double)z) + 1, z); }

template <typename V>
__device__ inline V wave_incl(V v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V y = __shfl_up(v, o);
    if ((int)(threadIdx.x & 63) >= o) v += y;
  }
  return v;
}
// Inclusive prefix over the NT threads of a workgroup, and the thread before's.
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

// The bin, if a thread has it, in which an inclusive sum first reaches a threshold; E bins
// a thread.  incl: the thread's inclusive sums, before: the sum before its first.
template <int E, typename V>
__device__ inline void own_bin(const V (&incl)[E], V before, V thr, int& at) {
  if (before >= thr || thr > incl[E - 1]) return;
  int n = 0;
#pragma unroll
  for (int e = 0; e < E - 1; ++e) n += incl[e] < thr;
  at = threadIdx.x * E + n;
}

// The plan of a row, with the inclusive sums of its bins in mass and cnt (LDS).
template <int NT>
__device__ inline Plan plan(const RowWs& w, const Setting& s, u64* mass, uint32_t* cnt) {
  constexpr int E = BINS / NT;
  __shared__ u64 s_m[NT / 64];
  __shared__ uint32_t s_c[NT / 64];
  __shared__ int s_bin[2];
  u64 m = 0, hm[E], x[E];
  uint32_t c = 0, hc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = w.bin[threadIdx.x * E + e];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    m += mass_of(unit_of(threadIdx.x * E + e), units_of(x[e]));
    c += (uint32_t)(x[e] >> CNT_AT);
    hm[e] = m;
    hc[e] = c;
  }
  const u64 m0 = block_incl<NT>(m, s_m) - m;
  const uint32_t c0 = block_incl<NT>(c, s_c) - c;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    mass[threadIdx.x * E + e] = hm[e] += m0;
    cnt[threadIdx.x * E + e] = hc[e] += c0;
  }
  __syncthreads();
  Plan p;
  p.total = cnt[BINS - 1];
  p.z = mass[BINS - 1];
  // the bins of up to two thresholds
  auto find2 = [&](bool by_mass, u64 a, u64 b, int& ba, int& bb) {
    if (by_mass) {
      own_bin<E>(hm, m0, a, s_bin[0]);
      own_bin<E>(hm, m0, b, s_bin[1]);
    } else {
      own_bin<E>(hc, c0, (uint32_t)a, s_bin[0]);
      own_bin<E>(hc, c0, (uint32_t)b, s_bin[1]);
    }
    __syncthreads();
    ba = s_bin[0];
    bb = s_bin[1];
    __syncthreads();
  };
  auto before = [&](int b) { return b ? mass[b - 1] : 0; };
  u64 zlo = p.z, zhi = p.z;  // mass that top-k keeps
  p.k_bin = -1;
  int b, b2;
  if (s.k < p.total) {
    find2(false, s.k, s.k, b, b2);
    zlo = before(b);
    zhi = mass[b];
    if (zhi > zlo) p.k_bin = b;
    else p.z = zlo;
  }
  p.p_lo = BINS;
  p.p_hi = -1;
  if (s.top_p < 1.0) {
    find2(true, reach(s.top_p, max(zlo, (u64)1)), reach(s.top_p, zhi), p.p_lo, p.p_hi);
    zlo = before(p.p_lo) + 1;
    zhi = min(zhi, mass[p.p_hi]);
  }
  find2(true, exceed(s.u, max(zlo, (u64)1)), exceed(s.u, zhi), p.d_lo, p.d_hi);
  return p;
}

// grid (chunks, rows)
template <typename T>
__global__ __launch_bounds__(SCAN_T) void k_draw_max(DrawArgs a, int chunk) {
  __shared__ float s_m[SCAN_T / 64];
  const int b = blockIdx.x, NB = gridDim.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  for (int i = b * SCAN_T + threadIdx.x; i < BINS; i += NB * SCAN_T) w.bin[i] = 0;
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
  __shared__ u64 s_bin[BINS];
  const int b = blockIdx.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  for (int i = threadIdx.x; i < BINS; i += SCAN_T) s_bin[i] = 0;
  const Setting s = setting(a, r, row_max(w, gridDim.x));
  if (!s.entry(s.lmax)) return;
  __syncthreads();
  each_logit<SCAN_T>((const T*)a.logits + (size_t)r * a.ld, b * chunk,
                     min(a.vocab, (b + 1) * chunk), [&](float l, int) {
                       int bin;
                       uint32_t rem;
                       if (s.place(l, bin, rem))
                         atomicAdd(&s_bin[bin], (1ull << CNT_AT) + s.s_of(rem));
                     });
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += SCAN_T)
    if (s_bin[i]) atomicAdd(&w.bin[i], s_bin[i]);
}

template <typename T>
__global__ __launch_bounds__(SCAN_T) void k_draw_gather(DrawArgs a, int chunk) {
  __shared__ u64 s_e[CAP];  // the bins' sums, then entries
  __shared__ uint32_t s_n;
  static_assert(CAP * sizeof(u64) >= BINS * (sizeof(u64) + sizeof(uint32_t)));
  u64* const s_mass = s_e;
  uint32_t* const s_cnt = (uint32_t*)(s_e + BINS);
  const int b = blockIdx.x, r = blockIdx.y;
  RowWs& w = ((RowWs*)a.ws)[r];
  const Setting s = setting(a, r, row_max(w, gridDim.x));
  if (!s.entry(s.lmax)) return;
  const Plan p = plan<SCAN_T>(w, s, s_mass, s_cnt);
  if (b == 0) {  // for the next launch
    for (int i = threadIdx.x; i < BINS; i += SCAN_T) {
      w.mass[i] = s_mass[i];
      w.cnt[i] = s_cnt[i];
    }
    if (threadIdx.x == 0) w.plan = p;
  }
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();  // the sums' place takes entries from here on
  // logits that may lie in the bins lo .. hi: a float32 interval, wider by more than
  // its roundings
  const double w_bin = 1.0 / s.scale;
  auto interval = [&](int lo, int hi, float& from, float& to) {
    const double f = (double)s.lmax - (hi + 1) * w_bin, t = (double)s.lmax - lo * w_bin;
    const double wide = 1e-6 * (fabs((double)s.lmax) + (hi + 1) * w_bin) + 1e-30;
    from = hi >= BINS - 1 || !(f - wide >= -FLT_MAX) ? -INFINITY : (float)(f - wide);
    to = lo <= 0 || !(t + wide <= FLT_MAX) ? INFINITY : (float)(t + wide);
    if (lo > hi) from = INFINITY, to = -INFINITY;
  };
  float kf, kt, pf, pt, df, dt;
  interval(p.k_bin < 0 ? BINS : p.k_bin, p.k_bin, kf, kt);
  interval(p.p_lo, p.p_hi, pf, pt);
  interval(p.d_lo, p.d_hi, df, dt);
  const float lo = fminf(kf, fminf(pf, df)), hi = fmaxf(kt, fmaxf(pt, dt));
  // Entries of the intervals first, by float32 alone, then the bins' own of these.  (The
  // exact test at each logit's place in the loop makes its code several times as long.)  More than CAP count as more than CAP in the bins.
  each_logit<SCAN_T>((const T*)a.logits + (size_t)r * a.ld, b * chunk,
                     min(a.vocab, (b + 1) * chunk), [&](float l, int id) {
                       if (!(l >= lo && l <= hi)) return;
                       if (!((l >= kf && l <= kt) || (l >= pf && l <= pt) || (l >= df && l <= dt)))
                         return;
                       const uint32_t n = atomicAdd(&s_n, 1u);
                       if (n < CAP) s_e[n] = entry_of(l, id);
                     });
  __syncthreads();
  const uint32_t n = s_n;
  if (n > CAP) {
    if (threadIdx.x == 0) atomicAdd(&w.n_cand, CAP + 1u);
    return;
  }
  for (uint32_t i = threadIdx.x; i < n; i += SCAN_T) {
    const u64 e = s_e[i];
    int bin;
    uint32_t rem;
    if (!s.place(key_logit((uint32_t)(e >> 32)), bin, rem) || !p.wants(bin)) continue;
    const uint32_t at = atomicAdd(&w.n_cand, 1u);
    if (at < CAP) w.cand[at] = e;
  }
}

// The place searched for: the entry, and rank and cumulative mass up to it.
struct Place {
  u64 entry, cum;
  uint32_t rank;
};

// First entry, in order, of bin `bin` whose rank (by_mass: cumulative mass) reaches
// thr: radix search over the row, 11 bits of the entry a pass (the id has at most 20
// bits, so the order key's 32 bits and they take 5 passes).
template <typename T>
__device__ inline Place search(const T* row, int V, const Setting& s, const RowWs& w, int bin,
                               bool by_mass, u64 thr, u64* s_bin, u64* s_u, int* s_i) {
  constexpr int E = BINS / PICK_T;
  const u64 mass0 = bin ? w.mass[bin - 1] : 0;
  const uint32_t rank0 = bin ? w.cnt[bin - 1] : 0;
  const double unit = unit_of(bin);
  u64 want = thr - rank0;  // in entries, or in units: the fewest whose mass reaches it
  if (by_mass) {
    const u64 t = thr - mass0;
    want = (u64)((double)t / unit);
    while (mass_of(unit, want) < t) ++want;
    while (want > 0 && mass_of(unit, want - 1) >= t) --want;
  }
  // the entry's bits from the top: key 31..21, 20..10, 9..0, then 20..11 and 10..0 of the
  // id's complement, whose other bits are ones
  u64 prefix = 0, fixed = 0, done = 0;  // done: the word of what lies before the digit
  for (int d = 0; d < 5; ++d) {
    const int lo = d == 0 ? 53 : d == 1 ? 42 : d == 2 ? 32 : d == 3 ? 11 : 0;
    const int nb = d == 2 || d == 3 ? 10 : 11;
    for (int i = threadIdx.x; i < BINS; i += PICK_T) s_bin[i] = 0;
    if (threadIdx.x == 0) *s_i = BINS - 1;
    __syncthreads();
    const u64 mask = ((1ull << nb) - 1) << lo;
    each_logit<PICK_T>(row, 0, V, [&](float l, int id) {
      int b;
      uint32_t rem;
      const u64 e = entry_of(l, id);
      if (!s.place(l, b, rem) || b != bin || (e & fixed) != prefix) return;
      // digits in decreasing order
      atomicAdd(&s_bin[(mask - (e & mask)) >> lo], (1ull << CNT_AT) + s.s_of(rem));
    });
    __syncthreads();
    u64 incl[E], x = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) incl[e] = x += s_bin[threadIdx.x * E + e];
    u64 before = block_incl<PICK_T>(x, s_u) - x + done;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const u64 up = incl[e] + before;
      const u64 was = e ? incl[e - 1] + before : before;
      auto val = [&](u64 v) { return by_mass ? units_of(v) : v >> CNT_AT; };
      if (val(was) < want && want <= val(up)) {
        *s_i = threadIdx.x * E + e;
        s_u[PICK_T / 64] = was;
      }
    }
    __syncthreads();
    const int at = *s_i;
    done = s_u[PICK_T / 64];
    prefix |= mask - ((u64)at << lo);
    fixed |= mask;
    if (d == 2) {
      const u64 ones = 0xFFFFFFFFull & ~((1ull << 21) - 1);
      prefix |= ones;
      fixed |= ones;
    }
    __syncthreads();
  }
  // one entry is left
  int b;
  uint32_t rem = 0;
  s.place(key_logit((uint32_t)(prefix >> 32)), b, rem);
  const u64 up = done + (1ull << CNT_AT) + s.s_of(rem);
  return Place{prefix, mass0 + mass_of(unit, units_of(up)), rank0 + (uint32_t)(up >> CNT_AT)};
}

// The three searches, each with what the one before kept.  find(by_mass, thr).
template <typename F>
__device__ inline void places(const Plan& p, const Setting& s, F find, u64& ent, u64& z,
                              uint32_t& kept) {
  z = p.z;
  kept = min(s.k, p.total);
  ent = 0;
  for (int step = 0; step < 3; ++step) {
    if (step == 0 ? p.k_bin < 0 : step == 1 && !(s.top_p < 1.0)) continue;
    const Place q = find(step != 0, step == 0 ? (u64)s.k : step == 1 ? reach(s.top_p, z)
                                                                     : exceed(s.u, z));
    if (step < 2) z = q.cum;
    if (step == 1) kept = q.rank;
    ent = q.entry;
  }
}

// one workgroup a row
template <typename T>
__global__ __launch_bounds__(PICK_T) void k_draw_pick(DrawArgs a, int NB) {
  __shared__ u64 s_e[CAP];       // entries in order; the radix search's words
  __shared__ u64 s_head[BINS];   // units before a bin's first entry
  __shared__ uint32_t s_first[BINS];
  __shared__ u64 s_u[PICK_T / 64 + 1], s_cum, s_ent;
  __shared__ uint32_t s_rank;
  __shared__ int s_at;
  const int r = blockIdx.x, lane = threadIdx.x & 63;
  const RowWs& w = ((const RowWs*)a.ws)[r];
  const uint32_t n = w.n_cand;
  const Plan p = w.plan;
  const Setting s = setting(a, r, row_max(w, NB));
  u64 ent, z;
  uint32_t kept;
  if (!s.entry(s.lmax)) {  // every token is barred
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = -INFINITY;
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  if (n <= 64) {
    if (threadIdx.x >= 64) return;
    const u64 e0 = lane < (int)n ? w.cand[lane] : 0;
    int rank = 0;
    for (int i = 0; i < (int)n; ++i) {
      const u64 x = ((u64)(uint32_t)__builtin_amdgcn_readlane((int)(e0 >> 32), i) << 32) |
                    (uint32_t)__builtin_amdgcn_readlane((int)e0, i);
      rank += x > e0;
    }
    if (lane < (int)n) s_e[rank] = e0;
    __builtin_amdgcn_wave_barrier();
    const u64 e = lane < (int)n ? s_e[lane] : 0;
    int bin = -1;
    uint32_t rem = 0;
    if (lane < (int)n) s.place(key_logit((uint32_t)(e >> 32)), bin, rem);
    const u64 own = bin < 0 ? 0 : (1ull << UNIT) - s.s_of(rem);
    const u64 incl = wave_incl(own);
    const int prev = __shfl_up(bin, 1);
    const bool head = lane == 0 || prev != bin;
    const uint64_t heads = __ballot(head) & (~0ull >> (63 - lane));
    const int first = 63 - __clzll((long long)heads);
    const u64 units = incl - __shfl(incl - own, first);
    u64 cum = 0;
    uint32_t rk = 0;
    if (bin >= 0) {
      cum = (bin ? w.mass[bin - 1] : 0) + mass_of(unit_of(bin), units);
      rk = (bin ? w.cnt[bin - 1] : 0) + lane - first + 1;
    }
    places(p, s, [&](bool by_mass, u64 thr) {
      const uint64_t hit = __ballot(bin >= 0 && (by_mass ? cum >= thr : (u64)rk >= thr));
      const int at = hit ? __ffsll((unsigned long long)hit) - 1 : (int)n - 1;
      return Place{__shfl(e, at), __shfl(cum, at), (uint32_t)__shfl((int)rk, at)};
    }, ent, z, kept);
  } else if (n <= CAP) {
    // into decreasing order: up to one a thread by counting the larger ones, N a power of
    // two of places and PICK_T / N threads a place; more by a bitonic sort, padded with
    // zeros.  (The sort alone: 256 rows of 128256 16 us for 13.)
    int N = 128;
    while (N < (int)n) N <<= 1;
    for (int i = threadIdx.x; i < N; i += PICK_T) s_e[i] = i < (int)n ? w.cand[i] : 0;
    if (N <= PICK_T) {
      const int at = threadIdx.x & (N - 1), part = threadIdx.x / N;
      const int per = ((int)n + PICK_T / N - 1) / (PICK_T / N);
      s_first[threadIdx.x] = 0;
      __syncthreads();
      const u64 x = s_e[at];
      uint32_t larger = 0;
      for (int i = part * per; i < min((int)n, (part + 1) * per); ++i) larger += s_e[i] > x;
      if (at < (int)n) atomicAdd(&s_first[at], larger);
      __syncthreads();
      if (part == 0 && at < (int)n) s_e[s_first[at]] = x;
    } else for (int k = 2; k <= N; k <<= 1)
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
    __syncthreads();
    // rank and cumulative mass of each entry, CAP / PICK_T a thread
    constexpr int E = CAP / PICK_T;
    u64 cum[E], m = 0;
    uint32_t rank[E];
    int bin[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = threadIdx.x * E + e;
      bin[e] = -1;
      if (i < (int)n) {
        uint32_t rem = 0;
        s.place(key_logit((uint32_t)(s_e[i] >> 32)), bin[e], rem);
        m += (1ull << UNIT) - s.s_of(rem);
      }
      cum[e] = m;
    }
    const u64 m0 = block_incl<PICK_T>(m, s_u) - m;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = threadIdx.x * E + e;
      if (bin[e] < 0) continue;
      const int prev = i ? s.bin_of(key_logit((uint32_t)(s_e[i - 1] >> 32))) : -1;
      if (prev != bin[e]) {
        s_head[bin[e]] = m0 + (e ? cum[e - 1] : 0);
        s_first[bin[e]] = i;
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int b = bin[e];
      if (b < 0) continue;
      cum[e] = (b ? w.mass[b - 1] : 0) + mass_of(unit_of(b), cum[e] + m0 - s_head[b]);
      rank[e] = (b ? w.cnt[b - 1] : 0) + threadIdx.x * E + e - s_first[b] + 1;
    }
    // first entry that reaches a rank or a mass
    places(p, s, [&](bool by_mass, u64 thr) {
      if (threadIdx.x == 0) s_at = (int)n - 1;
      __syncthreads();
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (bin[e] >= 0 && (by_mass ? cum[e] >= thr : (u64)rank[e] >= thr) &&
            !(e > 0 && (by_mass ? cum[e - 1] >= thr : (u64)rank[e - 1] >= thr)))
          atomicMin(&s_at, (int)threadIdx.x * E + e);
      __syncthreads();
      const int at = s_at;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((int)threadIdx.x * E + e == at) {
          s_cum = cum[e];
          s_rank = rank[e];
          s_ent = s_e[at];
        }
      __syncthreads();
      return Place{s_ent, s_cum, s_rank};
    }, ent, z, kept);
  } else {
    const T* row = (const T*)a.logits + (size_t)r * a.ld;
    places(p, s, [&](bool by_mass, u64 thr) {
      // the place's bin
      constexpr int E = BINS / PICK_T;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int b = threadIdx.x * E + e;
        const u64 up = by_mass ? w.mass[b] : w.cnt[b];
        const u64 was = !b ? 0 : by_mass ? w.mass[b - 1] : w.cnt[b - 1];
        if (was < thr && thr <= up) s_at = b;
      }
      __syncthreads();
      const int b = s_at;
      __syncthreads();
      return search<T>(row, a.vocab, s, w, b, by_mass, thr, s_e, s_u, &s_at);
    }, ent, z, kept);
  }
  if (threadIdx.x == 0) {
    a.tokens[r] = (int32_t)~(uint32_t)ent;
    const double x = s.y_of(key_logit((uint32_t)(ent >> 32))) * (-1.0 / BIN_W);
    if (a.logprob) a.logprob[r] = (float)(x - log((double)z * (1.0 / (double)(1ull << FRAC))));
    if (a.kept) a.kept[r] = (int32_t)kept;
  }
}

}  // namespace

size_t draw_ws_bytes(int rows) { return (size_t)rows * sizeof(RowWs); }

void draw_rows(const DrawArgs& a, hipStream_t st) {
  // chunks: about 1024 workgroups over the rows, of at least 2560 logits: more chunks add
  // more bins to memory (7 rows of 151936 in chunks of 1220: k_draw_hist 11.5 us, of 2560
  // 6.9), fewer leave the chip empty (one row of 128256 in chunks of 4096: 5.9 for 4.8);
  // 512 workgroups for 256 rows: 48 us for 40 in k_draw_gather, 2048 the same
  int NB = std::min(std::min(NB_MAX, (1024 + a.rows - 1) / a.rows), (a.vocab + 2560 - 1) / 2560);
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
