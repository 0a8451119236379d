// Paged cache of keys and values: the append of new rows (with the rotation of
// queries and keys) and causal attention of ragged rows over it.
//
// A cache holds pages of `page` tokens, every kv head apart, in bf16 or in 8-bit
// floating point (e4m3: 4 exponent and 3 mantissa bits, largest value 448) with
// one float32 scale, a power of two, per `block` tokens and head:
//
//   keys    [n_pages][hkv][page][hd]            token-major
//   values  [n_pages][hkv][page / 16][hd][16]   dimension-major in granules of 16 tokens
//   scales  [n_pages][hkv][page / block]
//
// A 16x16x32 matrix instruction reads 8 consecutive contraction elements per lane:
// dimensions of one key in S = K Q^T, tokens of one dimension in O^T = V^T P^T.  The
// value layout is that operand as it stands (16 lanes read 256 contiguous bytes), so
// values go from memory to operand registers; keys, whose rows lie on different
// lanes, pass through LDS.
//
// A power of two as scale costs e4m3 nothing (its relative step does not depend on
// the scale) and makes every change of scale exact but for codes that reach the
// subnormal range, so earlier tokens of a block survive a later, larger token.
//
//  k_pg_append  new rows: rotation, scales, codes, and the rotated queries
//  k_pg_dec     attention of few rows a sequence, split over the context
//  k_pg_chunk   attention of many rows (prompt chunks)
//  k_pg_merge   joins the splits of a row
#include "ks_internal.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace ks {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int GRAN = 16;     // tokens of a value granule
constexpr int E_MIN = -100;  // smallest scale: 2^E_MIN
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// ------------------------------------------------------------------- 8 bits
// Smallest power of two s with amax <= 448 s, at least 2^E_MIN: 448 = 1.75 2^8, so
// the exponent of amax decides, and whether its mantissa lies above 1.75.
__device__ inline float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = max(e, E_MIN);
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
// 1 / s of a power of two in [2^-126, 2^126]
__device__ inline float inv_pow2(float s) {
  return __uint_as_float((254u << 23) - (__float_as_uint(s) & 0x7F800000u));
}
__device__ inline bool finite_f(float x) { return fabsf(x) <= FLT_MAX; }
// nearest code (ties to even) of a finite |x| <= 448; what is not finite becomes NaN
__device__ inline uint32_t code_of(float x) {
  const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.f, 0, false) & 0xFFu;
  return finite_f(x) ? c : 0x7Fu;
}
__device__ inline float value_of(uint32_t code) {
  return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

__device__ inline float ld1(const float* p) { return *p; }
__device__ inline float ld1(const bf16_t* p) { return bf2f(*p); }
__device__ inline void st1(float* p, float x) { *p = x; }
__device__ inline void st1(bf16_t* p, float x) { *p = f2bf(x); }

template <int N>  // sum over aligned groups of N lanes
__device__ inline float group_sum(float v) {
#pragma unroll
  for (int o = N / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ inline float wave_max64(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// Rows of sequence b, as far as the call's tensors and bounds hold them.
struct SeqRows {
  int r0, n;
  bool over;  // it has more rows than max_rows
};
__device__ inline SeqRows seq_rows(const PagedRows& s, int b) {
  if (!s.row_start) return SeqRows{0, s.rows, false};
  const int a = min(max(s.row_start[b], 0), s.rows);
  const int e = min(max(s.row_start[b + 1], a), s.rows);
  return SeqRows{a, min(e - a, s.max_rows), e - a > s.max_rows};
}

// Position of sequence b's first row; far outside any cache it stands for the same
// as here, with room to add a row number.
__device__ inline int first_pos(const PagedRows& s, int b) {
  return min(max(s.pos0[b], -(1 << 30)), 1 << 30);
}
// Positions that a row attends, in [0, max_len]; over: there are more.
__device__ inline int row_len(const PagedAttn& a, const SeqRows& sr, int b, int r, bool& over) {
  const int n = a.len ? a.len[sr.r0 + r] : first_pos(a.rows, b) + r + 1;
  over |= n > a.rows.max_len;
  return min(max(n, 0), a.rows.max_len);
}

// Row r's sequence (the last b with row_start[b] <= r), its place i in it and the
// sequence's first position; b = -1 for a row behind the last sequence or past
// max_rows.  Boundaries and positions of 63 sequences are asked for at once, so that
// a wave waits for one memory latency.  Wave-uniform r.
struct RowAt {
  int b, i, n, p0;
};
__device__ inline RowAt row_at(const PagedRows& s, int r) {
  if (!s.row_start) return RowAt{r < s.rows ? 0 : -1, r, s.rows, s.pos0 ? first_pos(s, 0) : 0};
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < s.B; b0 += 63) {
    const int at = min(max(s.row_start[min(b0 + lane, s.B)], 0), s.rows);
    const int p0 = first_pos(s, min(b0 + lane, s.B - 1));
    const uint64_t past = __ballot(lane > 0 && b0 + lane <= s.B && at > r);
    if (!past) continue;
    const int x = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
    RowAt y{b0 + x - 1, 0, 0, __builtin_amdgcn_readlane(p0, x - 1)};
    const int r0 = __builtin_amdgcn_readlane(at, x - 1);
    y.i = r - r0;
    y.n = __builtin_amdgcn_readlane(at, x) - r0;
    if (y.i < 0 || y.i >= s.max_rows) y.b = -1;
    return y;
  }
  return RowAt{-1, 0, 0, 0};
}

// ------------------------------------------------------------------- append
// 8 elements as they are, and as float32.  VEC: at a 16-byte address.
template <typename T>
struct Raw8 {
  T x[8];
};
template <bool VEC, typename T>
__device__ inline Raw8<T> load8(const T* p) {
  Raw8<T> r;
  if (VEC) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(r) / 16; ++i) ((uint4*)r.x)[i] = ((const uint4*)p)[i];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = p[e];
  }
  return r;
}
template <typename T>
__device__ inline void floats8(const Raw8<T>& r, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = ld1(&r.x[e]);
}
// f with whether rows are aligned as a constant: one branch around all loads of a
// pass, which are then in flight together
template <typename F>
__device__ inline void with_vec(bool vec, F f) {
  if (vec) f(std::true_type{});
  else f(std::false_type{});
}
template <bool VEC>
__device__ inline void store8(float* p, const float (&x)[8]) {
  if (VEC) {
    ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = x[e];
  }
}
template <bool VEC>
__device__ inline void store8(bf16_t* p, const float (&x)[8]) {
  if (VEC) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (uint32_t)f2bf(x[2 * i]) | ((uint32_t)f2bf(x[2 * i + 1]) << 16);
    *(u32x4*)p = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = f2bf(x[e]);
  }
}
// 8 codes of x s, in pairs; what is not finite becomes NaN
__device__ inline uint2 codes8(const float (&x)[8], float s) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int y = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * s, x[4 * i + 1] * s, 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * s, x[4 * i + 3] * s, y, true);
  }
  float z = 0.f;  // 0 times what is not finite is NaN
#pragma unroll
  for (int e = 0; e < 8; ++e) z = fmaf(x[e], 0.f, z);
  if (__any(z != 0.f))
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!finite_f(x[e])) w[e >> 2] |= 0x7Fu << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}
__device__ inline float amax8(float m, const float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_f(x[e]) ? fabsf(x[e]) : 0.f);
  return m;
}

// A lane's part of a head: dims d .. d + 7, HD / 8 lanes a head.  An optional RMS norm
// over the head, then the rotation of the pairs (f, f + hd/2) by the table's angles of
// the position; the other half of a pair lies HD / 16 lanes away.
template <int HD>
__device__ inline void turn(float (&x)[8], const float* cs, const float* gain, float eps, int d) {
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
    const float r = 1.0f / sqrtf(group_sum<HD / 8>(ss) / (float)HD + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * r * gain[d + e];
  }
  if (!cs) return;
  const bool low = d < HD / 2;
  const float4* c = (const float4*)(cs + 2 * (low ? d : d - HD / 2));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float4 t = c[e / 2];  // (cos, sin) of two pairs
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int bits = __float_as_int(x[e + u]);
      const float y = __int_as_float(HD == 128
                                         ? __builtin_amdgcn_update_dpp(0, bits, 0x128, 0xF, 0xF, true)
                                         : __builtin_amdgcn_ds_swizzle(bits, 0x101F));
      x[e + u] = x[e + u] * (u ? t.z : t.x) + (low ? -y : y) * (u ? t.w : t.y);
    }
  }
}

// n_kv workgroups take one scale block (bf16: 16 tokens) of one head of one sequence
// each; waves 0 and 1 take its keys, 2 and 3 its values.  A workgroup
// owns all codes of its block, so it may change the block's scale.  Its new rows stay
// in registers (keys) and LDS (values, which change from token-major to
// dimension-major there) between the search for the largest and the codes; blocks of
// more than 64 tokens read them again.  The other workgroups turn query heads, a row a
// wave.  All rows move 16 bytes a lane where they are aligned.
//
// Memory bounds it: 10900 rows of 48 heads, 252 MB, in 62 us (a copy: 54).  The cache
// blocks first and the queries in a launch of their own took 75.  Three workgroups a CU
// cost float32 rows of 128 dims eight spilled registers and gain more: 10000 rows 100 us,
// 115 with two.  A block whose scale grows, 63 earlier tokens: 13.6 us for a call of 48
// sequences, 16.8 with a code a lane at a time.
constexpr int APP_T = 64;   // tokens of a pass
constexpr int APP_QW = 32;  // query heads of a wave at head dim 128

template <typename T, int HD, bool E4>
__global__ __launch_bounds__(256, 3) void k_pg_append(PagedAppend a, int n_kv, int touched) {
  constexpr int HL = HD / 8;            // lanes of a row of a head
  constexpr int TW = 64 / HL;           // rows of a wave at a time
  constexpr int KIT = APP_T / (2 * TW); // rows a lane
  const PagedCache& c = a.cache;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane % HL * 8;  // this lane's dims, and their place in a row
  const int cd = a.perm ? (d < HD / 2 ? 2 * d : 2 * (d - HD / 2) + 8) : d;  // (see qkv_perm)

  const int wg = blockIdx.x;
  if (wg >= n_kv) {
    constexpr int QW = APP_QW * 128 / HD;  // query heads of a wave
    const int per = (a.hq + QW - 1) / QW;
    const int job = (wg - n_kv) * 4 + wave;
    const int r = job / per, h0 = job % per * QW + lane / HL;
    if (r >= a.rows.rows) return;
    Raw8<T> rx[QW / TW];
    with_vec(a.vec & 1, [&](auto vec) {
#pragma unroll
      for (int i = 0; i < QW / TW; ++i) {
        const T* src = (const T*)a.q + (size_t)r * a.ldq + (size_t)min(h0 + TW * i, a.hq - 1) * HD;
        rx[i] = load8<decltype(vec)::value>(src + cd);
      }
    });
    const RowAt ra = row_at(a.rows, r);
    if (ra.b < 0) return;
    const int p = ra.p0 + ra.i;
    const bool ok = p >= 0 && (!a.rope || p < a.rope_rows);
    const float* cs = a.rope && ok ? a.rope + (size_t)p * HD : nullptr;
    with_vec(a.vec & 2, [&](auto vec) {
#pragma unroll
      for (int i = 0; i < QW / TW; ++i) {
        float x[8];
        floats8(rx[i], x);
        turn<HD>(x, cs, a.q_gain, a.eps, d);
        if (!ok)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
        const int h = h0 + TW * i;
        if (h < a.hq)
          store8<decltype(vec)::value>((T*)a.q_out + (size_t)r * a.ldqo + (size_t)h * HD + d, x);
      }
    });
    return;
  }

  __shared__ __align__(16) T s_v[APP_T][HD];
  __shared__ float s_max[4];
  const int t = wg % touched;
  const int h = wg / touched % c.hkv;
  const int b = wg / touched / c.hkv;
  const SeqRows sr = seq_rows(a.rows, b);
  const int p0 = first_pos(a.rows, b);
  const int lblock = E4 ? c.lblock : 4, block = 1 << lblock;
  // new tokens are [pa, pe); rows at negative positions are padding
  const int pa = max(p0, 0);
  const int cap = min(a.rope ? a.rope_rows : INT32_MAX, a.rows.max_len);
  const int pe = min(p0 + sr.n, cap);
  if (a.rows.err && t == 0 && threadIdx.x == 0 && (sr.over || p0 + sr.n > cap)) a.rows.err[b] = 1;
  const long long bs_ = ((long long)(pa >> lblock) + t) << lblock;  // first token of the block
  if (bs_ >= pe) return;
  const int bs = (int)bs_;
  const int n0 = max(bs, pa), n1 = min(bs + block, pe);  // its new tokens
  if (n0 >= n1) return;
  const int pid = a.rows.table[(size_t)b * a.rows.table_ld + (bs >> c.lpage)];
  const bool is_k = wave < 2;
  const int w2 = wave & 1;
  const int row_of = sr.r0 - p0;  // row of position p: row_of + p

  // keys t0 .. of a pass, rotated; rows at or past n1 repeat the last
  float x[KIT][8];
  auto keys = [&](int t0) __attribute__((always_inline)) {
    const T* src = (const T*)a.k + (size_t)h * HD;
    Raw8<T> rx[KIT];
    with_vec(a.vec & 4, [&](auto vec) {
#pragma unroll
      for (int i = 0; i < KIT; ++i) {
        const int p = t0 + 2 * TW * i + TW * w2 + lane / HL;
        if (t0 + 2 * TW * i + TW * w2 >= n1) break;
        const T* r = src + (size_t)(row_of + min(p, n1 - 1)) * a.ldk;
        rx[i] = load8<decltype(vec)::value>(r + cd);
      }
    });
#pragma unroll
    for (int i = 0; i < KIT; ++i) {
      const int p = t0 + 2 * TW * i + TW * w2 + lane / HL;
      if (t0 + 2 * TW * i + TW * w2 >= n1) break;
      floats8(rx[i], x[i]);
      turn<HD>(x[i], a.rope ? a.rope + (size_t)min(p, n1 - 1) * HD : nullptr, a.k_gain, a.eps, d);
    }
  };
  // values into LDS; returns the largest of this lane's
  auto values = [&](int t0) __attribute__((always_inline)) {
    const T* src = (const T*)a.v + (size_t)h * HD;
    float m = 0.f;
    Raw8<T> z[KIT];
    with_vec(a.vec & 8, [&](auto vec) {
#pragma unroll
      for (int i = 0; i < KIT; ++i) {
        const int p = t0 + 2 * TW * i + TW * w2 + lane / HL;
        if (t0 + 2 * TW * i + TW * w2 >= n1) break;
        z[i] = load8<decltype(vec)::value>(src + (size_t)(row_of + min(p, n1 - 1)) * a.ldv + cd);
      }
    });
#pragma unroll
    for (int i = 0; i < KIT; ++i) {
      const int q = 2 * TW * i + TW * w2 + lane / HL;
      if (t0 + 2 * TW * i + TW * w2 >= n1) break;
      float x[8];
      floats8(z[i], x);
      m = amax8(m, x);
#pragma unroll
      for (int u = 0; u < (int)sizeof(z[i]) / 16; ++u)
        ((uint4*)&s_v[q][d])[u] = ((const uint4*)z[i].x)[u];
    }
    return m;
  };

  const int passes = (n1 - n0 + APP_T - 1) / APP_T;
  if (is_k) keys(n0);
  float amax = is_k ? 0.f : values(n0);
  if (pid < 0 || pid >= c.n_pages) {
    if (a.rows.err && threadIdx.x == 0) a.rows.err[b] = 1;
    return;
  }
  const int s0 = bs & (c.page - 1);  // the block's first slot in its page
  const size_t head = (size_t)pid * c.hkv + h;
  float s = 1.f, inv = 1.f, ratio = 1.f;
  if (E4) {
    float* sp = (is_k ? c.k_scale : c.v_scale) + (head << (c.lpage - lblock)) + (s0 >> lblock);
    float s_old = n0 > bs ? *sp : 0.f;  // earlier tokens only
    if (!(s_old > 0.f && s_old <= FLT_MAX)) s_old = 0.f;
    for (int u = 0; u < passes; ++u) {
      if (u > 0) {
        if (is_k) keys(n0 + APP_T * u);
        else amax = fmaxf(amax, values(n0 + APP_T * u));
      }
      if (is_k)
#pragma unroll
        for (int i = 0; i < KIT; ++i) {
          if (n0 + APP_T * u + 2 * TW * i + TW * w2 >= n1) break;
          amax = amax8(amax, x[i]);
        }
    }
    amax = wave_max64(amax);
    if (lane == 0) s_max[wave] = amax;
    __syncthreads();
    s = fmaxf(s_old, scale_for(is_k ? fmaxf(s_max[0], s_max[1]) : fmaxf(s_max[2], s_max[3])));
    inv = inv_pow2(s);
    ratio = s_old * inv;  // earlier codes are multiplied by it
    if ((threadIdx.x & 127) == 0) *sp = s;
  } else {
    __syncthreads();
  }

  for (int u = 0; u < passes; ++u) {
    const int t0 = n0 + APP_T * u;
    if (passes > 1) {  // the rows again
      __syncthreads();
      if (is_k) keys(t0);
      else values(t0);
      __syncthreads();
    }
    if (is_k) {
      const size_t base = (head << c.lpage) * HD + (size_t)s0 * HD;
      if (E4 && u == 0 && n0 > bs && ratio != 1.f) {
        uint8_t* kc = (uint8_t*)c.k + base;
        for (int i = (w2 * 64 + lane) * 8; i < (n0 - bs) * HD; i += 1024) {
          const uint2 y = *(const uint2*)(kc + i);
          float z[8];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int u = e ? y.y : y.x;
            z[4 * e] = __builtin_amdgcn_cvt_f32_fp8(u, 0);
            z[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8(u, 1);
            z[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8(u, 2);
            z[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8(u, 3);
          }
          *(uint2*)(kc + i) = codes8(z, ratio);
        }
      }
#pragma unroll
      for (int i = 0; i < KIT; ++i) {
        const int p = t0 + 2 * TW * i + TW * w2 + lane / HL;
        if (t0 + 2 * TW * i + TW * w2 >= n1) break;
        if (p >= n1) continue;
        const size_t at = base + (size_t)(p - bs) * HD + d;
        if (E4) *(uint2*)((uint8_t*)c.k + at) = codes8(x[i], inv);
        else store8<true>((bf16_t*)c.k + at, x[i]);
      }
      continue;
    }
    const int dim = threadIdx.x - 128;
    if (dim >= HD) continue;
    const int t1 = min(t0 + APP_T, n1);
    // granules that this pass reaches (the first also those of earlier tokens)
    for (int g0 = u == 0 && ratio != 1.f ? bs : t0 & ~(GRAN - 1); g0 < t1; g0 += GRAN) {
      const size_t off = ((head << c.lpage) + (size_t)(s0 + g0 - bs)) * HD + (size_t)dim * GRAN;
      if (E4) {
        uint8_t* vc = (uint8_t*)c.v + off;
        uint32_t w[4];
        if (g0 < t0 || g0 + GRAN > t1) *(uint4*)w = *(const uint4*)vc;
#pragma unroll
        for (int i = 0; i < GRAN; ++i) {
          const int p = g0 + i;
          if (p >= t0 && p < t1) {
            const uint32_t cd = code_of(ld1(&s_v[p - t0][dim]) * inv);
            w[i / 4] = (w[i / 4] & ~(0xFFu << (8 * (i % 4)))) | cd << (8 * (i % 4));
          } else if (p < n0 && ratio != 1.f) {
            const uint32_t cd = code_of(value_of((w[i / 4] >> (8 * (i % 4))) & 0xFFu) * ratio);
            w[i / 4] = (w[i / 4] & ~(0xFFu << (8 * (i % 4)))) | cd << (8 * (i % 4));
          }
        }
        *(uint4*)vc = *(const uint4*)w;
      } else {
        bf16_t* vc = (bf16_t*)c.v + off;
        if (g0 >= t0 && g0 + GRAN <= t1) {
          float z[2][8];
#pragma unroll
          for (int i = 0; i < GRAN; ++i) z[i >> 3][i & 7] = ld1(&s_v[g0 + i - t0][dim]);
          store8<true>(vc, z[0]);
          store8<true>(vc + 8, z[1]);
        } else {
          for (int i = max(g0, t0) - g0; i < min(g0 + GRAN, t1) - g0; ++i)
            vc[i] = f2bf(ld1(&s_v[g0 + i - t0][dim]));
        }
      }
    }
  }
}

// ---------------------------------------------------------------- attention
constexpr int DEC_NW = 4;       // waves of a split workgroup
constexpr int KT = 64;          // keys of a tile

// One wave's tile in flight: 64 keys, 64 values.  Key row i of subtile kt is key
// 16 (i / 4) + 4 kt + i % 4 of the tile, so lane group g of the score registers holds
// the 16 consecutive keys from 16 g: one granule of values.
//  keys    as they lie in memory: register u, lane l has bytes 1024 u + 16 l of the
//          tile's rows.  (Loaded as operands instead, every lane of a quad another
//          row, the loads take four times the cache accesses; 64 sequences of 500 to
//          15000 tokens took 249 us for 238.)
//  values  lane (i, g): dim 16 db + i, tokens 16 g..16 g + 15
template <int HD, bool E4>
struct Tile {
  static constexpr int RB = E4 ? HD : 2 * HD;  // bytes of a key row
  static constexpr int CH = RB / 16;           // its 16-byte chunks
  static constexpr int KU = KT * RB / 1024;    // key registers
  static constexpr int PG = KU / 4;            // of them per granule of 16 keys
  static constexpr int VJ = E4 ? 1 : 2;
  u32x4 k[KU];
  u32x4 v[HD / 16][VJ];
  // Where chunk c of key row r lies in LDS: 8 lanes of an operand read have rows
  // 4 kt + 0..3 and those 16 up, so these bits decide the bank.
  __device__ static int at(int r, int c) {
    const int f = CH == 4 ? ((r >> 1) & 1) | ((r >> 4) & 1) << 1 : (r & 3) | ((r >> 4) & 1) << 2;
    return r * RB + ((c ^ f) << 4);
  }
};

// 8 codes of two words as bf16, times the scale (exact)
__device__ inline bf16x8 widen(uint32_t w0, uint32_t w1, float s) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w0, s, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w0, s, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w1, s, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w1, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Dimension of element e of contraction step s, lane group g: the order in which
// the key loads deliver them.
template <bool E4>
__device__ inline int dim_of(int s, int g) {
  return E4 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
}

// x as N bf16 planes that add up to it, 8 bits each.  All have x's sign and none is 0
// unless x is: times an infinite key or value every plane then gives the infinity
// that x gives, where opposite ones or a 0 among them would give NaN.  (2^-126 in
// the place of 0 is below what float32 keeps of any sum here.)
template <int N>
__device__ inline void planes_of(float x, __bf16 (&o)[N]) {
  float r = x;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n + 1 < N)
      o[n] = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(r) >> 16));  // towards 0
    else
      o[n] = (__bf16)r;
    const float y = (float)o[n];
    r -= y;
    if (n > 0) {  // |y| at least the smaller of |x| and 2^-126
      const float z = fmaxf(fabsf(y), fminf(fabsf(x), 1.17549435e-38f));
      o[n] = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(copysignf(z, x)) >> 16));
    }
  }
}

// 8 query elements as QP bf16 planes: one holds bf16 queries exactly, two hold
// float32 ones to 16 bits and three to 24
template <int QP>
__device__ inline void load_q(const void* p, bool f32, bf16x8 (&o)[QP]) {
  if (QP == 1) {
    o[0] = __builtin_bit_cast(bf16x8, *(const u32x4*)p);
    return;
  }
  const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
  const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    __bf16 y[QP];
    planes_of<QP>(x[e], y);
#pragma unroll
    for (int n = 0; n < QP; ++n) o[n][e] = y[n];
  }
}

__device__ inline uint32_t bytes_below(int n) {  // mask of the first n of 4 bytes
  return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

// Workgroups of a CU that the registers are cut for.  Two hide the start of one and
// the joining of its waves behind the other; where that would spill (two column
// blocks of head dim 128, three planes of queries against bf16) one is faster: 8 rows
// of 64 sequences of 8192 tokens 240 us, 289 with spills.  Three spill everywhere.
constexpr int dec_wgs(int HD, bool E4, int QP, int CB) {
  return (CB == 1 || HD == 64) && (E4 || QP < 3) ? 2 : 1;
}

// Few rows.  A workgroup of four waves owns one split of `span` positions of one
// kv head of one sequence and 16 CB of its query columns (column c: row c / G,
// query head c % G of the kv head); wave w takes the split's tiles w, w + 4, ...
// and runs a softmax with a running maximum and sum over them.  The next keys are
// requested when these have gone to LDS and the next values when these are added,
// so a tile's loads are in flight during the arithmetic of the one before.  The four
// results meet in LDS, in wave order.
//
// A column's arithmetic depends on its own query and length and on the split
// only, never on the other columns or on CB.
//
// Memory bounds it: 64 sequences of 7700 tokens at 5.4 TB/s of cache, 512 of 8192 at
// 5.8, with the arithmetic left out 5.7 and 6.2 (a plain stream of that size 7.0).
//
// Masked places: a key past a column's length is masked in the scores, whatever
// it holds; a value there meets probability 0, so it must not be infinite or
// NaN: values past the longest length are zeroed, and where those between the
// shortest and the longest length hold one, the rows are added one at a time.
template <int HD, bool E4, int QP, int CB>
__global__ __launch_bounds__(64 * DEC_NW, dec_wgs(HD, E4, QP, CB)) void k_pg_dec(PagedAttn a) {
  constexpr int PP = QP == 3 ? 3 : 1;  // probability planes
  constexpr int NS = HD / 32;          // contraction steps of a score
  constexpr int ND = HD / 16;          // blocks of 16 output dims
  constexpr int RS = HD + 4;           // LDS merge record per column (bank-shifted)
  typedef Tile<HD, E4> TileT;
  extern __shared__ __align__(16) unsigned char smem[];
  const PagedCache& c = a.cache;
  const int G = a.hq / c.hkv;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;

  int id = blockIdx.x;
  const int kvh = id % c.hkv;
  id /= c.hkv;
  const int col0 = id % a.cblocks * 16 * CB;
  id /= a.cblocks;
  const int b = id % a.rows.B, split = id / a.rows.B;
  const int start = split * a.span;
  // the split's page ids, requested before the lengths say how many are needed
  const int* tab = a.rows.table + (size_t)b * a.rows.table_ld + (start >> c.lpage);
  const int np_most =
      ((min(start + a.span, a.rows.max_len) - 1) >> c.lpage) - (start >> c.lpage) + 1;
  int pid0 = 0;
  if ((int)threadIdx.x < np_most) pid0 = tab[threadIdx.x];
  const SeqRows sr = seq_rows(a.rows, b);
  if (a.rows.err && threadIdx.x == 0 && sr.over) a.rows.err[b] = 1;
  const int ncol = min(sr.n * G - col0, 16 * CB);
  if (ncol <= 0) return;
  if (sr.n * G > a.col_max) return;  // a sequence of the chunk kernel

  // lengths: of this lane's columns, and the shortest and longest of the block
  int len[CB], lmin = INT32_MAX, lmax = 0;
  bool over = false;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int cc = 16 * cb + i16;
    const int r = (col0 + min(cc, ncol - 1)) / G;
    len[cb] = row_len(a, sr, b, r, over);
    lmin = min(lmin, len[cb]);
    lmax = max(lmax, len[cb]);
  }
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) {
    lmin = min(lmin, __shfl_xor(lmin, o));
    lmax = max(lmax, __shfl_xor(lmax, o));
  }
  lmin = __builtin_amdgcn_readfirstlane(lmin);
  lmax = __builtin_amdgcn_readfirstlane(lmax);
  if (a.rows.err && over) a.rows.err[b] = 1;
  const int stop = min(lmax, start + a.span);
  if (start >= stop && split > 0) return;  // no partial is read from here

  // the split's page ids
  int* s_page = (int*)smem;
  const int np = stop > start ? ((stop - 1) >> c.lpage) - (start >> c.lpage) + 1 : 0;
  bool lost = false;
  for (int i0 = 0; i0 < np; i0 += 64 * DEC_NW) {  // the last id again by who has none left
    const int i = min(i0 + (int)threadIdx.x, np - 1);
    const int pid = i0 == 0 && (int)threadIdx.x < np ? pid0 : tab[i];
    const bool ok = pid >= 0 && pid < c.n_pages;
    s_page[i] = ok ? pid : -1;
    lost |= !ok;
  }
  if (a.rows.err && __any(lost)) a.rows.err[b] = 1;

  // the query columns' operands, in LDS for all waves: block (cb, step, plane), 16
  // bytes a lane
  bf16x8* s_q = (bf16x8*)(smem + a.lds_pages);
  const size_t es = QP == 1 ? 2 : 4;
  for (int x = w; x < CB * NS; x += DEC_NW) {
    const int cc = col0 + min(16 * (x / NS) + i16, ncol - 1);
    const char* p = (const char*)a.q +
                    ((size_t)(sr.r0 + cc / G) * a.ldq + (size_t)(kvh * G + cc % G) * HD) * es;
    bf16x8 y[QP];
    load_q<QP>(p + dim_of<E4>(x % NS, g) * es, QP != 1, y);
#pragma unroll
    for (int n = 0; n < QP; ++n) s_q[(x * QP + n) * 64 + lane] = y[n];
  }
  __syncthreads();

  f32x4 o[CB][ND];
  float m[CB], l[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    m[cb] = -FLT_MAX;
    l[cb] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[cb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // granule gr of the tile at t0: its page's first token of this head, or -1
  auto granule = [&](int t0, int gr) -> long long {
    const int p = t0 + GRAN * gr;
    if (p >= stop) return -1;
    const int pid = s_page[(p >> c.lpage) - (start >> c.lpage)];
    if (pid < 0) return -1;
    return (((long long)pid * c.hkv + kvh) << c.lpage) + (p & (c.page - 1));
  };
  // Loads of places that hold no token (past the end, invalid pages) read the
  // cache's first page; what they bring is masked.
  constexpr size_t eb = E4 ? 1 : 2;
  auto load_k = [&](TileT& t, int t0) {
#pragma unroll
    for (int gr = 0; gr < 4; ++gr) {
      const long long tok = max(granule(t0, gr), 0ll);
      const int hi = __builtin_amdgcn_readfirstlane((int)(tok >> 32));
      const uint32_t lo = __builtin_amdgcn_readfirstlane((int)tok);
      const char* p = (const char*)c.k + (((size_t)hi << 32) | lo) * TileT::RB;
#pragma unroll
      for (int u = 0; u < TileT::PG; ++u)
        t.k[gr * TileT::PG + u] = *(const u32x4*)(p + 1024 * u + 16 * lane);
    }
  };
  auto load_v = [&](TileT& t, long long tok) {
    const char* p = (const char*)c.v + ((size_t)max(tok, 0ll) * HD + (size_t)i16 * GRAN) * eb;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < TileT::VJ; ++j)
        t.v[d][j] = *(const u32x4*)(p + (size_t)(16 * d) * GRAN * eb + 16 * j);
  };
  auto load_s = [&](float& ks, float& vs, long long tok) {
    if (!E4) return;
    ks = c.k_scale[(size_t)(max(tok, 0ll) >> c.lblock)];
    vs = c.v_scale[(size_t)(max(tok, 0ll) >> c.lblock)];
  };

  const float sc = a.scale * LOG2E;
  unsigned char* kb =  // this wave's keys
      smem + a.lds_pages + CB * NS * QP * 1024 + w * (KT * TileT::RB);
  TileT t;
  auto stage = [&]() {
#pragma unroll
    for (int u = 0; u < TileT::KU; ++u)
      *(u32x4*)(kb + TileT::at((64 / TileT::CH) * u + lane / TileT::CH, lane % TileT::CH)) = t.k[u];
  };
  // One tile whose keys lie in LDS and whose values are in flight.  MASK: some of its
  // keys are past a column's length or on an invalid page.  Both forms compute the
  // same bits of what is not masked.
  auto tile = [&](auto mask_, int t0, bool have, float ksc,
                  float vsc) __attribute__((always_inline)) {
#pragma clang fp contract(off)
    constexpr bool MASK = decltype(mask_)::value;
    // scores: row 4 g + v of subtile kt is key 16 g + 4 kt + v, column lane % 16
    f32x4 s[CB][4];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) s[cb][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int row = 16 * (i16 >> 2) + (i16 & 3);
    u32x4 x[4];
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      if (!E4 || (st & 1) == 0)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
          x[kt] = *(const u32x4*)(kb + TileT::at(row + 4 * kt, (E4 ? 2 : 4) * st + g));
      bf16x8 qq[CB][QP];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int n = 0; n < QP; ++n) qq[cb][n] = s_q[((cb * NS + st) * QP + n) * 64 + lane];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        const bf16x8 kk = !E4        ? __builtin_bit_cast(bf16x8, x[kt])
                          : (st & 1) ? widen(x[kt][2], x[kt][3], 1.f)
                                     : widen(x[kt][0], x[kt][1], 1.f);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int n = 0; n < QP; ++n)
            s[cb][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qq[cb][n], s[cb][kt], 0, 0, 0);
      }
      if (CB > 1) __builtin_amdgcn_sched_barrier(0);  // keeps operands from piling up
    }
    // softmax step
    bf16x8 p[CB][2][PP];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          float x = s[cb][kt][v] * ksc;
          if (MASK && !(have && t0 + 16 * g + 4 * kt + v < len[cb])) x = -INFINITY;
          s[cb][kt][v] = x;
          mx = fmaxf(mx, x);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m[cb], mx);
      if (__any(mn != m[cb])) {  // otherwise the factor is 1
        const float al = __builtin_amdgcn_exp2f(m[cb] - mn);
        m[cb] = mn;
        l[cb] *= al;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[cb][d] *= al;
      }
      float sum = 0.f;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float e = __builtin_amdgcn_exp2f(s[cb][kt][v] - mn);
          sum += e;
          // one plane holds a probability to 2^-8, as a bf16 output is held; three
          // (float32 rows) to 2^-24 (two, 2^-16, lose digits of the output)
          __bf16 y[PP];
          planes_of<PP>(e, y);
#pragma unroll
          for (int n = 0; n < PP; ++n) p[cb][kt >> 1][n][4 * (kt & 1) + v] = y[n];
        }
      l[cb] += sum;  // of this lane group's keys
      if (CB > 1) __builtin_amdgcn_sched_barrier(0);
    }
    // values
    auto operand = [&](int d, int st, int upto) {  // tokens from `upto` on as 0
      if (E4) {
        uint32_t w0 = t.v[d][0][2 * st], w1 = t.v[d][0][2 * st + 1];
        if (MASK) {
          w0 &= bytes_below(upto - 8 * st);
          w1 &= bytes_below(upto - 8 * st - 4);
        }
        return widen(w0, w1, vsc);
      }
      u32x4 x = t.v[d][TileT::VJ == 2 ? st : 0];
      if (MASK)
#pragma unroll
        for (int y = 0; y < 4; ++y) x[y] &= bytes_below(2 * (upto - 8 * st - 2 * y));
      return __builtin_bit_cast(bf16x8, x);
    };
    // this lane group's tokens below the longest and below the shortest length
    const int upto = MASK && have ? min(lmax - (t0 + GRAN * g), GRAN) : 0;
    if (MASK) {
      const int from = have ? min(lmin - (t0 + GRAN * g), GRAN) : 0;
      uint32_t odd = 0;  // an infinite or NaN value between the two
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < TileT::VJ; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            if (E4) {
              const uint32_t in = bytes_below(upto - 4 * x) & ~bytes_below(from - 4 * x);
              odd |= ((t.v[d][j][x] & 0x7F7F7F7Fu & in) + 0x01010101u) & 0x80808080u;
            } else {
              const int at = 8 * j + 2 * x;
              const uint32_t in = bytes_below(2 * (upto - at)) & ~bytes_below(2 * (from - at));
              const uint32_t z = t.v[d][j][x] & 0x7FFF7FFFu & in;
              odd |= (z & 0xFFFFu) >= 0x7F80u || (z >> 16) >= 0x7F80u;
            }
          }
      if (__any(odd != 0)) {  // row by row, every one with its own length
        for (int r = col0 / G; r <= (col0 + ncol - 1) / G; ++r) {
          const int rl = row_len(a, sr, b, r, over);
          const int mine = have ? min(rl - (t0 + GRAN * g), GRAN) : 0;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            f32x4 add[CB];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) add[cb] = o[cb][d];
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              const bf16x8 vv = operand(d, st, mine);
#pragma unroll
              for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int n = 0; n < PP; ++n)
                  add[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p[cb][st][n], add[cb], 0, 0, 0);
            }
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
              if ((col0 + 16 * cb + i16) / G == r) o[cb][d] = add[cb];
          }
        }
        return;
      }
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) {
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const bf16x8 vv = operand(d, st, upto);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int n = 0; n < PP; ++n)
            o[cb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p[cb][st][n], o[cb][d], 0, 0, 0);
      }
      if (CB > 1 && (d & 1)) __builtin_amdgcn_sched_barrier(0);
    }
  };

  // tiles that every column attends whole, each one's loads in flight during the
  // arithmetic of the one before; then the others
  constexpr int STEP = DEC_NW * KT;
  const int whole = min(stop, lmin);
  int t0 = start + w * KT;
  bool bad = false;  // an invalid page among them
  float ks = 1.f, vs = 1.f;
  if (t0 + KT <= whole) {
    long long tok = granule(t0, g);  // of this lane group's keys and values
    load_k(t, t0);
    load_s(ks, vs, tok);
    load_v(t, tok);
    for (; t0 + KT <= whole; t0 += STEP) {
      const bool ok = __all(tok >= 0);
      const float ksc = ks * sc, vsc = vs;
      stage();
      tok = granule(t0 + STEP, g);
      load_k(t, t0 + STEP);
      load_s(ks, vs, tok);
      if (ok) tile(std::false_type{}, t0, true, ksc, vsc);
      bad |= !ok;
      load_v(t, tok);
    }
  }
  if (bad) t0 = start + w * KT;
  for (; t0 < stop; t0 += STEP) {
    const long long tok = granule(t0, g);
    const bool have = tok >= 0;
    if (t0 + KT <= whole && __all(have)) continue;
    load_k(t, t0);
    load_s(ks, vs, tok);
    load_v(t, tok);
    stage();
    tile(std::true_type{}, t0, have, ks * sc, have ? vs : 1.f);
  }
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    l[cb] += __shfl_xor(l[cb], 16);
    l[cb] += __shfl_xor(l[cb], 32);
  }

  // merge of the waves: record of wave w, column cc at (w 16 CB + cc) RS
  __syncthreads();  // the page ids and keys are no longer read
  float* rec = (float*)smem;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    float* x = rec + (size_t)(w * 16 * CB + 16 * cb + i16) * RS;
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f32x4*)(x + 16 * d + 4 * g) = o[cb][d];
    if (g == 0) {
      x[HD] = m[cb];
      x[HD + 1] = l[cb];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < ncol * (HD / 4); e += 64 * DEC_NW) {
    const int cc = e / (HD / 4), d = e % (HD / 4) * 4;
    const int row = (col0 + cc) / G, h = kvh * G + (col0 + cc) % G;
    const int n = row_len(a, sr, b, row, over);
    if (n <= start && a.part) continue;  // not read by the merge
    float mm = -FLT_MAX;
#pragma unroll
    for (int k = 0; k < DEC_NW; ++k) mm = fmaxf(mm, rec[(size_t)(k * 16 * CB + cc) * RS + HD]);
    float ll = 0.f;
    f32x4 oo{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < DEC_NW; ++k) {
      const float* x = rec + (size_t)(k * 16 * CB + cc) * RS;
      const float f = __builtin_amdgcn_exp2f(x[HD] - mm);
      ll = fmaf(x[HD + 1], f, ll);
      const f32x4 y = *(const f32x4*)(x + d);
#pragma unroll
      for (int v = 0; v < 4; ++v) oo[v] = fmaf(y[v], f, oo[v]);
    }
    const size_t r = sr.r0 + row;
    if (a.part) {
      float* x = a.part + ((r * a.hq + h) * a.nsplit_ld + split) * (HD + 2);
      *(float2*)(x + d) = make_float2(oo[0], oo[1]);
      *(float2*)(x + d + 2) = make_float2(oo[2], oo[3]);
      if (d == 0) *(float2*)(x + HD) = make_float2(mm * LN2, ll);
      continue;
    }
    const bool any = ll != 0.f;  // else the row attends nothing
    const float inv = 1.0f / ll;
    const size_t at = r * a.ldo + (size_t)h * HD + d;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float y = any ? oo[v] * inv : 0.f;
      if (QP == 1) ((bf16_t*)a.out)[at + v] = f2bf(y);
      else ((float*)a.out)[at + v] = y;
    }
    if (d == 0 && a.lse) a.lse[r * a.hq + h] = any ? mm * LN2 + logf(ll) : -INFINITY;
  }
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// max over the two lanes l and l + 32, to both: the instruction swaps the upper half
// of its first register with the lower half of the second
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One column by a wave, without matrix instructions: lanes take keys, then dims.  Only
// what it attends is read.
template <int HD, bool E4, int QP>
__device__ inline void column(const PagedAttn& a, const SeqRows& sr, int b,
                                                 int kvh, int cc, int start, int stop, int split) {
  constexpr int DPL = HD / 64;
  const PagedCache& c = a.cache;
  const int G = a.hq / c.hkv, lane = threadIdx.x & 63;
  const int h = kvh * G + cc % G;
  const size_t r = sr.r0 + cc / G;
  bool over = false;
  const int n = row_len(a, sr, b, cc / G, over);
  if (a.part && n <= start) return;
  const int* tab = a.rows.table + (size_t)b * a.rows.table_ld;
  float m = -FLT_MAX, l = 0.f, o[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) o[e] = 0.f;
  auto qv = [&](int d) {
    const size_t at = r * a.ldq + (size_t)h * HD + d;
    return QP == 1 ? bf2f(((const bf16_t*)a.q)[at]) : ((const float*)a.q)[at];
  };
  auto cached = [&](const void* p, size_t at) {
    return E4 ? value_of(((const uint8_t*)p)[at]) : bf2f(((const bf16_t*)p)[at]);
  };
  for (int t0 = start; t0 < min(stop, n); t0 += 64) {
    const int p = min(t0 + lane, min(stop, n) - 1);
    const int pid = tab[p >> c.lpage];
    const bool ok = t0 + lane < min(stop, n) && pid >= 0 && pid < c.n_pages;
    const size_t tok = ok ? (((size_t)pid * c.hkv + kvh) << c.lpage) + (p & (c.page - 1)) : 0;
    float s = 0.f;
    for (int d = 0; d < HD; ++d) s = fmaf(qv(d), cached(c.k, tok * HD + d), s);
    if (E4) s *= c.k_scale[tok >> c.lblock];
    s = ok ? s * (a.scale * LOG2E) : -INFINITY;
    const float mn = fmaxf(m, wave_max64(s));
    const float al = __builtin_amdgcn_exp2f(m - mn), e = __builtin_amdgcn_exp2f(s - mn);
    m = mn;
    l = l * al + group_sum<64>(e);
#pragma unroll
    for (int x = 0; x < DPL; ++x) o[x] *= al;
    for (int t = 0; t < 64; ++t) {
      if (!__shfl((int)ok, t)) continue;
      const float pt = __shfl(e, t);
      const size_t tt = ((size_t)__shfl((int)(tok >> 32), t) << 32) | (uint32_t)__shfl((int)tok, t);
      const float vsc = E4 ? c.v_scale[tt >> c.lblock] : 1.f;
#pragma unroll
      for (int x = 0; x < DPL; ++x) {
        const int d = DPL * lane + x;
        o[x] += pt * (cached(c.v, (tt & ~(size_t)15) * HD + (size_t)d * GRAN + (tt & 15)) * vsc);
      }
    }
  }
  const bool any = l != 0.f;
  if (a.part) {
    float* x = a.part + ((r * a.hq + h) * a.nsplit_ld + split) * (HD + 2);
#pragma unroll
    for (int e = 0; e < DPL; ++e) x[DPL * lane + e] = o[e];
    if (lane == 0) {
      x[HD] = m * LN2;
      x[HD + 1] = l;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) {
    const size_t at = r * a.ldo + (size_t)h * HD + DPL * lane + e;
    const float y = any ? o[e] / l : 0.f;
    if (QP == 1) ((bf16_t*)a.out)[at] = f2bf(y);
    else ((float*)a.out)[at] = y;
  }
  if (lane == 0 && a.lse) a.lse[r * a.hq + h] = any ? m * LN2 + logf(l) : -INFINITY;
}

// Many rows: a workgroup of four waves owns 128 query columns of one kv head of one
// sequence (a wave 32 of them) and walks the 64-key tiles of its split.  Wave w
// brings granule w of a tile (16 keys, 16 values): loaded one tile ahead, widened to
// bf16 once for all waves and put in LDS, where tiles alternate between two buffers,
// one barrier a tile.  Products are 32x32x16: S^T = K Q^T, key row i of a 32-key block
// being key 16 (i / 16) + 8 ((i / 4) % 2) + 4 ((i / 8) % 2) + i % 4, so that a lane's
// scores are, in order, the probabilities of 8 consecutive tokens that O^T = V^T P^T
// takes from it.
//  keys in LDS    row r: its 16-byte chunk c at slot c ^ f(r) ^ c / 8 (f: the bits of
//                 r in which the 8 lanes of a read differ; those of a write have
//                 every second chunk)
//  values in LDS  [granule][half of 8 tokens][dim], 16 bytes
// The matrix units bound it, with the vector arithmetic of the softmax between their
// products: 2048 rows of 32 heads, 235 GFLOP, in 306 us (770 TFLOP/s; a library product
// of 8192 cubed 1239).  128 columns a workgroup and two of them a CU: one works on its
// scores while the other multiplies; 64 columns with 16x16x32 products took 560 us.
// Masked places as in k_pg_dec; where an infinite or NaN value lies between the
// shortest and the longest length of a wave's columns they are computed again, one at
// a time (`column`).
template <int HD, bool E4, int QP>
__global__ __launch_bounds__(256, 2) void k_pg_chunk(PagedAttn a) {
#pragma clang fp contract(off)
  constexpr int PP = QP == 3 ? 3 : 1;
  constexpr int NK = HD / 16;                 // contraction steps of a score
  constexpr int ND = HD / 32;                 // blocks of 32 output dims
  constexpr int LU = E4 ? HD / 64 : HD / 32;  // 16-byte loads a lane of a granule
  constexpr int RB = 2 * HD;                  // bytes of a key row in LDS
  __shared__ __align__(16) unsigned char s_k[2][KT * RB];
  __shared__ __align__(16) unsigned char s_v[2][KT * RB];
  __shared__ __align__(16) int s_ok[2][4], s_odd[2][4];
  const PagedCache& c = a.cache;
  const int G = a.hq / c.hkv;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i32 = lane & 31, hf = lane >> 5;

  int id = blockIdx.x;
  const int kvh = id % c.hkv;
  id /= c.hkv;
  // blocks of late columns, which attend the most, first
  const int col0 = (a.cblocks - 1 - id % a.cblocks) * 128;
  id /= a.cblocks;
  const int b = id % a.rows.B, split = id / a.rows.B;
  const int start = split * a.span;
  const SeqRows sr = seq_rows(a.rows, b);
  if (a.rows.err && threadIdx.x == 0 && sr.over) a.rows.err[b] = 1;
  const int ncols = sr.n * G;
  if (ncols <= col0 || ncols <= a.col_min) return;

  // lengths: of this lane's columns, of the wave's, of the workgroup's
  bool over = false;
  const int wcol = col0 + 32 * w;  // the wave's first column
  const int col = min(wcol + i32, ncols - 1);
  const int len = row_len(a, sr, b, col / G, over);
  int lmin = len, lmax = len, wmin = INT32_MAX, wmax = 0;
  for (int x = 0; x < 2; ++x) {
    const int n = row_len(a, sr, b, min(col0 + 64 * x + lane, ncols - 1) / G, over);
    wmin = min(wmin, n);
    wmax = max(wmax, n);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lmin = min(lmin, __shfl_xor(lmin, o));
    lmax = max(lmax, __shfl_xor(lmax, o));
    wmin = min(wmin, __shfl_xor(wmin, o));
    wmax = max(wmax, __shfl_xor(wmax, o));
  }
  wmin = __builtin_amdgcn_readfirstlane(wmin);
  lmin = __builtin_amdgcn_readfirstlane(lmin);
  lmax = __builtin_amdgcn_readfirstlane(lmax);
  wmax = __builtin_amdgcn_readfirstlane(wmax);
  if (a.rows.err && __any(over)) a.rows.err[b] = 1;
  const int stop = min(wmax, start + a.span);
  if (start >= stop && split > 0) return;

  // query columns
  bf16x8 q[NK][QP];
  constexpr size_t es = QP == 1 ? 2 : 4;
  const char* qp = (const char*)a.q +
                   ((size_t)(sr.r0 + col / G) * a.ldq + (size_t)(kvh * G + col % G) * HD) * es;
#pragma unroll
  for (int s = 0; s < NK; ++s) {
    load_q<QP>(qp + (16 * s + 8 * hf) * es, QP != 1, q[s]);
    if (a.scale < 0.f)
#pragma unroll
      for (int n = 0; n < QP; ++n)
        q[s][n] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[s][n]) ^ 0x80008000u);
  }
  f32x16 o[ND];
  float m = -FLT_MAX, l = 0.f;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[d][v] = 0.f;

  // this wave's granule of a tile
  const int* tab = a.rows.table + (size_t)b * a.rows.table_ld;
  const int last_page = (a.rows.max_len - 1) >> c.lpage;
  u32x4 kr[LU], vr[LU];
  float ks = 1.f, vs = 1.f;
  int pid_next = 0;  // the next tile's page
  auto ask = [&](int t0) { return tab[min((t0 + GRAN * w) >> c.lpage, last_page)]; };
  int n_tok = 0;  // tokens of the registers' granule
  auto load = [&](int t0) __attribute__((always_inline)) {
    const int p = t0 + GRAN * w;
    const int pid = __builtin_amdgcn_readfirstlane(pid_next);
    pid_next = ask(t0 + KT);
    const bool in = pid >= 0 && pid < c.n_pages;
    if (p < stop && !in && a.rows.err) a.rows.err[b] = 1;
    n_tok = in ? min(max(stop - p, 0), GRAN) : 0;
    const size_t tok =
        n_tok > 0 ? (((size_t)pid * c.hkv + kvh) << c.lpage) + (p & (c.page - 1)) : 0;
    const char* kp = (const char*)c.k + tok * HD * (E4 ? 1 : 2) + 16 * lane;
    const char* vp = (const char*)c.v + tok * HD * (E4 ? 1 : 2) + 16 * lane;
#pragma unroll
    for (int u = 0; u < LU; ++u) kr[u] = *(const u32x4*)(kp + 1024 * u);
#pragma unroll
    for (int u = 0; u < LU; ++u) vr[u] = *(const u32x4*)(vp + 1024 * u);
    if (E4) {
      ks = c.k_scale[tok >> c.lblock];
      vs = c.v_scale[tok >> c.lblock];
    }
  };
  auto key_at = [](int r, int ch) {
    return r * RB + ((ch ^ ((r & 3) | ((r >> 3) & 1) << 2) ^ (ch >> 3)) << 4);
  };
  // into buffer buf; ragged: some column does not attend all of the tile
  auto put = [&](int buf, bool ragged) __attribute__((always_inline)) {
    if (ragged || n_tok < GRAN) {
      uint32_t odd = 0;
#pragma unroll
      for (int u = 0; u < LU; ++u)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if (E4) {
            vr[u][y] &= bytes_below(n_tok - 4 * y);
            odd |= ((vr[u][y] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
          } else {
            vr[u][y] &= bytes_below(2 * (n_tok - 8 * (lane & 1) - 2 * y));
            const uint32_t z = vr[u][y] & 0x7FFF7FFFu;
            odd |= (z & 0xFFFFu) >= 0x7F80u || (z >> 16) >= 0x7F80u;
          }
        }
      const bool any = __any(odd != 0);
      if (lane == 0) s_odd[buf][w] = any;
      if (n_tok == 0) vs = 1.f;
    }
#pragma unroll
    for (int u = 0; u < LU; ++u) {
      const int at = 1024 * u + 16 * lane;  // byte in the granule
      if (E4) {
        const int r = GRAN * w + at / HD, ch = at % HD / 8;
        *(bf16x8*)(s_k[buf] + key_at(r, ch)) = widen(kr[u][0], kr[u][1], ks);
        *(bf16x8*)(s_k[buf] + key_at(r, ch + 1)) = widen(kr[u][2], kr[u][3], ks);
        unsigned char* p = s_v[buf] + (2 * w * HD + at / 16) * 16;
        *(bf16x8*)p = widen(vr[u][0], vr[u][1], vs);
        *(bf16x8*)(p + 16 * HD) = widen(vr[u][2], vr[u][3], vs);
      } else {
        *(u32x4*)(s_k[buf] + key_at(GRAN * w + at / RB, at % RB / 16)) = kr[u];
        *(u32x4*)(s_v[buf] + ((2 * w + (lane & 1)) * HD + at / 32) * 16) = vr[u];
      }
    }
    if (lane == 0) s_ok[buf][w] = n_tok;
  };

  const float sc = fmaxf(fabsf(a.scale) * LOG2E, FLT_MIN);  // > 0: times -inf no NaN
  bool redo = false;
  auto tile = [&](int buf, int t0, bool mask) __attribute__((always_inline)) {
#pragma clang fp contract(off)
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
    const int r = 16 * (i32 >> 4) + 8 * ((i32 >> 2) & 1) + 4 * ((i32 >> 3) & 1) + (i32 & 3);
#pragma unroll
    for (int st = 0; st < NK; ++st)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8 kk = *(const bf16x8*)(s_k[buf] + key_at(r + 32 * kb, 2 * st + hf));
#pragma unroll
        for (int n = 0; n < QP; ++n)
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, q[st][n], s[kb], 0, 0, 0);
      }
    // register v of block kb is token 32 kb + 16 (v / 8) + 8 hf + v % 8
    if (mask) {
      const int n = len - t0 - 8 * hf;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int gr = 2 * kb + (v >> 3);
          if (!s_ok[buf][gr] || GRAN * gr + (v & 7) >= n) s[kb][v] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
    // queries carry the scale's sign, so sc > 0
    const float mn = fmaxf(m, max_halves(mx) * sc);
    if (__any(mn != m)) {
      const float al = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= al;
    }
    bf16x8 p[4][PP];
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[kb][v], sc, -mn));
        sum += e;
        __bf16 y[PP];
        planes_of<PP>(e, y);  // see k_pg_dec
#pragma unroll
        for (int n = 0; n < PP; ++n) p[2 * kb + (v >> 3)][n][v & 7] = y[n];
      }
    l += sum;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const bf16x8 vv = *(const bf16x8*)(s_v[buf] + ((2 * st + hf) * HD + 32 * d + i32) * 16);
#pragma unroll
        for (int n = 0; n < PP; ++n)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, p[st][n], o[d], 0, 0, 0);
      }
  };

  // tile t0 lies in buffer buf, the next one in the registers
  auto step = [&](auto buf_, int t0) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_)::value;
    put(buf ^ 1, t0 + 2 * KT > wmin);
    load(t0 + 2 * KT);
    __builtin_amdgcn_sched_barrier(0);  // the loads leave before the products
    if (t0 < lmax) {
      const int4 ok = *(const int4*)s_ok[buf];
      const bool mask = !__all(t0 + KT <= lmin && ok.x && ok.y && ok.z && ok.w);
      if (mask && t0 + KT > wmin) {
        const int4 odd = *(const int4*)s_odd[buf];
        redo |= __any(odd.x | odd.y | odd.z | odd.w);
      }
      tile(buf, t0, mask);
    }
    __syncthreads();
  };
  if (start < stop) {
    pid_next = ask(start);
    load(start);
    put(0, start + KT > wmin);
    load(start + KT);
    __syncthreads();
    for (int t0 = start; t0 < stop; t0 += 2 * KT) {
      step(std::integral_constant<int, 0>{}, t0);
      if (t0 + KT < stop) step(std::integral_constant<int, 1>{}, t0 + KT);
    }
  }
  if (redo) {  // an infinite or NaN value where some columns must not see it
    for (int cc = wcol; cc < min(wcol + 32, ncols); ++cc)
      column<HD, E4, QP>(a, sr, b, kvh, cc, start, stop, split);
    return;
  }

  // results: lane (i32, hf) has dims 32 d + 8 (v / 4) + 4 hf + v % 4 of its column
  l += __shfl_xor(l, 32);
  if (wcol + i32 >= ncols || (a.part && len <= start)) return;
  const size_t r = sr.r0 + col / G;
  const int h = kvh * G + col % G;
  const bool any = l != 0.f;
  const float inv = 1.0f / l;
  float* part = a.part ? a.part + ((r * a.hq + h) * a.nsplit_ld + split) * (HD + 2) : nullptr;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      const int dim = 32 * d + 2 * v + 4 * hf;
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = o[d][v + e];
      if (part) {
        *(float2*)(part + dim) = make_float2(y[0], y[1]);
        *(float2*)(part + dim + 2) = make_float2(y[2], y[3]);
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = any ? y[e] * inv : 0.f;
      const size_t at = r * a.ldo + (size_t)h * HD + dim;
      if (QP == 1) {
        bf16_t z[4] = {f2bf(y[0]), f2bf(y[1]), f2bf(y[2]), f2bf(y[3])};
        *(uint2*)((bf16_t*)a.out + at) = *(const uint2*)z;
      } else {
        *(float4*)((float*)a.out + at) = make_float4(y[0], y[1], y[2], y[3]);
      }
    }
  if (hf == 0) {
    if (part) *(float2*)(part + HD) = make_float2(m * LN2, l);
    else if (a.lse) a.lse[r * a.hq + h] = any ? m * LN2 + logf(l) : -INFINITY;
  }
}

// NW waves per (row, query head), U splits a wave at a time, join the splits that hold keys of the row, each of
// them every NW-th, in order, then the waves' results.  Partials are (o[hd], max,
// sum) with the maximum in natural units.  The first partials are requested before
// the row's length is known (what they hold then is not used), so the loads of a
// launch lie one memory latency deep, not three: 32 splits of one row's 32 heads 4.0 us
// with four waves, 12.2 with one that asks for the length first.
template <typename T, int HD, int NW, int U>
__global__ __launch_bounds__(256) void k_pg_merge(PagedAttn a) {
  constexpr int DPL = HD / 64;
  __shared__ float s_o[4][HD], s_m[4], s_l[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % NW;
  const int job = blockIdx.x * (4 / NW) + wave / NW;
  const int r = min(job / a.hq, a.rows.rows - 1), h = job % a.hq;
  const float* p = a.part + ((size_t)r * a.hq + h) * a.nsplit_ld * (HD + 2);
  float ms[U], ls[U], ov[U][DPL];
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float* x = p + (size_t)min(s0 + NW * k, a.nsplit - 1) * (HD + 2);
      ms[k] = x[HD];
      ls[k] = x[HD + 1];
#pragma unroll
      for (int e = 0; e < DPL; ++e) ov[k][e] = x[DPL * lane + e];
    }
  };
  load(w);
  const RowAt ra = row_at(a.rows, r);
  const bool mine = job < a.rows.rows * a.hq && ra.b >= 0;
  const int n = min(max(ra.p0 + ra.i + 1, 0), a.rows.max_len);
  const int ns = mine ? (n + a.span - 1) / a.span : 0;
  float m = -FLT_MAX, l = 0.f, o[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) o[e] = 0.f;
  for (int s0 = w; s0 < ns; s0 += NW * U) {
    if (s0 != w) load(s0);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (s0 + NW * k >= ns) break;
      const float mn = fmaxf(m, ms[k]);
      const float ea = __expf(m - mn), eb = __expf(ms[k] - mn);
      l = fmaf(ls[k], eb, l * ea);
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[e] = fmaf(ov[k][e], eb, o[e] * ea);
      m = mn;
    }
  }
  if (NW > 1) {
#pragma unroll
    for (int e = 0; e < DPL; ++e) s_o[wave][DPL * lane + e] = o[e];
    if (lane == 0) {
      s_m[wave] = m;
      s_l[wave] = l;
    }
    __syncthreads();
    if (w != 0) return;
    m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    l = 0.f;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float f = __expf(s_m[k] - m);
      l = fmaf(s_l[k], f, l);
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[e] = fmaf(s_o[k][DPL * lane + e], f, o[e]);
    }
  }
  if (!mine) return;
  T* dst = (T*)a.out + (size_t)r * a.ldo + (size_t)h * HD + DPL * lane;
  const bool any = l != 0.f;
  const float inv = 1.0f / l;
#pragma unroll
  for (int e = 0; e < DPL; ++e) st1(dst + e, any ? o[e] * inv : 0.f);
  if (lane == 0 && a.lse) a.lse[(size_t)r * a.hq + h] = any ? m + logf(l) : -INFINITY;
}

}  // namespace

void paged_append(const PagedAppend& a_, hipStream_t st) {
  PagedAppend a = a_;
  const PagedCache& c = a.cache;
  const int block = c.kind == KS_E4M3 ? c.block : GRAN;
  const int touched = (a.rows.max_rows + block - 2) / block + 1;
  const int n_kv = a.rows.B * c.hkv * touched;
  const int qw = APP_QW * 128 / c.hd;
  const int jobs = a.q ? a.rows.rows * ((a.hq + qw - 1) / qw) : 0;
  const dim3 grid(n_kv + (jobs + 3) / 4);
  const size_t es = a.dtype == KS_BF16 ? 2 : 4;
  auto al = [&](const void* p, size_t ld) { return (((uintptr_t)p | ld * es) & 15) == 0; };
  a.vec = (al(a.q, a.ldq) ? 1 : 0) | (al(a.q_out, a.ldqo) ? 2 : 0) | (al(a.k, a.ldk) ? 4 : 0) |
          (al(a.v, a.ldv) ? 8 : 0);
#define KS_APP(T_, HD_, E_) \
  KS_LAUNCH((k_pg_append<T_, HD_, E_>), grid, dim3(256), 0, st, a, n_kv, touched)
#define KS_APP_T(T_)                                                   \
  do {                                                                 \
    if (c.hd == 128 && c.kind == KS_E4M3) KS_APP(T_, 128, true);       \
    else if (c.hd == 128) KS_APP(T_, 128, false);                      \
    else if (c.kind == KS_E4M3) KS_APP(T_, 64, true);                  \
    else KS_APP(T_, 64, false);                                        \
  } while (0)
  if (a.dtype == KS_BF16) KS_APP_T(bf16_t);
  else KS_APP_T(float);
#undef KS_APP_T
#undef KS_APP
}

// Which kernel: a sequence of up to DEC_COLS query columns (rows times query heads of
// a kv head) goes to the split kernel, which reads the cache once per 32 of them, one of
// more to the chunk kernel, once per 128.  Split and chunk kernel, e4m3, 8 kv heads: 64
// columns over 8192 tokens 19 and 24 us, over 32768 34 and 39, 16 sequences over 4096 52
// and 59; 96 columns 32 and 23, 78 and 40, 99 and 59.
constexpr int DEC_COLS = 64;

constexpr int SPAN_MAX = 4096;
constexpr int SPAN_MIN = 4 * KT;
// rows times splits that a call with few blocks may add to its rows (see paged_plan):
// 255 workgroups of 32 columns, or 512 of 128
static int split_room(int hq, int cols) {
  return ((cols > DEC_COLS ? 512 * 128 : 255 * 32) + hq - 1) / hq;
}

PagedPlan paged_plan(int B, int hkv, int G, int rows, int max_rows, int max_len) {
  PagedPlan p;
  const int cols = max_rows * G;
  const bool chunk = cols > DEC_COLS;
  // Splits of the split kernel: as many as give every CU a workgroup (one sequence of
  // 32768 tokens: 17.8 us with 256 workgroups, 21.1 with 384 and 27.5 with 1024, the
  // rest being their start and the merge), none shorter than a tile for every wave,
  // and none longer than 4096 positions, which keeps sequences of different lengths
  // level (64 of 500 to 15000 tokens: 216 us, 225 to 250 with one split each).
  // Of the chunk kernel: as many as give every CU two workgroups, none shorter than 4
  // tiles (256 rows of 4 heads a kv head, one sequence of 32768: 167 us, 215 with one
  // workgroup a CU, 182 with four; 32 rows over 2048 tokens: 17 us, 22 with 8 tiles).
  const int width = chunk ? 128 : 32;
  const int blocks = B * hkv * ((cols + width - 1) / width);
  const int most = std::max(1, (max_len + SPAN_MIN - 1) / SPAN_MIN);
  int want = chunk ? 512 / std::max(1, std::min(blocks, 512)) : (255 + blocks) / blocks;
  // rows <= B max_rows: no limit, as blocks >= rows hq / width.  Rows behind the last
  // sequence have places in the workspace, too, so many of them mean fewer splits.
  want = (int)std::min<long long>(want, 1 + (long long)split_room(hkv * G, cols) / rows);
  if (!chunk || B > 1) want = std::max(want, (max_len + SPAN_MAX - 1) / SPAN_MAX);
  p.nsplit = std::max(1, std::min(want, most));
  p.span = ((max_len + p.nsplit - 1) / p.nsplit + KT - 1) / KT * KT;
  return p;
}

// Largest rows * nsplit (with nsplit > 1) of a plan with at most these rows and lengths.
long long paged_split_rows(int hq, int G, int rows, int max_rows, int max_len) {
  const long long room = split_room(hq, max_rows * G);
  const long long len = (max_len + SPAN_MAX - 1) / SPAN_MAX;
  const long long n = std::max(std::min<long long>(rows, room) + room, len > 1 ? rows * len : 0);
  return max_len <= SPAN_MIN ? 0 : std::min(n, (long long)rows * ((max_len + SPAN_MIN - 1) / SPAN_MIN));
}

void paged_attention(const PagedAttn& a_, hipStream_t st) {
  PagedAttn a = a_;
  const PagedCache& c = a.cache;
  const int G = a.hq / c.hkv;
  const int planes = a.planes ? a.planes : a.dtype == KS_BF16 ? 1 : 3;
  const bool chunk = !a.few && a.rows.max_rows * G > DEC_COLS;
#define KS_ATT_T(X_, QP_)                                              \
  do {                                                                 \
    if (c.hd == 128 && c.kind == KS_E4M3) X_(128, true, QP_);          \
    else if (c.hd == 128) X_(128, false, QP_);                         \
    else if (c.kind == KS_E4M3) X_(64, true, QP_);                     \
    else X_(64, false, QP_);                                           \
  } while (0)
#define KS_ATT(X_)                                                     \
  do {                                                                 \
    if (planes == 1) KS_ATT_T(X_, 1);                                  \
    else if (planes == 2) KS_ATT_T(X_, 2);                             \
    else KS_ATT_T(X_, 3);                                              \
  } while (0)
  if (chunk) {
    const int width = 128;
    a.col_min = a.rows.B > 1 ? DEC_COLS : 0;  // shorter sequences: below
    a.cblocks = (a.rows.max_rows * G + width - 1) / width;
    const dim3 grid((unsigned)((size_t)a.nsplit * c.hkv * a.cblocks * a.rows.B));
#define KS_CHK(HD_, E_, QP_) \
  KS_LAUNCH((k_pg_chunk<HD_, E_, QP_>), grid, dim3(256), 0, st, a)
    KS_ATT(KS_CHK);
#undef KS_CHK
  }
  if (!chunk || a.rows.B > 1) {
    a.col_max = chunk ? DEC_COLS : INT32_MAX;
    const int cols = std::min(a.rows.max_rows * G, a.col_max);
    const int CB = cols <= 16 ? 1 : 2;
    a.cblocks = (cols + 16 * CB - 1) / (16 * CB);
    const dim3 grid((unsigned)((size_t)a.nsplit * c.hkv * a.cblocks * a.rows.B));
    a.lds_pages = (a.span / c.page + 2) * 4 + 15 & ~15;
    const size_t lds = std::max((size_t)DEC_NW * 16 * CB * (c.hd + 4) * 4,
                                (size_t)a.lds_pages + CB * c.hd / 32 * planes * 1024 +
                                    DEC_NW * KT * c.hd * (c.kind == KS_E4M3 ? 1 : 2));
#define KS_DEC(HD_, E_, QP_)                                                              \
  do {                                                                                    \
    if (CB == 1) KS_LAUNCH((k_pg_dec<HD_, E_, QP_, 1>), grid, dim3(256), lds, st, a);     \
    else KS_LAUNCH((k_pg_dec<HD_, E_, QP_, 2>), grid, dim3(256), lds, st, a);             \
  } while (0)
    KS_ATT(KS_DEC);
#undef KS_DEC
  }
#undef KS_ATT
#undef KS_ATT_T
  if (!a.part || !a.out) return;
  // Up to eight splits are one wave's loads; as many as there may be, since the places of
  // missing ones are loaded, too (64 sequences of 8000 tokens, 128 rows each, 2 splits:
  // 1318 us, 1366 with eight loads).
  const int per = a.nsplit > 8 ? 1 : 4;  // (row, head) pairs of a workgroup
  const dim3 mgrid((unsigned)(((size_t)a.rows.rows * a.hq + per - 1) / per));
#define KS_MRG(T_, HD_)                                                                 \
  do {                                                                                  \
    if (per == 1) KS_LAUNCH((k_pg_merge<T_, HD_, 4, 8>), mgrid, dim3(256), 0, st, a);   \
    else if (a.nsplit > 4)                                                              \
      KS_LAUNCH((k_pg_merge<T_, HD_, 1, 8>), mgrid, dim3(256), 0, st, a);               \
    else if (a.nsplit > 2)                                                              \
      KS_LAUNCH((k_pg_merge<T_, HD_, 1, 4>), mgrid, dim3(256), 0, st, a);               \
    else                                                                                \
      KS_LAUNCH((k_pg_merge<T_, HD_, 1, 2>), mgrid, dim3(256), 0, st, a);               \
  } while (0)
  if (a.dtype == KS_BF16) {
    if (c.hd == 128) KS_MRG(bf16_t, 128);
    else KS_MRG(bf16_t, 64);
  } else {
    if (c.hd == 128) KS_MRG(float, 128);
    else KS_MRG(float, 64);
  }
#undef KS_MRG
}

}  // namespace ks
