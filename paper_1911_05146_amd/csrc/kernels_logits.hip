// Row operators on logits: log probability of a label with entropy, rank and the most likely classes, its gradient, and the
// distillation loss with its gradient.  A row's softmax is held as {m, rest, dot}: m its maximum, rest the sum of exp(s - m) over
// all classes but the one that holds the maximum, dot the sum of exp(s - m) (s - m).  With Z = 1 + rest, log Z = log1p(rest), so
// that log p and 1 - p keep their digits where one class is all but certain, and the entropy log Z - dot / Z adds two terms that
// are never negative.
//
// What none of them can do without is reading the logits once (and writing the gradient once).  A row, or one part of it, is read into registers as
// it is stored, 16 bytes per thread and unit, by one wave or by one work-group; every pass over it -- maximum, sums, list, gradient
// -- then takes it from there.  Long rows of few are divided among work-groups whose records a second launch joins.
#include <type_traits>

#include "hpf_answer.h"
#include "hpf_device.h"

namespace hpf {
namespace {

constexpr float INF = __builtin_huge_valf();
constexpr float LOG2E = 1.44269504f;
typedef unsigned long long Key;

__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }

struct RowSum {
  float m, rest, dot;
  static __device__ __forceinline__ RowSum none() { return RowSum{-INF, 0.f, 0.f}; }
  // this, but seen from the larger maximum o.m
  __device__ __forceinline__ void merge_into(const RowSum& o) {
    if (m == -INF) { const float r = rest; *this = o; rest += r; return; }   // r: 0, or NaN if there was a NaN but no number
    const float d = m - o.m, e = expf(d), z = rest + 1.f;
    const float dd = e > 0.f || e != e ? e * (dot + d * z) : 0.f;
    rest = o.rest + z * e;
    dot = o.dot + dd;
    m = o.m;
  }
  __device__ __forceinline__ void merge(const RowSum& o) {
    if (o.m > m) merge_into(o);
    else if (o.m == -INF) rest += o.rest;
    else { RowSum t = *this; *this = o; merge_into(t); }
  }
  __device__ __forceinline__ bool broken() const { return rest != rest || dot != dot || m == INF; }   // NaN or +infinity in the row
  __device__ __forceinline__ bool empty() const { return m == -INF; }                                 // every class masked
};

// Order of the list: larger value first, then lower index.  An unmasked class has a number above 0 in the upper half; 0 stands for none.
__device__ __forceinline__ unsigned order_of(float s) {
  const unsigned u = __float_as_uint(s + 0.f);   // -0 counts as 0
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
constexpr unsigned LOWEST = 0x00800000u;           // order of the lowest finite number
__device__ __forceinline__ float value_at(unsigned order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }
__device__ __forceinline__ Key key_of(float s, int c) { return (Key)order_of(s) << 32 | (0xffffffffu - (unsigned)c); }
__device__ __forceinline__ int class_of(Key k) { return (int)(0xffffffffu - (unsigned)k); }
__device__ __forceinline__ float value_of(Key k) { return value_at((unsigned)(k >> 32)); }

__device__ __forceinline__ Key shfl_xor(Key v, int o) {
  return (Key)(unsigned)__shfl_xor((int)(v >> 32), o) << 32 | (unsigned)__shfl_xor((int)(unsigned)v, o);
}

// Reductions over a wave without a trip through LDS: rotations within rows of 16 lanes, then the swaps of rows and halves.  Every lane gets
// the result, and the order is the same everywhere.
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <class V, class OP>
__device__ __forceinline__ V rows16(V v, OP op) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two registers");
  auto step = [&](auto c) {
    if constexpr (sizeof(V) == 4) {
      v = op(v, __builtin_bit_cast(V, dpp<decltype(c)::value>(__builtin_bit_cast(int, v))));
    } else {
      const Key k = __builtin_bit_cast(Key, v);
      v = op(v, __builtin_bit_cast(V, (Key)(unsigned)dpp<decltype(c)::value>((int)(k >> 32)) << 32 | (unsigned)dpp<decltype(c)::value>((int)(unsigned)k)));
    }
  };
  step(std::integral_constant<int, 0x128>{});   // row_ror 8, 4, 2, 1
  step(std::integral_constant<int, 0x124>{});
  step(std::integral_constant<int, 0x122>{});
  step(std::integral_constant<int, 0x121>{});
  return v;
}
template <class V, class OP>
__device__ __forceinline__ V wave_all(V v, OP op) {
  v = rows16(v, op);
  if constexpr (sizeof(V) == 4) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = op(__builtin_bit_cast(V, (unsigned)p[0]), __builtin_bit_cast(V, (unsigned)p[1]));
    const unsigned w = __builtin_bit_cast(unsigned, v);
    const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__builtin_bit_cast(V, (unsigned)q[0]), __builtin_bit_cast(V, (unsigned)q[1]));
  } else {
    for (int i = 0; i < 2; ++i) {
      const Key k = __builtin_bit_cast(Key, v);
      const unsigned lo = (unsigned)k, hi = (unsigned)(k >> 32);
      const auto a = i ? __builtin_amdgcn_permlane32_swap(lo, lo, false, false) : __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
      const auto b = i ? __builtin_amdgcn_permlane32_swap(hi, hi, false, false) : __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
      v = op(__builtin_bit_cast(V, (Key)(unsigned)b[0] << 32 | (unsigned)a[0]), __builtin_bit_cast(V, (Key)(unsigned)b[1] << 32 | (unsigned)a[1]));
    }
    return v;
  }
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

// NT threads that have a row together: 64 (a wave, with the LDS of its own that it is given) or a work-group.  LDS of a group:
template <int NT>
struct GroupSpace {
  static constexpr int CANDIDATES = NT == 64 ? 512 : 2048;
  float f[3][16];
  int i[16], n;
  unsigned bounds[NT == 64 ? 1 : 256], least;
  Key waves[16], list[64], next[64];
  __align__(16) Key keys[CANDIDATES];
};
template <int NT>
struct Group {
  GroupSpace<NT>& sh;
  int tid;      // 0 ... NT - 1
  __device__ __forceinline__ void sync() const {
    if (NT == 64) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); else __syncthreads();
  }
  // over all threads, the same order everywhere; every thread gets the results
  template <int N, class OP>
  __device__ __forceinline__ void reduce(float (&v)[N], OP op) const {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_all(v[k], op);
    if (NT == 64) return;
    __syncthreads();
    if ((tid & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) sh.f[k][tid >> 6] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if constexpr (NT == 1024) v[k] = rows16(sh.f[k][tid & 15], op);
      else {
        v[k] = sh.f[k][0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) v[k] = op(v[k], sh.f[k][w]);
      }
    }
  }
  __device__ __forceinline__ float max(float v) const {
    float a[1] = {v};
    reduce(a, larger);
    return a[0];
  }
  // sum over the waves of a number that all lanes of a wave have
  __device__ __forceinline__ int total(int per_wave) const {
    if (NT == 64) return per_wave;
    __syncthreads();
    if ((tid & 63) == 0) sh.i[tid >> 6] = per_wave;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t += sh.i[w];
    return t;
  }
  __device__ __forceinline__ Key max(Key v) const {
    v = wave_all(v, [](Key a, Key b) { return a > b ? a : b; });
    if (NT == 64) return v;
    __syncthreads();
    if ((tid & 63) == 0) sh.waves[tid >> 6] = v;
    __syncthreads();
    v = sh.waves[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = sh.waves[w] > v ? sh.waves[w] : v;
    return v;
  }
  // The `top` largest of everybody's keys, in order, to out(j, key); 0 where there are no more.  mine[]: the order of the largest value in each
  // quarter of what this thread has (0: none; a work-group of more than a wave needs mine[0] alone); each(border, f) calls f for all of its keys of
  // a value >= border; at(i), i < n, are all keys once more (0: none), those of equal values in the order of their classes.
  // A number that at least `top` of 256 groups' maxima reach is a lower bound of the last entry, a good one: what is not below it is
  // collected and ordered by counting.  Where that is too much, thousands of equal logits most likely, only what is above the bound is
  // collected, and of those at the bound the first; where that is too much still, `top` rounds of maxima decide: fp32 logits that the bound's 19 bits
  // do not tell apart, with a common offset of 1e4 for one, take 1222 us for 256 rows of 50257 and lists of 64 where others take 23.
  template <class EACH, class AT, class OUT>
  __device__ __forceinline__ void select(int top, const unsigned (&mine)[4], EACH each, AT at, int n, OUT out) const {
    constexpr int LANES = NT / 256;       // per group
    unsigned g[4] = {mine[0], mine[1], mine[2], mine[3]};
    if (NT > 64) {
      if (LANES >= 2) { const unsigned w = (unsigned)dpp<0xb1>((int)g[0]); g[0] = w > g[0] ? w : g[0]; }    // quad_perm 1 0 3 2
      if (LANES >= 4) { const unsigned w = (unsigned)dpp<0x4e>((int)g[0]); g[0] = w > g[0] ? w : g[0]; }    // quad_perm 2 3 0 1
      __syncthreads();
      if (tid % (LANES < 1 ? 1 : LANES) == 0) sh.bounds[tid / (LANES < 1 ? 1 : LANES)] = g[0];
      if (tid == 0) sh.n = 0;
      __syncthreads();
      if (tid < 64) {
        const uint4 q = *reinterpret_cast<const uint4*>(&sh.bounds[tid * 4]);
        g[0] = q.x; g[1] = q.y; g[2] = q.z; g[3] = q.w;
      }
    } else if (tid == 0) {
      sh.n = 0;
    }
    unsigned least = 0;
    if (tid < 64) {
      for (unsigned bit = 0x80000000u; bit >= 0x2000u; bit >>= 1) {       // 19 bits: as fine as bf16 and three more
        const unsigned t = least | bit;
        const int c = __popcll(__ballot(g[0] >= t)) + __popcll(__ballot(g[1] >= t)) + __popcll(__ballot(g[2] >= t)) + __popcll(__ballot(g[3] >= t));
        if (c >= top) least = t;
        if (c == top) break;
      }
      if (least < LOWEST) least = LOWEST;
      if (NT > 64 && tid == 0) sh.least = least;
    }
    sync();
    if (NT > 64) least = sh.least;
    auto collect = [&](Key k) {
      const int i = atomicAdd(&sh.n, 1);
      if (i < GroupSpace<NT>::CANDIDATES) sh.keys[i] = k;
    };
    if (mine[0] >= least || mine[1] >= least || mine[2] >= least || mine[3] >= least) each(value_at(least), collect);
    sync();
    int found = sh.n;
    if (found > GroupSpace<NT>::CANDIDATES) {
      sync();
      if (tid == 0) sh.n = 0;
      sync();
      for (int i = tid; i < n; i += NT) {
        const Key k = at(i);
        if ((unsigned)(k >> 32) > least) collect(k);
      }
      sync();
      found = sh.n;
      const bool few = found <= GroupSpace<NT>::CANDIDATES - 64;
      for (int i0 = 0; few && i0 < n && found < top; i0 += NT) {      // the first ones at the bound
        const Key k = i0 + tid < n ? at(i0 + tid) : 0;
        const bool is = (unsigned)(k >> 32) == least;
        const unsigned long long lanes = __ballot(is);
        if (NT > 64) {
          __syncthreads();
          if ((tid & 63) == 0) sh.i[tid >> 6] = __popcll(lanes);
          __syncthreads();
        }
        int place = found + __popcll(lanes & ((1ull << (tid & 63)) - 1)), all = 0;
        if (NT > 64) {
          for (int w = 0; w < NT / 64; ++w) {
            if (w < tid >> 6) place += sh.i[w];
            all += sh.i[w];
          }
        } else {
          all = __popcll(lanes);
        }
        if (is && place < top) sh.keys[place] = k;
        found = found + all < top ? found + all : top;
      }
      sync();
    }
    if (found <= GroupSpace<NT>::CANDIDATES) {
      for (int i = tid; i < found; i += NT) {
        const Key k = sh.keys[i];
        int above = 0, j = 0;
        for (; j + 8 <= found; j += 8) {
          const ulonglong2* q = reinterpret_cast<const ulonglong2*>(&sh.keys[j]);
          const ulonglong2 a = q[0], b = q[1], c = q[2], d = q[3];
          above += (a.x > k) + (a.y > k) + (b.x > k) + (b.y > k) + (c.x > k) + (c.y > k) + (d.x > k) + (d.y > k);
        }
        for (; j < found; ++j) above += sh.keys[j] > k;
        if (above < top) out(above, k);
      }
      for (int j = found + tid; j < top; j += NT) out(j, 0);
    } else {
      Key last = ~0ull;
      for (int j = 0; j < top; ++j) {
        Key best = 0;
        for (int i = tid; i < n; i += NT) {
          const Key k = at(i);
          if (k < last && k > best) best = k;
        }
        last = max(best);
        if (tid == 0) out(j, last);
      }
    }
    sync();
  }
};

// `len` elements from p on, held by NT threads as they are stored: unit j of thread t is 16-byte unit t + j * NT, counted from the 16-byte
// boundary at or before p.  Elements before p or behind the end read as -infinity.  Only the first and the last unit can lie across an end;
// these two are read and written element by element.
template <class T, int NT, int J>
struct Held {
  static constexpr int E = 16 / sizeof(T), CAPACITY = NT * J * E, UNITS = J, THREADS = NT;
  uint32_t v[J][4];
  int shift, len, tid;        // first element's place in its unit

  __device__ __forceinline__ bool used(int j) const { return j * NT * E - shift < len; }      // uniform
  __device__ __forceinline__ int first(int j) const { return (tid + j * NT) * E - shift; }
  __device__ __forceinline__ bool inside(int j) const { const int u = tid + j * NT; return u >= (shift ? 1 : 0) && u < (shift + len) / E; }

  // The units j < AHEAD of a row on their way to LDS, past the registers: each thread's own 16 bytes of `room` (NT * AHEAD units)
  template <int AHEAD>
  static __device__ __forceinline__ void fetch(const T* p, int n, int t, uint4* room) {
    const int shift = (int)(((uintptr_t)p & 15) / sizeof(T)), whole = (shift + n) / E, low = shift ? 1 : 0;
    const char* units = (const char*)(p - shift);      // uniform; a thread's offset is the same for every j
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (j * NT * E - shift >= n) break;
      if (t + j * NT >= low && t + j * NT < whole)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(units + j * (NT * 16) + (unsigned)t * 16u),
                                         (__attribute__((address_space(3))) void*)(room + j * NT + (t & ~63)), 16, 0, 0);
    }
  }
  // unit j of a row, from memory (or from `room`); an end's unit is left to edge
  __device__ __forceinline__ void load_unit(const T* p, int n, int t, int j, const uint4* room) {
    constexpr uint32_t NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    const int shift_ = (int)(((uintptr_t)p & 15) / sizeof(T)), u = t + j * NT;
    const char* units = (const char*)(p - shift_);
    uint4 q = make_uint4(NONE, NONE, NONE, NONE);
    if (u >= (shift_ ? 1 : 0) && u < (shift_ + n) / E) q = room ? room[u] : *reinterpret_cast<const uint4*>(units + j * (NT * 16) + (unsigned)t * 16u);
    v[j][0] = q.x; v[j][1] = q.y; v[j][2] = q.z; v[j][3] = q.w;
  }
  // Units j < AHEAD come from `room`, where fetch has brought them; units from DONE on are there already
  template <int AHEAD = 0, int DONE = J>
  __device__ __forceinline__ void load(const T* p, int n, int t, const uint4* room = nullptr) {
    shift = (int)(((uintptr_t)p & 15) / sizeof(T));
    len = n;
    tid = t;
    constexpr uint32_t NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
    for (int j = 0; j < DONE; ++j) {
      if (!used(j)) break;
      load_unit(p, n, t, j, j < AHEAD ? room : nullptr);
    }
    const int whole = (shift + n) / E;
    if (shift) edge(p, 0, NONE);
    if ((shift + n) % E && whole >= (shift ? 1 : 0)) edge(p, whole, NONE);
  }
  // unit u lies across an end of the row
  __device__ __forceinline__ void edge(const T* p, int u, uint32_t none) {
    uint32_t w[4] = {none, none, none, none};
    if (u % NT == tid) {
      uint32_t x[E];              // none behind a condition, so that all are on their way together
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = u * E - shift + e, at = i < 0 ? 0 : i < len ? i : len - 1;
        if constexpr (sizeof(T) == 4) x[e] = __float_as_uint(p[at]); else x[e] = p[at];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = u * E - shift + e;
        if (i >= 0 && i < len) {
          if constexpr (sizeof(T) == 4) w[e] = x[e];
          else w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | x[e] << 16 : (w[e >> 1] & 0xffff0000u) | x[e];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (u / NT == j && u % NT == tid) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = w[i];
      }
  }
  __device__ __forceinline__ float get(int j, int e) const {
    if (sizeof(T) == 4) return __uint_as_float(v[j][e]);
    return __uint_as_float(e & 1 ? v[j][e >> 1] & 0xffff0000u : v[j][e >> 1] << 16);
  }
  // Before a pass that converts what is stored again: without it the compiler keeps the fp32 values of one pass for the next, twice the registers
  __device__ __forceinline__ void renew() {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w) asm("" : "+v"(v[j][w]));
  }
  // Every element's f(value, j, e) to the same element of d.  Where d's elements do not have the same places within 16 bytes they are stored
  // one by one.  after(j): called when unit j is out of the way.
  template <class F, class G>
  __device__ __forceinline__ void store(T* d, F f, G after) {
    const bool alike = (int)(((uintptr_t)d & 15) / sizeof(T)) == shift;
    const int whole = (shift + len) / E;
    char* units = (char*)(d - shift);
    float x[E];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (!used(j)) break;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = f(get(j, e), j, e);
      T* at = (T*)(units + j * (NT * 16) + (unsigned)tid * 16u);
      if (inside(j)) {
        if (alike) {
          if constexpr (sizeof(T) == 2) store8((bf16_t*)at, x);
          else *reinterpret_cast<float4*>(at) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) from_f32(at + e, x[e]);
        }
      } else if (j == 0 || whole / NT == j) {
        const int e0 = first(j);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e0 + e >= 0 && e0 + e < len) from_f32(at + e, x[e]);
      }
      after(j);
    }
  }
  // f(value, j, e) for all units in use
  template <class F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (!used(j)) break;
#pragma unroll
      for (int e = 0; e < E; ++e) f(get(j, e), j, e);
    }
  }
};

// v_max3_f32: fmaxf would spend an instruction more per operand on signalling NaNs
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// One pass: the largest of the thread's elements, part[]: of the units j with j % 4 == i; and how many classes are before `label`, whose logit is
// `mine`: larger ones, and equal ones of lower index (COUNT; per wave).  base: class of the first element.  Counted with one comparison per
// element: units before the label's take the next smaller number as their border.
template <bool COUNT, class H>
__device__ __forceinline__ float look(H& h, float (&part)[4], int base, int label, float mine, int& before) {
  constexpr int E = H::E;
  const unsigned b = __float_as_uint(mine);
  const float below = mine == 0.f ? -__uint_as_float(1) : __uint_as_float(mine > 0.f ? b - 1 : b + 1);
  int n = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) part[i] = -INF;
#pragma unroll
  for (int j = 0; j < H::UNITS; ++j) {
    if (!h.used(j)) break;
    const float border = base + h.first(j) + E <= label ? below : mine;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float x = h.get(j, e), y = h.get(j, e + 1);
      part[j & 3] = max3(part[j & 3], x, y);
      if (COUNT) n += __popcll(__ballot(x > border)) + __popcll(__ballot(y > border));
    }
  }
  if (COUNT) {
    if (mine == -INF) {                        // a masked label, for which there is no smaller number
      n = 0;
      h.each([&](float s, int j, int e) {
        const int c = h.first(j) + e;
        n += __popcll(__ballot(s > mine || (s == mine && c >= 0 && c < h.len && base + c < label)));
      });
    } else if (label >= base && label - base < h.len) {
      // the label's own unit: equal logits in front of it, counted by the thread that holds it
      const int at = label - base + h.shift, unit = at / E, uj = unit / H::THREADS, ut = unit % H::THREADS;
#pragma unroll
      for (int j = 0; j < H::UNITS; ++j)
        if (uj == j)
#pragma unroll
          for (int e = 0; e < E; ++e) n += __popcll(__ballot(h.tid == ut && e < at % E && h.get(j, e) == mine));
    }
    before = n;
  }
  return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// {m, rest, dot} of what a group holds.  Only waves that hold a maximum keep it apart from the sum.  (s - m) log2 e stays a subtraction and a
// product: as one multiply-add it would be off by the rounding of m log2 e, without bound for large m.
template <class T, int NT, int J>
__device__ __forceinline__ RowSum sum_of(const Group<NT>& g, Held<T, NT, J>& h, float largest) {
  const float m = g.max(largest), mm = m == -INF ? 0.f : m;
  h.renew();
  float v[3] = {0.f, 0.f, 0.f};                // rest, dot (times log2 e), classes at the maximum
  if (NT == 64 || __any(largest == m)) {
    int ties = 0;
    h.each([&](float s, int, int) {
      const float x = (s - mm) * LOG2E, e = __builtin_amdgcn_exp2f(x);
      v[0] += x == 0.f ? 0.f : e;
      v[1] = fmaf(e, fmaxf(x, -200.f), v[1]);
      ties += __popcll(__ballot(x == 0.f));
    });
    v[2] = (g.tid & 63) == 0 ? (float)ties : 0.f;
  } else {
    h.each([&](float s, int, int) {
      const float x = (s - mm) * LOG2E, e = __builtin_amdgcn_exp2f(x);     // 0 below -150, in a masked class for one
      v[0] += e;
      v[1] = fmaf(e, fmaxf(x, -200.f), v[1]);
    });
  }
  g.reduce(v, [](float a, float b) { return a + b; });
  return RowSum{m, m == -INF ? v[0] : v[0] + (v[2] - 1.f), v[1] * 0.693147181f};
}

// ---- log probabilities ------------------------------------------------------------------------------------------------
// What a part of a row leaves for the join: its sum, how many of its classes are before the label, its list
struct PartRecord { RowSum sum; int before; };

__device__ __forceinline__ void write_row(const LogprobForward& a, int row, const RowSum& v, int before, int label, bool has, float mine) {
  const bool broken = v.broken();
  const float lz = v.empty() ? -INF : log1pf(v.rest);
  if (a.logprob)
    a.logprob[row] = label == -1 ? 0.f : (broken || !has) ? quiet_nan() : v.empty() ? -INF : (mine - v.m) - lz;   // both terms are <= 0
  if (a.rank) a.rank[row] = has && !broken ? before : -1;
  if (a.entropy) a.entropy[row] = broken ? quiet_nan() : v.empty() ? 0.f : lz - v.dot / (1.f + v.rest);
  if (a.stats) {
    a.stats[2 * (long)row] = broken ? quiet_nan() : v.m;
    a.stats[2 * (long)row + 1] = broken ? quiet_nan() : lz;
  }
}
__device__ __forceinline__ void write_entry(const LogprobForward& a, int row, int j, Key k, const RowSum& v, float lz) {
  const long at = (long)row * a.top + j;
  const bool broken = v.broken();
  a.top_index[at] = k && !broken ? class_of(k) : -1;
  a.top_logprob[at] = broken ? quiet_nan() : k ? (value_of(k) - v.m) - lz : -INF;
}

// the order of the largest value in each quarter of what a thread holds
template <int NT>
__device__ __forceinline__ void orders(unsigned (&best)[4], const float (&quarter)[4], float largest) {
#pragma unroll
  for (int i = 0; i < 4; ++i) best[i] = 0;
  if (NT == 64) {
#pragma unroll
    for (int i = 0; i < 4; ++i) best[i] = quarter[i] > -INF ? order_of(quarter[i]) : 0;
  } else if (largest > -INF) {
    best[0] = order_of(largest);
  }
}

// f for the keys of all elements >= border
template <class H, class F>
__device__ __forceinline__ void above(const H& h, const float (&quarter)[4], float border, int base, F f) {
#pragma unroll
  for (int j = 0; j < H::UNITS; ++j) {
    if (!h.used(j)) break;
    if (quarter[j & 3] >= border)
#pragma unroll
      for (int e = 0; e < H::E; ++e) {
        const float t = h.get(j, e);
        if (t >= border) f(key_of(t, base + h.first(j) + e));
      }
  }
}

// A row that a group holds whole.  s, label and mine are the same in all lanes.
template <class T, int NT, int J>
__device__ __forceinline__ void logprob_row(const LogprobForward& a, const Group<NT>& g, Held<T, NT, J>& h, const T* s, int row, int label, float mine) {
  const bool has = label >= 0 && label < a.classes;
  float quarter[4];
  int before = 0;
  const float largest = has ? look<true>(h, quarter, 0, label, mine, before) : look<false>(h, quarter, 0, label, mine, before);
  const RowSum v = sum_of(g, h, largest);
  if (has) before = g.total(before);
  if (g.tid == 0) write_row(a, row, v, before, label, has, mine);
  if (!a.top) return;
  if (v.broken()) {
    for (int j = g.tid; j < a.top; j += NT) write_entry(a, row, j, 0, v, 0.f);
    return;
  }
  unsigned best[4];
  orders<NT>(best, quarter, largest);
  const float lz = v.empty() ? 0.f : log1pf(v.rest);
  h.renew();
  g.select(a.top, best, [&](float border, auto f) { above(h, quarter, border, 0, f); }, [&](int i) -> Key {
    const float t = to_f32(s[i]);
    return t > -INF ? key_of(t, i) : 0;
  }, a.classes, [&](int j, Key k) { write_entry(a, row, j, k, v, lz); });
}

__device__ __forceinline__ int label_of(const int* labels, int row) { return labels ? __builtin_amdgcn_readfirstlane(labels[row]) : -1; }
template <class T>
__device__ __forceinline__ float logit_of(const T* s, int label, int classes) {
  return label >= 0 && label < classes ? __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(to_f32(s[label])))) : INF;
}

// Rows that a wave, 256 or 512 threads hold.  Bound by instructions and by what the row's phases wait for (its bytes, reductions, the list),
// not by memory, so several rows are on a CU at a time, each in another phase: of 512 threads with 128 registers two.  2048 rows of 50257 bf16
// logits with lists of 64: 88 us (2.3 TB/s; 57 without lists), where one work-group of 1024 threads per CU took 131 although the next
// row was on its way to LDS meanwhile, and 256 threads with 28 units 101.  8192 rows of 1000 fp32 logits, a wave each: 16.6 us (2.0 TB/s).
template <class T, int NT, int J, int PER>       // PER: rows per work-group
__global__ __launch_bounds__(NT * PER, NT == 512 ? 4 : 1) void k_logprob_forward(LogprobForward a) {
  __shared__ GroupSpace<NT> space[PER];
  const int which = PER == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / NT);
  const Group<NT> g{space[which], (int)threadIdx.x % NT};
  const int row = blockIdx.x * PER + which;
  if (row >= a.rows) return;                           // a whole wave, or nobody
  const T* s = (const T*)a.logits + row * a.ld;
  Held<T, NT, J> h;
  h.load(s, a.classes, g.tid);
  const int label = label_of(a.labels, row);
  logprob_row(a, g, h, s, row, label, logit_of(s, label, a.classes));
}

// Rows that fill a CU's registers (more than 8192 units): one work-group per CU goes through rows one after the other.  While it works on one row
// in registers half of the next one is on its way to LDS (AHEAD units per thread).  2048 rows of 131072 bf16 logits: 200 us (2.7 TB/s).
template <class T, int J, int AHEAD>
__global__ __launch_bounds__(1024) void k_logprob_rows(LogprobForward a) {
  typedef Held<T, 1024, J> H;
  __shared__ GroupSpace<1024> space;
  extern __shared__ __align__(16) uint4 room[];
  int row = blockIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  H::template fetch<AHEAD>(s, a.classes, (int)threadIdx.x, room);
  for (; row < a.rows; row += gridDim.x) {
    s = (const T*)a.logits + row * a.ld;
    int t = (int)threadIdx.x;
    asm("" : "+v"(t));                               // a row's own: else the compiler keeps what all rows have in common, indices above all
    const Group<1024> g{space, t};
    H h;
    __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0): the thread's units are in LDS
    h.template load<AHEAD>(s, a.classes, g.tid, room);
    const int label = label_of(a.labels, row);
    const float mine = logit_of(s, label, a.classes);
    __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0): they are read
    if (row + (int)gridDim.x < a.rows) H::template fetch<AHEAD>(s + gridDim.x * a.ld, a.classes, g.tid, room);
    logprob_row(a, g, h, s, row, label, mine);
  }
}

// Few long rows (one of 131072 bf16 logits with a list of 20: 8.6 us, and 5.5 for the join; a launch alone takes 3.6).
// Rows divided among work-groups: group `part` of `parts` takes every chunk of CAPACITY elements from part * per_part on
template <class T, int J>
__global__ __launch_bounds__(256) void k_logprob_part(LogprobForward a, int parts, long per_part, PartRecord* records, Key* lists) {
  typedef Held<T, 256, J> H;
  __shared__ GroupSpace<256> space;
  const Group<256> g{space, (int)threadIdx.x};
  const unsigned unit = blockIdx.x;
  const int row = (int)(unit / (unsigned)parts), part = (int)(unit - (unsigned)row * parts);
  const T* s = (const T*)a.logits + row * a.ld;
  const int label = label_of(a.labels, row);
  const bool has = label >= 0 && label < a.classes;
  const long c_begin = part * per_part, c_end = c_begin + per_part < a.classes ? c_begin + per_part : a.classes;
  RowSum v = RowSum::none();
  float mine = INF;
  int before = 0;
  Key held = 0;                                        // entry g.tid of the list of the chunks so far, which is in LDS too
  int kept = 0;
  H h;
  auto load = [&](long c0) {
    const long room = H::CAPACITY - (long)(((uintptr_t)(s + c0) & 15) / sizeof(T)), step = c_end - c0 < room ? c_end - c0 : room;
    h.load(s + c0, (int)step, g.tid);
    return step;
  };
  long step = load(c_begin);
  mine = logit_of(s, label, a.classes);
  for (long c0 = c_begin;;) {
    float quarter[4];
    int n = 0;
    const float largest = has ? look<true>(h, quarter, (int)c0, label, mine, n) : look<false>(h, quarter, (int)c0, label, mine, n);
    before += n;
    const RowSum w = sum_of(g, h, largest);
    if (c0 == c_begin) v = w; else v.merge(w);
    const bool more = c0 + step < c_end;
    if (a.top && !v.broken()) {
      unsigned best[4];
      orders<256>(best, quarter, largest);
      if ((unsigned)(held >> 32) > best[0]) best[0] = (unsigned)(held >> 32);
      h.renew();
      g.select(a.top, best, [&](float border, auto f) {
        if (held && value_of(held) >= border) f(held);
        above(h, quarter, border, (int)c0, f);
      }, [&](int i) -> Key {
        if (i < a.top) return i < kept ? g.sh.list[i] : 0;             // classes of earlier chunks come first
        const float t = to_f32(s[c0 + i - a.top]);
        return t > -INF ? key_of(t, (int)c0 + i - a.top) : 0;
      }, (int)step + a.top, [&](int j, Key k) {
        if (more) g.sh.next[j] = k;                                    // the list goes on, in LDS
        else lists[(long)unit * a.top + j] = k;
      });
      if (more) {
        held = g.tid < a.top ? g.sh.next[g.tid] : 0;
        if (g.tid < a.top) g.sh.list[g.tid] = held;
        kept = a.top;
        g.sync();
      }
    }
    if (!more) break;
    c0 += step;
    step = load(c0);
  }
  if (a.top && v.broken())
    for (int j = g.tid; j < a.top; j += 256) lists[(long)unit * a.top + j] = 0;
  before = g.total(before);
  if (g.tid == 0) records[unit] = PartRecord{v, before};
}

// The sums of a row from those of its parts, one per thread (RowSum::none() where there is none): seen from the largest maximum, which the first
// part that holds it keeps out of its sum
__device__ __forceinline__ bool holds_maximum(const Group<256>& g, float m, float& top) {
  const Key k = g.max((Key)order_of(m) << 32 | (0xffffffffu - (unsigned)g.tid));
  top = value_of(k);
  return (unsigned)k == 0xffffffffu - (unsigned)g.tid;
}
__device__ __forceinline__ RowSum join_parts(const Group<256>& g, const RowSum& p) {
  float m;
  const bool base = holds_maximum(g, p.m, m);
  float v[2] = {p.rest, p.dot};
  if (!base && p.m != -INF) {
    const float d = p.m - m, e = expf(d), z = 1.f + p.rest;
    v[0] = z * e;
    v[1] = e > 0.f || e != e ? e * (p.dot + d * z) : 0.f;
  }
  g.reduce(v, [](float a, float b) { return a + b; });
  return RowSum{m, v[0], v[1]};
}

// a.parts <= 256 records and lists of a row
template <class T>
__global__ __launch_bounds__(256) void k_logprob_join(LogprobForward a, int parts, const PartRecord* __restrict__ records, const Key* __restrict__ lists) {
  __shared__ GroupSpace<256> space;
  const Group<256> g{space, (int)threadIdx.x};
  const int row = blockIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  const int label = a.labels ? a.labels[row] : -1;
  const bool has = label >= 0 && label < a.classes;
  const float mine = has ? to_f32(s[label]) : 0.f;
  PartRecord rec{RowSum::none(), 0};
  if (g.tid < parts) rec = records[(long)row * parts + g.tid];
  const Key* list = lists + (long)row * parts * a.top;
  const int n = parts * a.top;
  unsigned best[4] = {0, 0, 0, 0};
  for (int i = g.tid; i < n; i += 256) best[0] = (unsigned)(list[i] >> 32) > best[0] ? (unsigned)(list[i] >> 32) : best[0];
  const RowSum v = join_parts(g, rec.sum);
  const int before = g.total(wave_all(rec.before, [](int a, int b) { return a + b; }));
  if (g.tid == 0) write_row(a, row, v, before, label, has, mine);
  if (!a.top) return;
  const float lz = v.empty() ? 0.f : log1pf(v.rest);
  g.select(a.top, best, [&](float border, auto f) { for (int i = g.tid; i < n; i += 256) if (list[i] && value_of(list[i]) >= border) f(list[i]); },
           [&](int i) { return list[i]; }, n, [&](int j, Key k) { write_entry(a, row, j, k, v, lz); });
}

// ---- gradient of log probability and entropy ---------------------------------------------------------------------------
// Every work-group has 1024 16-byte units of a row, all on their way before the first is used.  Bound by memory: 2048 rows of 50257 bf16 logits
// in 76 us (5.4 TB/s read and written; a copy reaches 6.3).
template <class T>
__global__ __launch_bounds__(256) void k_logprob_backward(LogprobBackward a, unsigned blocks_per_row) {
  constexpr int U = 4;
  typedef Held<T, 256, U> H;
  const int row = (int)(blockIdx.x / blocks_per_row);
  const int b = (int)(blockIdx.x - (unsigned)row * blocks_per_row);
  const T* s = (const T*)a.logits + row * a.ld;
  T* d = (T*)a.dlogits + row * a.ldd;
  // blocks of whole units, counted from the 16-byte boundary at or before the row
  const int shift = (int)(((uintptr_t)s & 15) / sizeof(T));
  const long c0 = b ? (long)b * H::CAPACITY - shift : 0, c1 = (long)(b + 1) * H::CAPACITY - shift;
  if (c0 >= a.classes) return;
  H h;
  h.load(s + c0, (int)((c1 < a.classes ? c1 : a.classes) - c0), threadIdx.x);
  const int label = a.grad_logprob ? a.labels[row] : -1;
  const float m = a.stats[2 * (long)row], lz = a.stats[2 * (long)row + 1];
  float g = label != -1 ? a.grad_logprob[row] : 0.f;
  if (label < -1 || label >= a.classes) g = quiet_nan();
  const float gh = a.grad_entropy ? a.grad_entropy[row] : 0.f, entropy = a.grad_entropy ? a.entropy[row] : 0.f;
  const float ng = -g, ngh = -gh;
  auto grad = [&](float x) {
    const float logp = (x - m) - lz, p = __builtin_amdgcn_exp2f(logp * LOG2E);
    // p is 0 below exp(-104), in a masked class for one, and the entropy's p log p with it
    return m == -INF ? 0.f : p * fmaf(ngh, fmaxf(logp, -120.f) + entropy, ng);
  };
  auto grad_label = [&](float x) {             // 1 - p from log p
    const float logp = (x - m) - lz, p = __builtin_amdgcn_exp2f(logp * LOG2E);
    return m == -INF ? 0.f : fmaf(ngh * p, fmaxf(logp, -120.f) + entropy, ng * expm1f(logp));
  };
  const int at_label = label - (int)c0;
  h.store(d + c0, [&](float x, int, int) { return grad(x); }, [](int) {});
  // the label's, once more
  const int unit = (at_label + h.shift) / H::E;
  if (label >= 0 && label < a.classes && at_label >= 0 && at_label < h.len && unit % 256 == h.tid) {
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (unit / 256 == j)
#pragma unroll
        for (int e = 0; e < H::E; ++e)
          if (h.first(j) + e == at_label) from_f32(d + label, grad_label(h.get(j, e)));
  }
}

// ---- distillation --------------------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v) { return wave_all(v, [](double a, double b) { return a + b; }); }

// What the student's row leaves for the loss: the maximum and the sums of the other classes at temperature 1 and T
struct Soft { float m, rest1, restt; };
__device__ __forceinline__ void merge(Soft& v, const Soft& o, float it) {
  RowSum a{v.m, v.rest1, 0.f};
  a.merge(RowSum{o.m, o.rest1, 0.f});
  // at temperature T the distance of the maxima counts 1 / T of itself
  float t;
  if (v.m == -INF || o.m == -INF) t = v.restt + o.restt;     // of a part of masked classes: 0, or NaN
  else if (v.m >= o.m) t = v.restt + (1.f + o.restt) * expf((o.m - v.m) * it);
  else t = o.restt + (1.f + v.restt) * expf((v.m - o.m) * it);
  v = Soft{a.m, a.rest, t};
}

// What a row's list says, one entry per lane, by one wave: the loss's soft part and the gradient at the listed classes
struct List {
  bool on, some, broken;     // entry there; any entry there; an index outside the classes
  int index;
  float mine;                // the student's logit at the entry's class
  double p, logp;            // probability of the entry
  double soft;               // sum_j p_j (log p_j - log q_j)
  double diff;               // q_c - P_c, P_c: probability of the entry's class in the list (all entries of that class)
};
// what does not need the row's sums
template <class T>
__device__ __forceinline__ List read_list(const Distill& a, const T* s, int row, int lane) {
  List l{};
  const long at = (long)row * a.top + lane;
  l.index = lane < a.top ? a.top_index[at] : -1;
  const float t = l.index >= 0 ? a.top_logit[at] : -INF;
  l.on = t != -INF;
  l.broken = __any(l.on && l.index >= a.classes);
  l.some = __any(l.on);
  l.mine = l.on && l.index < a.classes ? to_f32(s[l.index]) : 0.f;
  if (!l.some) return l;
  const double d = ((double)t - (double)wave_all(t, larger)) / (double)a.temperature;
  const double e = l.on ? exp(d) : 0.0, z = wave_sum(e);
  l.p = e / z;
  l.logp = d - log(z);
  return l;
}
__device__ __forceinline__ void finish_list(const Distill& a, List& l, const Soft& v) {
  if (!l.some) return;
  const double logq = l.on ? ((double)l.mine - (double)v.m) / (double)a.temperature - log1p((double)v.restt) : 0.0;
  l.soft = wave_sum(l.on && l.p != 0.0 ? l.p * (l.logp - logq) : 0.0);
  int same = 0;              // entries of this lane's class
  for (int j = 0; j < a.top; ++j) same += __builtin_amdgcn_readlane(l.index, j) == l.index;
  double p = l.p, logp = l.logp;
  if (__any(l.on && same > 1)) {
    p = 0.0;
    for (int j = 0; j < a.top; ++j) {
      const double pj = __shfl(l.p, j);
      if (__builtin_amdgcn_readlane(l.index, j) == l.index) p += pj;
    }
    logp = log(p);
  }
  // by the difference of the logarithms only where the two are close: expm1 overflows where p is a number below 2^-1022, and beyond a factor of e
  // the subtraction loses less than a digit
  const double d = logq - logp;
  l.diff = fabs(d) < 1.0 ? p * expm1(d) : exp(logq) - p;
}

// exp at temperature 1 next to exp at temperature T: HARD_EXP of its own, or HARD_ONE / HARD_TWO / HARD_FOUR: e^(1/T) to the power T = 1, 2, 4
// (an exponential costs four times a multiplication: rows by 512 threads and more, 2048 of 131072 classes at T = 2: 278 us, at T = 3: 296; shorter
// rows and divided ones take HARD_EXP)
enum : int { HARD_NONE = 0, HARD_EXP = 1, HARD_ONE = 2, HARD_TWO = 3, HARD_FOUR = 4 };
struct Exponents {
  float m, ct;
  __device__ __forceinline__ Exponents(float m_, float it) : m(m_ == -INF ? 0.f : m_), ct(it * LOG2E) {}
  __device__ __forceinline__ float soft(float s) const { return __builtin_amdgcn_exp2f((s - m) * ct); }
  template <int HARD>
  __device__ __forceinline__ float hard(float s, float et) const {
    if (HARD == HARD_ONE) return et;
    if (HARD == HARD_TWO) return et * et;
    if (HARD == HARD_FOUR) { const float q = et * et; return q * q; }
    return __builtin_amdgcn_exp2f((s - m) * LOG2E);
  }
};

// Sums of what a group holds at temperatures 1 (if HARD) and T, as in sum_of
template <int HARD, class T, int NT, int J>
__device__ __forceinline__ Soft soft_of(const Group<NT>& g, Held<T, NT, J>& h, float it) {
  float quarter[4];
  int none;
  const float largest = look<false>(h, quarter, 0, -1, 0.f, none), m = g.max(largest);
  const Exponents x(m, it);
  h.renew();
  float v[3] = {0.f, 0.f, 0.f};                // rest at T, rest at 1, classes at the maximum
  if (NT == 64 || __any(largest == m)) {
    int ties = 0;
    h.each([&](float s, int, int) {
      const bool is = s == m;
      const float e = x.soft(s);
      v[0] += is ? 0.f : e;
      if (HARD) v[1] += is ? 0.f : x.hard<HARD>(s, e);
      ties += __popcll(__ballot(is));
    });
    v[2] = (g.tid & 63) == 0 ? (float)ties : 0.f;
  } else {
    h.each([&](float s, int, int) {
      const float e = x.soft(s);
      v[0] += e;
      if (HARD) v[1] += x.hard<HARD>(s, e);
    });
  }
  g.reduce(v, [](float a, float b) { return a + b; });
  const float ties = m == -INF ? 0.f : v[2] - 1.f;
  return Soft{m, v[1] + ties, v[0] + ties};
}

// Loss of a row, its gradient's factors, and the entries that are taken from the logarithms
template <class T>
struct Answer {
  const Distill& a;
  const T* s;
  int row, label;
  bool has, bad, empty;
  float mine;                // logit of the label
  double logl, ws, wh;       // log softmax at the label; weights of the soft and the hard term
  float fs, fh, weight;      // the same over Z; the row's weight
  Soft v;

  // what does not need the row's sums: loads that are on their way with the row
  __device__ __forceinline__ Answer(const Distill& a_, const T* s_, int row_) : a(a_), s(s_), row(row_) {
    label = label_of(a.labels, row);
    has = label >= 0 && label < a.classes;
    weight = a.row_weight ? a.row_weight[row] : 1.f;
    mine = logit_of(s, label, a.classes);
  }
  __device__ __forceinline__ void finish(const Soft& v_, bool some, bool list_broken) {
    v = v_;
    const bool hard = a.hard_weight != 0.f;
    empty = v.m == -INF;
    bad = v.m == INF || v.restt != v.restt || (hard && v.rest1 != v.rest1) || list_broken || (label != -1 && !has);
    const double hw = (double)a.hard_weight, w = (double)weight;
    logl = has && hard ? (double)mine - (double)v.m - log1p((double)v.rest1) : 0.0;
    ws = some ? w * (1.0 - hw) * a.temperature : 0.0;
    wh = has ? w * hw : 0.0;
    fs = bad ? quiet_nan() : empty ? 0.f : (float)(ws / (1.0 + v.restt));
    fh = bad ? quiet_nan() : hard && !empty ? (float)(wh / (1.0 + v.rest1)) : 0.f;
  }
  __device__ __forceinline__ void write_loss(const List& l) const {
    const double hw = (double)a.hard_weight;
    double loss = 0.0;
    if (l.some && hw != 1.0) loss += (1.0 - hw) * a.temperature * a.temperature * l.soft;
    if (has && hw != 0.0) loss -= hw * logl;
    a.loss[row] = bad ? quiet_nan() : empty ? 0.f : (float)loss;
  }
  // The gradient at the listed classes and the label, where q - p and p - 1 may cancel: by one wave, before the others are written
  struct Entries { int index, label; float at_index, at_label; };      // -1: none
  __device__ __forceinline__ Entries entries(const List& l, int lane) const {
    Entries r{-1, -1, 0.f, 0.f};
    if (bad || empty) return r;
    const bool listed = __any(l.on && l.index == label);
    if (l.on) {
      const double hard = wh == 0.0 ? 0.0 : l.index == label ? expm1(logl) : (double)expf(l.mine - v.m) / (1.0 + (double)v.rest1);
      r.index = l.index;
      r.at_index = (float)((ws != 0.0 ? ws * l.diff : 0.0) + wh * hard);       // without weight the list has no say, as in the loss
    }
    if (has && !listed && lane == 0) {
      const double q = (double)expf((mine - v.m) * (1.f / a.temperature)) / (1.0 + (double)v.restt);
      r.label = label;
      r.at_label = (float)(ws * q + wh * expm1(logl));
    }
    return r;
  }
  static __device__ __forceinline__ void write(const Entries& r, T* d, long c0, long c1) {       // those among classes [c0, c1)
    if (r.index >= c0 && r.index < c1) from_f32(d + r.index, r.at_index);
    if (r.label >= c0 && r.label < c1) from_f32(d + r.label, r.at_label);
  }
};

// gradient of the `len` held elements to d
template <int HARD, class T, int NT, int J, class G>
__device__ __forceinline__ void write_gradient(Held<T, NT, J>& h, T* d, float m, float it, float fs, float fh, G after) {
  const Exponents x(m, it);
  h.renew();
  h.store(d, [&](float s, int, int) {
    const float e = x.soft(s);
    float y = fs * e;
    if (HARD) y = fmaf(fh, x.hard<HARD>(s, e), y);
    return y;
  }, after);
}

// A row that a group holds whole
template <int HARD, class T, int NT, int J>
__device__ __forceinline__ void distill_row(const Distill& a, const Group<NT>& g, Held<T, NT, J>& h, Answer<T>& ans, List& l, int row) {
  const float it = 1.f / a.temperature;
  const Soft v = soft_of<HARD>(g, h, it);
  // every wave needs to know whether the list has entries and bad ones; the first one has read it
  bool some = l.some, broken = l.broken;
  if (NT > 64) {
    if (g.tid == 0) g.sh.n = (int)l.some | (int)l.broken << 1;
    __syncthreads();
    some = g.sh.n & 1;
    broken = g.sh.n & 2;
  }
  ans.finish(v, some, broken);
  if (g.tid < 64) finish_list(a, l, v);
  if (g.tid == 0) ans.write_loss(l);
  if (!a.dlogits) return;
  T* d = (T*)a.dlogits + row * a.ldd;
  typename Answer<T>::Entries entries{-1, -1, 0.f, 0.f};
  if (g.tid < 64) entries = ans.entries(l, g.tid);
  write_gradient<HARD>(h, d, v.m, it, ans.fs, ans.fh, [](int) {});
  if (NT > 64) __syncthreads(); else __builtin_amdgcn_s_waitcnt(0x0f70);   // the stores above are done before the entries replace some of them
  if (g.tid < 64) Answer<T>::write(entries, d, 0, a.classes);
}
// Rows of a wave, or of 256 threads where they are few: all in one launch (256 rows of 1000 fp32 logits, lists of 32: 8.1 us)
template <int HARD, class T, int NT, int J, int PER>
__global__ __launch_bounds__(NT * PER) void k_distill(Distill a) {
  __shared__ GroupSpace<NT> space[PER];
  const int which = PER == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / NT);
  const Group<NT> g{space[which], (int)threadIdx.x % NT};
  const int row = blockIdx.x * PER + which;
  if (row >= a.rows) return;
  const T* s = (const T*)a.logits + row * a.ld;
  Held<T, NT, J> h;
  h.load(s, a.classes, g.tid);
  Answer<T> ans(a, s, row);
  List l{};
  if (g.tid < 64) l = read_list(a, s, row, g.tid);
  distill_row<HARD>(a, g, h, ans, l, row);
}
// Long rows: loss and entries are left to k_distill_entries, which finds the rows' sums in `records`: their double arithmetic next to a row in
// registers costs more registers than there are.  What there is to know before the sums, and the gradient's factors from them:
struct Before {
  int label; bool has; float weight;
  __device__ __forceinline__ Before(const Distill& a, int row, int tid, int& flags) {      // flags: in LDS, to be read behind a barrier
    label = label_of(a.labels, row);
    has = label >= 0 && label < a.classes;
    weight = a.row_weight ? a.row_weight[row] : 1.f;
    if (tid < 64) {
      const int index = tid < a.top ? a.top_index[(long)row * a.top + tid] : -1;
      const bool on = index >= 0 && a.top_logit[(long)row * a.top + tid] != -INF;
      const bool some = __any(on), broken = __any(on && index >= a.classes);
      if (tid == 0) flags = (int)some | (int)broken << 1;
    }
  }
};
struct Factors {
  float soft, hard;
  template <int HARD>
  static __device__ __forceinline__ Factors of(const Distill& a, const Before& b, const Soft& v, int flags) {
    const bool some = (flags & 1) && v.m != -INF, hot = b.has && v.m != -INF;      // nothing for a row that is masked whole
    const bool bad = v.m == INF || v.restt != v.restt || (HARD && v.rest1 != v.rest1) || (flags & 2) || (b.label != -1 && !b.has);
    return Factors{bad ? quiet_nan() : some ? b.weight * (1.f - a.hard_weight) * a.temperature / (1.f + v.restt) : 0.f,
                   bad ? quiet_nan() : HARD && hot ? b.weight * a.hard_weight / (1.f + v.rest1) : 0.f};
  }
};
// Two rows of 512 threads on a CU, as in k_logprob_forward: 2048 rows of 50257 bf16 logits in 111 us (145 by k_distill_rows).
template <int HARD, class T, int NT, int J>
__global__ __launch_bounds__(NT, 4) void k_distill_held(Distill a, Soft* records) {
  __shared__ GroupSpace<NT> space;
  const Group<NT> g{space, (int)threadIdx.x};
  const float it = 1.f / a.temperature;
  const int row = blockIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  Held<T, NT, J> h;
  h.load(s, a.classes, g.tid);
  const Before b(a, row, g.tid, space.n);
  const Soft v = soft_of<HARD>(g, h, it);
  const Factors f = Factors::of<HARD>(a, b, v, space.n);
  if (g.tid == 0) records[row] = v;
  if (a.dlogits) write_gradient<HARD>(h, (T*)a.dlogits + row * a.ldd, v.m, it, f.soft, f.hard, [](int) {});
}
// Rows of more than 8192 units, like k_logprob_rows; the units that LDS has no room for follow into their registers as the gradient leaves them.
// 2048 rows of 131072 bf16 logits: 255 us, 4.2 TB/s read and written; instructions, 18 per element and two exponentials, takes
// 60 % of that by itself.
template <int HARD, class T, int J, int AHEAD>
__global__ __launch_bounds__(1024) void k_distill_rows(Distill a, Soft* records) {
  typedef Held<T, 1024, J> H;
  __shared__ GroupSpace<1024> space;
  extern __shared__ __align__(16) uint4 room[];
  const Group<1024> g{space, (int)threadIdx.x};
  const float it = 1.f / a.temperature;
  int row = blockIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  H h;
  H::template fetch<AHEAD>(s, a.classes, g.tid, room);
#pragma unroll
  for (int j = AHEAD; j < J; ++j) h.load_unit(s, a.classes, g.tid, j, nullptr);
  __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): the thread's units are in LDS
  for (; row < a.rows; row += gridDim.x) {
    s = (const T*)a.logits + row * a.ld;
    const bool more = row + (int)gridDim.x < a.rows;
    const T* next = s + gridDim.x * a.ld;
    h.template load<AHEAD, AHEAD>(s, a.classes, g.tid, room);
    const Before b(a, row, g.tid, space.n);
    __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0): they are read
    if (more) H::template fetch<AHEAD>(next, a.classes, g.tid, room);
    const Soft v = soft_of<HARD>(g, h, it);
    const Factors f = Factors::of<HARD>(a, b, v, space.n);
    if (g.tid == 0) records[row] = v;
    __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0): the next row's units are in LDS; before the stores, whose end nobody awaits
    auto after = [&](int j) { if (j >= AHEAD && more) h.load_unit(next, a.classes, g.tid, j, nullptr); };
    if (a.dlogits) write_gradient<HARD>(h, (T*)a.dlogits + row * a.ldd, v.m, it, f.soft, f.hard, after);
    if (!a.dlogits || !h.used(J - 1)) {                // units that this row does not have, but the next may
#pragma unroll
      for (int j = AHEAD; j < J; ++j)
        if (!a.dlogits || !h.used(j)) after(j);
    }
    __syncthreads();                                   // space.n is read
  }
}
// Loss, and the gradient at the listed classes and the label, a wave per row: 17 us for 2048 rows and lists of 64, the trips to memory one after
// the other and the logarithms in double.
template <class T>
__global__ __launch_bounds__(256) void k_distill_entries(Distill a, const Soft* __restrict__ records) {
  const int row = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64)), lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  const T* s = (const T*)a.logits + row * a.ld;
  Answer<T> ans(a, s, row);
  List l = read_list(a, s, row, lane);
  const Soft v = records[row];
  finish_list(a, l, v);
  ans.finish(v, l.some, l.broken);
  if (lane == 0) ans.write_loss(l);
  if (a.dlogits) Answer<T>::write(ans.entries(l, lane), (T*)a.dlogits + row * a.ldd, 0, a.classes);
}

// a row divided among work-groups: first their sums ...
template <int HARD, class T, int J>
__global__ __launch_bounds__(256) void k_distill_part(Distill a, int parts, long per_part, Soft* records) {
  typedef Held<T, 256, J> H;
  __shared__ GroupSpace<256> space;
  const Group<256> g{space, (int)threadIdx.x};
  const int row = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x - (unsigned)row * parts);
  const T* s = (const T*)a.logits + row * a.ld;
  const float it = 1.f / a.temperature;
  const long c_begin = part * per_part, c_end = c_begin + per_part < a.classes ? c_begin + per_part : a.classes;
  Soft v{-INF, 0.f, 0.f};
  long step;
  for (long c0 = c_begin; c0 < c_end; c0 += step) {
    const long room = H::CAPACITY - (long)(((uintptr_t)(s + c0) & 15) / sizeof(T));
    step = c_end - c0 < room ? c_end - c0 : room;
    H h;
    h.load(s + c0, (int)step, g.tid);
    const Soft w = soft_of<HARD>(g, h, it);
    if (c0 == c_begin) v = w; else merge(v, w, it);
  }
  if (g.tid == 0) records[blockIdx.x] = v;
}
// ... then loss and gradient
template <int HARD, class T, int J>
__global__ __launch_bounds__(256) void k_distill_join(Distill a, int parts, long per_part, const Soft* __restrict__ records) {
  typedef Held<T, 256, J> H;
  __shared__ GroupSpace<256> space;
  const Group<256> g{space, (int)threadIdx.x};
  const int row = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x - (unsigned)row * parts), tid = threadIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  const float it = 1.f / a.temperature;
  Soft p{-INF, 0.f, 0.f};
  if (tid < parts) p = records[(long)row * parts + tid];
  Soft v;
  float sum[2] = {p.rest1, p.restt};
  if (!holds_maximum(g, p.m, v.m) && p.m != -INF) {
    sum[0] = (1.f + p.rest1) * expf(p.m - v.m);
    sum[1] = (1.f + p.restt) * expf((p.m - v.m) * it);       // at temperature T the distance of the maxima counts 1 / T of itself
  }
  g.reduce(sum, [](float a, float b) { return a + b; });
  v.rest1 = sum[0];
  v.restt = sum[1];
  List l = read_list(a, s, row, tid & 63);
  finish_list(a, l, v);
  Answer<T> ans(a, s, row);
  ans.finish(v, l.some, l.broken);
  if (part == 0 && tid == 0) ans.write_loss(l);
  if (!a.dlogits) return;
  T* d = (T*)a.dlogits + row * a.ldd;
  const long c_begin = part * per_part, c_end = c_begin + per_part < a.classes ? c_begin + per_part : a.classes;
  long step;
  for (long c0 = c_begin; c0 < c_end; c0 += step) {
    const long room = H::CAPACITY - (long)(((uintptr_t)(s + c0) & 15) / sizeof(T));
    step = c_end - c0 < room ? c_end - c0 : room;
    H h;
    h.load(s + c0, (int)step, tid);
    write_gradient<HARD>(h, d + c0, v.m, it, ans.fs, ans.fh, [](int) {});
  }
  __syncthreads();
  if (tid < 64) Answer<T>::write(ans.entries(l, tid), d, c_begin, c_end);
}

// ---- how rows are cut ------------------------------------------------------------------------------------------------
constexpr int CUS = 256, MAX_PARTS = 256, PART_J = 4;
// up to so many short rows get a work-group each, on all CUs, instead of one for four (rows of 1000 fp32 logits, lists of 5: 64 to 512 rows 6.3 to
// 6.8 us instead of 7.0 to 7.2, 8192 rows 17.0 instead of 15.6)
constexpr int SPREAD_ROWS = 4 * CUS;

struct RowCut {
  int parts;
  long per_part;                 // classes
  int units;                     // 16-byte units of a row, with the one that a row across a boundary has more
};
// A row of 2048 units (32 KiB) and more is divided if there are at most 64 of them, and if no work-group holds it (a part of it may then need
// several chunks).  Lists of 5 and distillation, bf16, us: 64 rows of 131072 classes 19 and 21 divided, 23 and 32 undivided; 16 of 50000 12 and
// 12 against 16 and 17; but 128 of 50000 19 and 19 against 16 and 19.5, 128 of 131072 32 and 33 against 25 and 35.  16 to 64 rows of 16376,
// less than 2048 units: 12.5 and 11.5 against 10 and 10.7.
// aligned: every row starts on 16 bytes (a workspace is sized for rows that do not, which never have fewer parts).
RowCut row_cut(int dt, int rows, int classes, bool aligned) {
  const int E = dt == DT_BF16 ? 8 : 4;
  RowCut c;
  c.units = (classes + E - 1) / E + (aligned ? 0 : 1);
  const bool too_long = c.units > 1024 * 16;
  c.parts = 1;
  if (too_long || (rows <= CUS / 4 && c.units >= 2048)) {
    long p = (2 * CUS + rows - 1) / rows;
    const long most = c.units / 512;
    if (p > most) p = most;
    if (p > MAX_PARTS) p = MAX_PARTS;
    if (p < 2) p = 2;
    c.parts = (int)p;
  }
  c.per_part = ((classes + c.parts - 1) / c.parts + 63) / 64 * 64;
  c.parts = (int)((classes + c.per_part - 1) / c.per_part);     // none without classes
  return c;
}

// Whether an undivided row of a distillation leaves loss and entries to a second launch, for which the workspace holds the rows' sums.  A wave
// that has a row to itself never does; 256 threads do where there are rows enough for the second launch not to count (4096 rows of 8200: 48
// instead of 59 us; 300 of 5000: 16.8 instead of 12.1).
bool by_records(int rows, int units) { return units > 256 * 8 || (units > 64 * 4 && rows > SPREAD_ROWS); }

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
bool aligned16(const void* p, long ld, size_t elem) { return ((uintptr_t)p & 15) == 0 && ((size_t)ld * elem & 15) == 0; }

// one work-group of 1024 threads per CU with `ahead` units per thread in LDS
template <class K, class A, class... MORE>
hipError_t launch_rows(K kernel, int ahead, hipStream_t s, const A& a, MORE... more) {
  const int lds = 1024 * 16 * ahead;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)(a.rows < CUS ? a.rows : CUS), 1024, lds, s>>>(a, more...);
  return hipGetLastError();
}

template <class T>
hipError_t logprob_forward(int dt, const LogprobForward& a, void* workspace, hipStream_t s) {
  const RowCut c = row_cut(dt, a.rows, a.classes, aligned16(a.logits, a.ld, sizeof(T)));
  if (c.parts > 1) {
    const unsigned n = (unsigned)((long)a.rows * c.parts);
    PartRecord* records = (PartRecord*)workspace;
    Key* lists = (Key*)((char*)workspace + align256((size_t)n * sizeof(PartRecord)));
    k_logprob_part<T, PART_J><<<n, 256, 0, s>>>(a, c.parts, c.per_part, records, lists);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_logprob_join<T><<<(unsigned)a.rows, 256, 0, s>>>(a, c.parts, records, lists);
  } else if (c.units <= 64 * 4) {
    if (a.rows <= SPREAD_ROWS) k_logprob_forward<T, 64, 4, 1><<<(unsigned)a.rows, 64, 0, s>>>(a);
    else k_logprob_forward<T, 64, 4, 4><<<(unsigned)((a.rows + 3) / 4), 256, 0, s>>>(a);
  } else if (c.units <= 256 * 8) k_logprob_forward<T, 256, 8, 1><<<(unsigned)a.rows, 256, 0, s>>>(a);
  else if (c.units <= 512 * 8) k_logprob_forward<T, 512, 8, 1><<<(unsigned)a.rows, 512, 0, s>>>(a);
  else if (c.units <= 512 * 16) k_logprob_forward<T, 512, 16, 1><<<(unsigned)a.rows, 512, 0, s>>>(a);
  else return launch_rows(k_logprob_rows<T, 16, 8>, 8, s, a);
  return hipGetLastError();
}

template <class T>
hipError_t logprob_backward(const LogprobBackward& a, hipStream_t s) {
  const unsigned per_row = (unsigned)logprob_backward_pieces(sizeof(T), a.classes);
  k_logprob_backward<T><<<(unsigned)a.rows * per_row, 256, 0, s>>>(a, per_row);
  return hipGetLastError();
}

template <int HARD, class T>
hipError_t distill_as(int dt, const Distill& a, void* workspace, hipStream_t s) {
  const RowCut c = row_cut(dt, a.rows, a.classes, aligned16(a.logits, a.ld, sizeof(T)));
  if (c.parts > 1) {
    const unsigned n = (unsigned)((long)a.rows * c.parts);
    Soft* records = (Soft*)workspace;
    constexpr int ANY = HARD ? HARD_EXP : HARD_NONE;
    k_distill_part<ANY, T, PART_J><<<n, 256, 0, s>>>(a, c.parts, c.per_part, records);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_distill_join<ANY, T, PART_J><<<n, 256, 0, s>>>(a, c.parts, c.per_part, records);
  } else if (c.units <= 64 * 4) {
    constexpr int ANY = HARD ? HARD_EXP : HARD_NONE;
    if (a.rows <= SPREAD_ROWS) k_distill<ANY, T, 64, 4, 1><<<(unsigned)a.rows, 64, 0, s>>>(a);
    else k_distill<ANY, T, 64, 4, 4><<<(unsigned)((a.rows + 3) / 4), 256, 0, s>>>(a);
  } else if (!by_records(a.rows, c.units)) k_distill<HARD ? HARD_EXP : HARD_NONE, T, 256, 8, 1><<<(unsigned)a.rows, 256, 0, s>>>(a);
  else {
    Soft* records = (Soft*)workspace;
    hipError_t e = hipSuccess;
    if (c.units <= 256 * 8) k_distill_held<HARD, T, 256, 8><<<(unsigned)a.rows, 256, 0, s>>>(a, records);
    else if (c.units <= 512 * 8) k_distill_held<HARD, T, 512, 8><<<(unsigned)a.rows, 512, 0, s>>>(a, records);
    else if (c.units <= 512 * 16) k_distill_held<HARD, T, 512, 16><<<(unsigned)a.rows, 512, 0, s>>>(a, records);
    else e = launch_rows(k_distill_rows<HARD, T, 16, 8>, 8, s, a, records);
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_distill_entries<T><<<(unsigned)((a.rows + 3) / 4), 256, 0, s>>>(a, records);
  }
  return hipGetLastError();
}

template <class T>
hipError_t distill(int dt, const Distill& a, void* workspace, hipStream_t s) {
  if (a.hard_weight == 0.f) return distill_as<HARD_NONE, T>(dt, a, workspace, s);
  if (a.temperature == 1.f) return distill_as<HARD_ONE, T>(dt, a, workspace, s);
  if (a.temperature == 2.f) return distill_as<HARD_TWO, T>(dt, a, workspace, s);
  if (a.temperature == 4.f) return distill_as<HARD_FOUR, T>(dt, a, workspace, s);
  return distill_as<HARD_EXP, T>(dt, a, workspace, s);
}

}  // namespace

size_t logits_workspace_bytes(int dt, int rows, int classes, int top) {
  const RowCut c = row_cut(dt, rows, classes, false);
  const size_t n = (size_t)rows * c.parts;
  if (c.parts > 1) return align256(n * sizeof(PartRecord)) + align256(n * top * sizeof(Key));
  return by_records(rows, c.units) ? align256(n * sizeof(Soft)) : 0;
}

hipError_t launch_logprob_forward(int dt, const LogprobForward& a, void* workspace, hipStream_t stream) {
  return dt == DT_BF16 ? logprob_forward<bf16_t>(dt, a, workspace, stream) : logprob_forward<float>(dt, a, workspace, stream);
}
hipError_t launch_logprob_backward(int dt, const LogprobBackward& a, hipStream_t stream) {
  return dt == DT_BF16 ? logprob_backward<bf16_t>(a, stream) : logprob_backward<float>(a, stream);
}
hipError_t launch_distill(int dt, const Distill& a, void* workspace, hipStream_t stream) {
  return dt == DT_BF16 ? distill<bf16_t>(dt, a, workspace, stream) : distill<float>(dt, a, workspace, stream);
}

}  // namespace hpf
