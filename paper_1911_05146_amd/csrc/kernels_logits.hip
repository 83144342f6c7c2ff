// Row operators on logits: log probability of a label with entropy, rank and the most likely classes, its gradient, and the
// distillation loss with its gradient.  A row's softmax is held as {m, rest, dot}: m its maximum, rest the sum of exp(s - m) over
// all classes but the one that holds the maximum, dot the sum of exp(s - m) (s - m).  With Z = 1 + rest, log Z = log1p(rest), so
// that log p and 1 - p keep their digits where one class is all but certain, and the entropy log Z - dot / Z adds two terms that
// are never negative.
#include "hpf_answer.h"
#include "hpf_device.h"

namespace hpf {
namespace {

constexpr float INF = __builtin_huge_valf();

struct RowSum {
  float m, rest, dot;
  static __device__ __forceinline__ RowSum none() { return RowSum{-INF, 0.f, 0.f}; }
  __device__ __forceinline__ void add(float s) {
    if (s == -INF) return;                     // a masked class
    if (s > m) {
      merge_into(RowSum{s, 0.f, 0.f});
    } else {
      const float e = expf(s - m);
      rest += e;
      dot += e > 0.f || e != e ? e * (s - m) : 0.f;
    }
  }
  // this, but seen from the larger maximum o.m
  __device__ __forceinline__ void merge_into(const RowSum& o) {
    if (m == -INF) { const float r = rest; *this = o; rest += r; return; }   // r: 0, or NaN if a NaN came before the first number
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
  __device__ __forceinline__ float log_rest() const { return log1pf(rest); }                          // log Z
};

template <class V>
__device__ __forceinline__ V from_lane(const V& v, int lane) {
  static_assert(sizeof(V) % 4 == 0, "whole registers");
  V r;
  const int* p = reinterpret_cast<const int*>(&v);
  int* q = reinterpret_cast<int*>(&r);
#pragma unroll
  for (unsigned i = 0; i < sizeof(V) / 4; ++i) q[i] = __shfl(p[i], lane);
  return r;
}

// over the 256 threads; every thread gets the result
__device__ __forceinline__ RowSum block_sum(RowSum v, RowSum* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 32; o > 0; o >>= 1) {
    const RowSum w = from_lane(v, lane ^ o);
    if (lane & o) { RowSum t = w; t.merge(v); v = t; } else v.merge(w);   // one order for both
  }
  __syncthreads();
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < 4; ++i) v.merge(sh[i]);
  return v;
}

// order of the list: larger value first, then lower index; 0 is behind every class
__device__ __forceinline__ unsigned long long key_of(float s, int c) {
  const unsigned u = __float_as_uint(s + 0.f);   // -0 counts as 0
  return (unsigned long long)(u ^ (u >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - (unsigned)c);
}
__device__ __forceinline__ unsigned long long block_max(unsigned long long v, unsigned long long* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned long long w = from_lane(v, lane ^ o);
    v = w > v ? w : v;
  }
  __syncthreads();
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < 4; ++i) v = sh[i] > v ? sh[i] : v;
  return v;
}

__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }

template <class T>
__global__ __launch_bounds__(256) void k_logprob_forward(LogprobForward a) {
  __shared__ RowSum sh[4];
  __shared__ unsigned long long shk[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  const int label = a.labels ? a.labels[row] : -1;
  const bool has = label >= 0 && label < a.classes;
  const float mine = has ? to_f32(s[label]) : 0.f;
  RowSum v = RowSum::none();
  int before = 0;
  for (int c = tid; c < a.classes; c += 256) {
    const float t = to_f32(s[c]);
    v.add(t);
    before += t > mine || (t == mine && c < label);
  }
  v = block_sum(v, sh);
  const bool broken = v.broken();
  __shared__ int total;
  if (tid == 0) total = 0;
  __syncthreads();
  if (before) atomicAdd(&total, before);
  __syncthreads();
  if (tid == 0) {
    const float lz = v.empty() ? -INF : v.log_rest();
    if (a.logprob)
      a.logprob[row] = label == -1 ? 0.f : (broken || !has) ? quiet_nan() : v.empty() ? -INF : (float)((double)mine - v.m - log1p((double)v.rest));
    if (a.rank) a.rank[row] = has && !broken ? total : -1;
    if (a.entropy) a.entropy[row] = broken ? quiet_nan() : v.empty() ? 0.f : lz - v.dot / (1.f + v.rest);
    if (a.stats) {
      a.stats[2 * (long)row] = broken ? quiet_nan() : v.m;
      a.stats[2 * (long)row + 1] = broken ? quiet_nan() : lz;
    }
  }
  unsigned long long last = ~0ull;
  for (int j = 0; j < a.top; ++j) {
    unsigned long long best = 0;
    if (!broken && last)
      for (int c = tid; c < a.classes; c += 256) {
        const float t = to_f32(s[c]);
        const unsigned long long k = t == -INF ? 0 : key_of(t, c);
        if (k < last && k > best) best = k;
      }
    last = block_max(best, shk);
    if (tid == 0) {
      const int c = (int)(0xffffffffu - (unsigned)last);
      const long at = (long)row * a.top + j;
      a.top_index[at] = last ? c : -1;
      a.top_logprob[at] = broken ? quiet_nan() : last ? (float)((double)to_f32(s[c]) - v.m - log1p((double)v.rest)) : -INF;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_logprob_backward(LogprobBackward a) {
  const int row = blockIdx.x;
  const T* s = (const T*)a.logits + row * a.ld;
  T* d = (T*)a.dlogits + row * a.ldd;
  const int label = a.labels ? a.labels[row] : -1;
  const float m = a.stats[2 * (long)row], lz = a.stats[2 * (long)row + 1];
  float g = a.grad_logprob && label != -1 ? a.grad_logprob[row] : 0.f;
  if (label < -1 || label >= a.classes) g = quiet_nan();
  const float gh = a.grad_entropy ? a.grad_entropy[row] : 0.f, h = a.grad_entropy ? a.entropy[row] : 0.f;
  for (int c = threadIdx.x; c < a.classes; c += 256) {
    const float logp = (to_f32(s[c]) - m) - lz;
    const float p = expf(logp);
    float v = c == label ? -g * expm1f(logp) : -g * p;
    if (p > 0.f || p != p) v -= gh * p * (logp + h);
    from_f32(d + c, m == -INF ? 0.f : v);
  }
}

// sums over the wave, in double; every lane gets the result
__device__ __forceinline__ double wave_sum(double v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// What a row's list says, one entry per lane: the loss's soft part and the gradient at the listed classes
struct List {
  bool on, some, broken;     // entry there; any entry there; an index outside the classes
  int index;
  double soft;               // sum_j p_j (log p_j - log q_j)
  double diff;               // q_c - P_c, P_c: probability of the entry's class in the list (all entries of that class)
};
template <class T>
__device__ __forceinline__ List read_list(const Distill& a, const T* s, int row, const RowSum& v, int lane) {
  List l{};
  const long at = (long)row * a.top + lane;
  l.index = lane < a.top ? a.top_index[at] : -1;
  const double t = l.index >= 0 ? (double)a.top_logit[at] : -(double)INF;
  l.on = t != -(double)INF;
  l.broken = __any(l.on && l.index >= a.classes);
  l.some = __any(l.on);
  const bool in = l.on && l.index < a.classes;
  const double it = 1.0 / (double)a.temperature;
  double top = t;
  for (int o = 32; o > 0; o >>= 1) { const double u = __shfl_xor(top, o); top = u > top ? u : top; }
  const double e = l.on ? exp((t - top) * it) : 0.0;
  const double z = wave_sum(e);
  const double p = e / z;
  const double logp = (t - top) * it - log(z);
  const double logq = in ? ((double)to_f32(s[l.index]) - v.m) * it - log1p((double)v.rest) : 0.0;
  l.soft = wave_sum(l.on && p != 0.0 ? p * (logp - logq) : 0.0);
  double same = 0.0;
  for (int j = 0; j < a.top; ++j) {
    const double pj = __shfl(p, j);
    if (__shfl(l.index, j) == l.index) same += pj;
  }
  l.diff = same != 0.0 ? same * expm1(logq - log(same)) : exp(logq);
  return l;
}

template <class T>
__global__ __launch_bounds__(256) void k_distill(Distill a) {
  __shared__ RowSum sh[4];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const T* s = (const T*)a.logits + row * a.ld;
  const float it = 1.f / a.temperature;
  RowSum v1 = RowSum::none(), vt = RowSum::none();   // at temperature 1 and T; the maxima are those of the logits
  for (int c = tid; c < a.classes; c += 256) {
    const float t = to_f32(s[c]);
    v1.add(t);
  }
  v1 = block_sum(v1, sh);
  const bool broken = v1.broken(), empty = v1.empty();
  float z = 0.f;
  int ties = 0;
  for (int c = tid; c < a.classes; c += 256) {
    const float t = to_f32(s[c]);
    if (t == v1.m) ++ties;
    else z += expf((t - v1.m) * it);
  }
  __shared__ float zs[256];
  __shared__ int ts[256];
  zs[tid] = z; ts[tid] = ties;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (tid < o) { zs[tid] += zs[tid + o]; ts[tid] += ts[tid + o]; }
    __syncthreads();
  }
  vt.m = v1.m;
  vt.rest = zs[0] + (float)(ts[0] - 1);
  const int label = a.labels ? a.labels[row] : -1;
  const bool has = label >= 0 && label < a.classes;
  const List l = read_list(a, s, row, vt, lane);
  const bool bad = broken || l.broken || (label != -1 && !has);
  const double logl = has ? (double)to_f32(s[label]) - v1.m - log1p((double)v1.rest) : 0.0;
  const double hw = (double)a.hard_weight, T2 = (double)a.temperature * a.temperature;
  if (tid == 0) {
    double loss = 0.0;
    if (l.some && hw != 1.0) loss += (1.0 - hw) * T2 * l.soft;
    if (has && hw != 0.0) loss -= hw * logl;
    a.loss[row] = bad ? quiet_nan() : empty ? 0.f : (float)loss;
  }
  if (!a.dlogits) return;
  T* d = (T*)a.dlogits + row * a.ldd;
  const double w = a.row_weight ? (double)a.row_weight[row] : 1.0;
  const double ws = l.some ? w * (1.0 - hw) * a.temperature : 0.0, wh = has ? w * hw : 0.0;
  const float fs = bad ? quiet_nan() : (float)(ws / (1.0 + vt.rest)), fh = bad ? quiet_nan() : (float)(wh / (1.0 + v1.rest));
  for (int c = tid; c < a.classes; c += 256) {
    const float t = to_f32(s[c]) - v1.m;
    from_f32(d + c, empty && !bad ? 0.f : fs * expf(t * it) + fh * expf(t));
  }
  if (bad || empty) return;
  __syncthreads();             // the stores above are done before the entries below replace some of them
  if (tid >= 64) return;
  // at the listed classes and the label q - p and p - 1 are taken from the logarithms
  const bool listed = __any(l.on && l.index == label);
  if (l.on) {
    const double t = (double)to_f32(s[l.index]) - v1.m;
    const double hard = l.index == label ? expm1(logl) : exp(t - log1p((double)v1.rest));
    from_f32(d + l.index, (float)(ws * l.diff + wh * hard));
  }
  if (has && !listed && lane == 0) {
    const double q = exp(((double)to_f32(s[label]) - v1.m) * it - log1p((double)vt.rest));
    from_f32(d + label, (float)(ws * q + wh * expm1(logl)));
  }
}

}  // namespace

size_t logits_workspace_bytes(int, int, int, int) { return 0; }

hipError_t launch_logprob_forward(int dt, const LogprobForward& a, void*, hipStream_t stream) {
  if (dt == DT_BF16) k_logprob_forward<bf16_t><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  else k_logprob_forward<float><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  return hipGetLastError();
}
hipError_t launch_logprob_backward(int dt, const LogprobBackward& a, hipStream_t stream) {
  if (dt == DT_BF16) k_logprob_backward<bf16_t><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  else k_logprob_backward<float><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  return hipGetLastError();
}
hipError_t launch_distill(int dt, const Distill& a, void*, hipStream_t stream) {
  if (dt == DT_BF16) k_distill<bf16_t><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  else k_distill<float><<<(unsigned)a.rows, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace hpf
