// Matrix product with bias, activation and residual in its epilogue, and its gradients:
//     z = x W + bias,  y = act(z) + residual,  slope = act'(z)
//     dz = dy * slope,  dx = dz W^T,  dw = x^T dz,  db = column sums of dz
// The three products are one contraction C[m][n] = sum_k A(m, k) B(n, k) with other operands.  bf16: v_mfma_f32_16x16x32_bf16,
// sums in fp32, one rounding of y; the slope is taken from the unrounded z and rounded once, so that dz is the rounded product
// of two stored numbers and does not depend on the order of any sum.  fp32 (check mode): v_mfma_f64_16x16x4_f64 on the exact
// operands, epilogue in double.
#include "hpf_answer.h"
#include "hpf_device.h"

namespace hpf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef double doublex4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float f_exp(float v) { return expf(v); }
__device__ __forceinline__ double f_exp(double v) { return exp(v); }
__device__ __forceinline__ float f_erfc(float v) { return erfcf(v); }
__device__ __forceinline__ double f_erfc(double v) { return erfc(v); }

// act(z) and act'(z)
template <class A>
__device__ __forceinline__ void activate(int act, A z, A& y, A& slope) {
  if (act == ACT_RELU) {
    y = z > A(0) ? z : (z == z ? A(0) : z);
    slope = z > A(0) ? A(1) : (z == z ? A(0) : z);
  } else if (act == ACT_GELU) {
    const A below = A(0.5) * f_erfc(z * A(-0.70710678118654752));           // Phi(z)
    const A density = A(0.39894228040143268) * f_exp(A(-0.5) * z * z);
    y = z * below;
    slope = below + z * density;
  } else if (act == ACT_SILU) {
    const A q = A(1) / (A(1) + f_exp(-z));
    y = z * q;
    slope = q * (A(1) + z * (A(1) - q));
  } else {
    y = z;
    slope = A(1);
  }
}

// An operand of the contraction: element (row, k) at p[row * rs + k * ks]
template <class T>
struct Operand { const T* p; long rs, ks; };
template <class T>
struct Epilogue {
  const float* bias;
  const T* residual; long ldr;
  T* y; long ldy;
  T* slope;
  float* sum; int accumulate;     // instead of y: C in fp32, [M][N]
  int act;
};

template <class T> struct Mma;
template <> struct Mma<bf16_t> {
  typedef float Acc;
  typedef floatx4 Acc4;
  static constexpr int K = 32;
  typedef bf16x8 Frag;
  static __device__ __forceinline__ Frag frag(const bf16_t* row, int lane) { return *reinterpret_cast<const bf16x8*>(row + (lane >> 4) * 8); }
  static __device__ __forceinline__ Acc4 mma(Frag a, Frag b, Acc4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ int row(int lane, int r) { return (lane >> 4) * 4 + r; }   // of the first operand; column lane & 15
};
template <> struct Mma<float> {
  typedef double Acc;
  typedef doublex4 Acc4;
  static constexpr int K = 4;
  typedef double Frag;
  static __device__ __forceinline__ Frag frag(const float* row, int lane) { return (double)row[lane >> 4]; }
  static __device__ __forceinline__ Acc4 mma(Frag a, Frag b, Acc4 c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ int row(int lane, int r) { return (lane >> 4) + 4 * r; }
};

// C tile of 64 x 64 by four waves, 32 x 32 each; 32 steps of the contraction staged in LDS at a time.  Any sizes and strides.
template <class T>
__global__ __launch_bounds__(256) void k_linear_tile(Operand<T> A, Operand<T> B, Epilogue<T> e, int M, int N, int K) {
  typedef Mma<T> X;
  constexpr int KS = 32, LS = KS + 8;
  __shared__ __align__(16) T sA[64 * LS], sB[64 * LS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
  typename X::Acc4 acc[2][2] = {};
  auto stage = [&](const Operand<T>& o, T* s, int r0, int rows, int k0) {
    for (int i = tid; i < 64 * KS; i += 256) {
      const int r = o.ks == 1 ? i / KS : i % 64, k = o.ks == 1 ? i % KS : i / 64;
      s[r * LS + k] = r0 + r < rows && k0 + k < K ? o.p[(long)(r0 + r) * o.rs + (long)(k0 + k) * o.ks] : T(0);
    }
  };
  for (int k0 = 0; k0 < K; k0 += KS) {
    __syncthreads();
    stage(A, sA, m0, M, k0);
    stage(B, sB, n0, N, k0);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KS; k += X::K) {
      typename X::Frag a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = X::frag(&sA[(wm + i * 16 + (lane & 15)) * LS + k], lane);
        b[i] = X::frag(&sB[(wn + i * 16 + (lane & 15)) * LS + k], lane);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = X::mma(b[j], a[i], acc[i][j]);   // rows: n, columns: m
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = m0 + wm + i * 16 + (lane & 15), n = n0 + wn + j * 16 + X::row(lane, r);
        if (m >= M || n >= N) continue;
        typename X::Acc z = acc[i][j][r], y, slope;
        if (e.sum) {
          float* o = e.sum + (long)m * N + n;
          *o = (float)(e.accumulate ? z + *o : z);
          continue;
        }
        if (e.bias) z += e.bias[n];
        activate(e.act, z, y, slope);
        if (e.residual) y += to_f32(e.residual[m * e.ldr + n]);
        from_f32(e.y + m * e.ldy + n, (float)y);
        if (e.slope) from_f32(e.slope + (long)m * N + n, (float)slope);
      }
}

// packed copies of w: blocks of 64 x 64 through LDS
__global__ __launch_bounds__(256) void k_linear_pack(const float* __restrict__ w, bf16_t* __restrict__ packed, int K, int N, int Kp, int Np) {
  __shared__ float tile[64][65];
  const int k0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  bf16_t* wf = packed;
  bf16_t* wd = packed + (size_t)N * Kp;
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int k = k0 + i / 64, n = n0 + i % 64;
    const float v = k < K && n < N ? w[(size_t)k * N + n] : 0.f;
    tile[i / 64][i % 64] = v;
    if (k < K) wd[(size_t)k * Np + n] = f32_to_bf16(v);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int n = n0 + i / 64, k = k0 + i % 64;
    if (n < N) wf[(size_t)n * Kp + k] = f32_to_bf16(tile[i % 64][i / 64]);
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_linear_dz(const T* __restrict__ dy, long lddy, const T* __restrict__ slope, T* __restrict__ dz, int M, int N) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)M * N; i += (size_t)gridDim.x * 256) {
    const size_t m = i / N, n = i - m * N;
    from_f32(dz + i, to_f32(dy[m * lddy + n]) * to_f32(slope[i]));
  }
}

// db: 64 columns per work-group
template <class T>
__global__ __launch_bounds__(256) void k_linear_db(const T* __restrict__ dz, long ld, float* __restrict__ db, int accumulate, int M, int N) {
  __shared__ double part[4][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
  double s = 0.0;
  if (n < N)
    for (int m = g; m < M; m += 4) s += to_f32(dz[m * ld + n]);
  part[g][c] = s;
  __syncthreads();
  if (g == 0 && n < N) {
    s = part[0][c] + part[1][c] + part[2][c] + part[3][c];
    db[n] = (float)(accumulate ? s + db[n] : s);
  }
}

unsigned blocks64(int v) { return (unsigned)((v + 63) / 64); }

template <class T>
hipError_t tile(const Operand<T>& A, const Operand<T>& B, const Epilogue<T>& e, int M, int N, int K, hipStream_t s) {
  k_linear_tile<T><<<dim3(blocks64(N), blocks64(M)), 256, 0, s>>>(A, B, e, M, N, K);
  return hipGetLastError();
}

// The weights as operands: rows n for the forward product, rows k for dx
Operand<bf16_t> forward_operand(const void* p, int K, int, bf16_t) { return {(const bf16_t*)p, round_up64(K), 1}; }
Operand<float> forward_operand(const void* p, int, int N, float) { return {(const float*)p, 1, N}; }
Operand<bf16_t> dx_operand(const void* p, int K, int N, bf16_t) { return {(const bf16_t*)p + (size_t)N * round_up64(K), round_up64(N), 1}; }
Operand<float> dx_operand(const void* p, int, int N, float) { return {(const float*)p, N, 1}; }

template <class T>
hipError_t forward(const LinearForward& a, hipStream_t s) {
  Epilogue<T> e{a.bias, (const T*)a.residual, a.ldr, (T*)a.y, a.ldy, (T*)a.slope, nullptr, 0, a.act};
  return tile<T>({(const T*)a.x, a.ldx, 1}, forward_operand(a.weights, a.K, a.N, T{}), e, a.M, a.N, a.K, s);
}

template <class T>
hipError_t backward(const LinearBackward& a, void* workspace, hipStream_t s) {
  const T* dz = (const T*)a.dy;
  long ld = a.lddy;
  hipError_t err = hipSuccess;
  if (a.slope) {
    const size_t blocks = ((size_t)a.M * a.N + 2047) / 2048;
    k_linear_dz<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(dz, ld, (const T*)a.slope, (T*)workspace, a.M, a.N);
    dz = (const T*)workspace;
    ld = a.N;
    err = hipGetLastError();
  }
  if (err == hipSuccess && a.db) {
    k_linear_db<T><<<blocks64(a.N), 256, 0, s>>>(dz, ld, a.db, a.accumulate, a.M, a.N);
    err = hipGetLastError();
  }
  if (err == hipSuccess && a.dx) {
    Epilogue<T> e{};
    e.y = (T*)a.dx; e.ldy = a.lddx;
    err = tile<T>({dz, ld, 1}, dx_operand(a.weights, a.K, a.N, T{}), e, a.M, a.K, a.N, s);
  }
  if (err == hipSuccess && a.dw) {
    Epilogue<T> e{};
    e.sum = a.dw; e.accumulate = a.accumulate;
    err = tile<T>({(const T*)a.x, 1, a.ldx}, {dz, 1, ld}, e, a.K, a.N, a.M, s);
  }
  return err;
}

}  // namespace

hipError_t launch_linear_pack(const float* w, bf16_t* packed, int K, int N, hipStream_t stream) {
  k_linear_pack<<<dim3(blocks64(N), blocks64(K)), 256, 0, stream>>>(w, packed, K, N, round_up64(K), round_up64(N));
  return hipGetLastError();
}

size_t linear_workspace_bytes(int dt, int M, int, int N) { return (size_t)M * N * (dt == DT_BF16 ? 2 : 4); }

hipError_t launch_linear_forward(int dt, const LinearForward& a, void*, hipStream_t stream) {
  return dt == DT_BF16 ? forward<bf16_t>(a, stream) : forward<float>(a, stream);
}
hipError_t launch_linear_backward(int dt, const LinearBackward& a, void* workspace, hipStream_t stream) {
  return dt == DT_BF16 ? backward<bf16_t>(a, workspace, stream) : backward<float>(a, workspace, stream);
}

}  // namespace hpf
