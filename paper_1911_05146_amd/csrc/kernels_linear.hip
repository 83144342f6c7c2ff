// Matrix product with bias, activation and residual in its epilogue, and its gradients:
//     z = x W + bias,  y = act(z) + residual,  slope = act'(z)
//     dz = dy * slope,  dx = dz W^T,  dw = x^T dz,  db = column sums of dz
// The three products are one contraction C[m][n] = sum_k A(m, k) B(n, k) with other operands.  bf16: v_mfma_f32_16x16x32_bf16,
// sums in fp32, one rounding of y; the slope is taken from the unrounded z and rounded once, so that dz is the rounded product
// of two stored numbers and does not depend on the order of any sum.  fp32 (check mode): v_mfma_f64_16x16x4_f64 on the exact
// operands, epilogue in double.
#include <type_traits>

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
struct Operand { const float* p; long rs, ks; };
struct Epilogue {
  const float* bias;
  const float* residual; long ldr;
  float* y; long ldy;
  float* slope;
  float* sum; int accumulate;     // instead of y: C in fp32, [M][N]
  int act;
};

// fp32 (check mode): C tile of 32 x 32 by eight waves, four of 16 x 16 for each half of the 64 steps that are staged at a time; the halves are
// joined at the end.  v_mfma_f64_16x16x4_f64 takes 64 cycles, so small tiles, which give every CU one, cost nothing: 333 x 1000 x 517 has 187 of
// them (64 x 64 ones with four waves: 54, and 144 us instead of 25, a fifth of the rate of a large product in double).  Any sizes and strides.
__global__ __launch_bounds__(512) void k_linear_tile_f32(Operand A, Operand B, Epilogue e, int M, int N, int K) {
  constexpr int KS = 64, LS = KS + 4;
  __shared__ __align__(16) float sA[2][32 * LS], sB[2][32 * LS];
  __shared__ double join[4][64][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = wave >> 2;
  const unsigned cols = (unsigned)(N + 31) / 32;
  const int m0 = (int)(blockIdx.x / cols) * 32, n0 = (int)(blockIdx.x % cols) * 32;
  const int wm = (wave & 1) * 16, wn = (wave >> 1 & 1) * 16;
  doublex4 acc = {0.0, 0.0, 0.0, 0.0};
  float ra[2][4], rb[2][4];
  // A thread's four elements of an operand's 32 x 64: along whichever of row and k is contiguous.  Rows behind the last one read the last one, for
  // results that nobody stores.  In the step where the contraction ends, elements behind the end read the first one of the row and become 0 on the
  // way to LDS.  No load stands behind a condition or is looked at before, so nobody waits for it before it is due.
  struct Side { const float* p; long ks; int r, k, dk; bool vec; } a, b;
  auto side = [&](const Operand& o, int r0, int rows) {
    Side s;
    const bool along = o.ks == 1;
    s.r = along ? tid >> 4 : tid & 31;
    s.k = along ? (tid & 15) * 4 : tid >> 5;
    s.dk = along ? 1 : 16;
    s.ks = o.ks;
    s.p = o.p + (long)(r0 + s.r < rows ? r0 + s.r : rows - 1) * o.rs;
    s.vec = along && ((uintptr_t)o.p & 15) == 0 && (o.rs & 3) == 0;
    return s;
  };
  a = side(A, m0, M);
  b = side(B, n0, N);
  const float *next_a = a.p + a.k * a.ks, *next_b = b.p + b.k * b.ks;
  auto load = [&](const Side& s, const float*& next, int k0, float (&v)[4]) {
    if (k0 + KS > K) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = s.p[k0 + s.k + i * s.dk < K ? (k0 + s.k + i * s.dk) * s.ks : 0];
      return;
    }
    if (s.vec) {
      const float4 q = *reinterpret_cast<const float4*>(next);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = next[i * s.dk * s.ks];
    }
    next += KS * s.ks;
  };
  auto put = [&](const Side& s, float* to, int k0, float (&v)[4]) {
    if (k0 + KS > K)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k0 + s.k + i * s.dk >= K) v[i] = 0.f;
    if (s.dk == 1) {
      *reinterpret_cast<float4*>(to + s.r * LS + s.k) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) to[s.r * LS + s.k + 16 * i] = v[i];
    }
  };
  auto step = [&](int k0, auto set) {        // the registers of a step have been loaded two steps before
    constexpr int S = decltype(set)::value;
    put(a, sA[S], k0, ra[S]);
    put(b, sB[S], k0, rb[S]);
    if (k0 + 2 * KS < K) {
      load(a, next_a, k0 + 2 * KS, ra[S]);
      load(b, next_b, k0 + 2 * KS, rb[S]);
    }
    __syncthreads();
    float fa[KS / 8], fb[KS / 8];             // all fragments asked for ahead of the products
#pragma unroll
    for (int i = 0; i < KS / 8; ++i) {
      const int c = part * (KS / 2) + i * 4 + (lane >> 4);
      fa[i] = sA[S][(wm + (lane & 15)) * LS + c];
      fb[i] = sB[S][(wn + (lane & 15)) * LS + c];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < KS / 8; ++i) acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)fb[i], (double)fa[i], acc, 0, 0, 0);
  };
  load(a, next_a, 0, ra[0]);
  load(b, next_b, 0, rb[0]);
  if (KS < K) {
    load(a, next_a, KS, ra[1]);
    load(b, next_b, KS, rb[1]);
  }
  for (int k0 = 0; k0 < K; k0 += 2 * KS) {
    step(k0, std::integral_constant<int, 0>{});
    if (k0 + KS < K) step(k0 + KS, std::integral_constant<int, 1>{});
  }
  if (part)
#pragma unroll
    for (int r = 0; r < 4; ++r) join[wave & 3][lane][r] = acc[r];
  __syncthreads();
  if (part) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int m = m0 + wm + (lane & 15), n = n0 + wn + (lane >> 4) + 4 * r;      // rows of the first operand: n
    if (m >= M || n >= N) continue;
    double z = acc[r] + join[wave][lane][r], y, slope;
    if (e.sum) {
      float* o = e.sum + (long)m * N + n;
      *o = (float)(e.accumulate ? z + *o : z);
      continue;
    }
    if (e.bias) z += e.bias[n];
    activate(e.act, z, y, slope);
    if (e.residual) y += e.residual[m * e.ldr + n];
    e.y[m * e.ldy + n] = (float)y;
    if (e.slope) e.slope[(long)m * N + n] = (float)slope;
  }
}

// ---- bf16: tiles on matrix cores -------------------------------------------------------------------------------------
// C[m][n] = sum_k A[m][k] B[n][k], both operands with k contiguous, rows on 16 bytes; k >= K counts as 0 in A, and B's rows are padded
// with zeros to a multiple of 64.  ROWS: C[m][n] = sum_k A[k][m] B[k][n], the contraction over the operands' rows (dw = x^T dz), k >= K
// counts as 0 in both; M and N as wide as the rows, multiples of 8 that may count columns beyond the result's.
enum : int { OUT_Y = 0, OUT_SUM = 1, OUT_SLAB = 2 };
struct Product {
  const bf16_t* A; long lda;
  const bf16_t* B; long ldb;
  int M, N, K;
  int widthA, widthB;           // ROWS: readable columns
  // OUT_Y
  const float* bias;
  const bf16_t* residual; long ldr;
  bf16_t* y; long ldy;
  bf16_t* slope;
  int act;
  // OUT_SUM: C in fp32 [M][N]; OUT_SLAB: this share's C, [splits][M][slab_row(N)]
  float* sum; int accumulate;
};

__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};   // where lanes beyond the end of a row read

// Phi(z) and sqrt(2 pi) times the normal density by one exponential.  Phi(-x) exp(x^2 / 2) of x = |z| is a polynomial in t = 1 / (1 + 0.2885 x) without a
// constant term, fitted to the least largest deviation, absolute and relative at once: Phi(-x) is off by 1.9e-7 at most, rounding included (a
// hundredth of a bf16 step at 1), and by 1.4e-4 of itself at most down to 2^-126 (x = 13), a thirtieth of half a bf16 step, so that the tail of gelu
// keeps its digits.
__device__ __forceinline__ void normal(float z, float& below, float& e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.2885f, fabsf(z), 1.f));
  e = __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.44269504f));
  const float q = e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0916117206f, 0.300303638f), -0.112923115f), 0.190809026f), 0.0968033150f), 0.116618834f);
  below = z < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ void activate_fast(int act, float z, float& y, float& slope) {
  if (act == ACT_GELU) {
    float below, e;
    normal(z, below, e);
    y = z * below;
    slope = fmaf(z * 0.39894228f, e, below);
  } else if (act == ACT_SILU) {
    const float q = __builtin_amdgcn_rcpf(1.f + __expf(-z));
    y = z * q;
    slope = q * fmaf(z, 1.f - q, 1.f);
  } else {
    activate<float>(act, z, y, slope);
  }
}

// Eight consecutive results of a row, n a multiple of 8.  The bias and, where rows allow 16-byte loads, the residual are asked for ahead of the
// sums they join: one at a time they cost a trip to memory for every 16 rows of a tile.  With residual, bias, gelu and slope
// 8192 x 4096 x 4096 takes 254 us, 54 of them on top of the product; their bytes alone take 32.
struct Ahead { float bias[8]; };
__device__ __forceinline__ bool wide_rows(const bf16_t* p, long ld) { return (ld & 7) == 0 && ((uintptr_t)p & 15) == 0; }
template <int OUT>
__device__ __forceinline__ Ahead ahead(const Product& p, int n) {
  Ahead a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a.bias[e] = OUT == OUT_Y && p.bias && n + e < p.N ? p.bias[n + e] : 0.f;
  return a;
}
template <int OUT>
__device__ __forceinline__ uint4 residual8(const Product& p, int m, int n) {
  if (OUT == OUT_Y && p.residual && m < p.M && n + 8 <= p.N && wide_rows(p.residual, p.ldr)) return *reinterpret_cast<const uint4*>(p.residual + m * p.ldr + n);
  return make_uint4(0u, 0u, 0u, 0u);
}
template <int OUT>
__device__ __forceinline__ void finish8(const Product& p, int m, int n, float (&v)[8], unsigned split, const Ahead& a, const uint4& res) {
  const int left = p.N - n;
  if (OUT == OUT_SLAB) {
    store8(p.sum + ((size_t)split * p.M + m) * slab_row(p.N) + n, v);
    return;
  }
  if (OUT == OUT_SUM) {
    float* o = p.sum + (size_t)m * p.N + n;
    const bool add = p.accumulate;
    if (left >= 8 && (p.N & 3) == 0 && ((uintptr_t)p.sum & 15) == 0) {       // rows on 16 bytes
      if (add) {
        float w[8];
        load8(o, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[e];
      }
      store8(o, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) o[e] = add ? o[e] + v[e] : v[e];
    }
    return;
  }
  const bool whole = left >= 8;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += a.bias[e];
  if (p.act != ACT_NONE) {
    float sl[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y;
      activate_fast(p.act, v[e], y, sl[e]);
      v[e] = y;
    }
    if (p.slope) {
      bf16_t* o = p.slope + (size_t)m * p.N + n;
      if (whole && wide_rows(p.slope, p.N)) store8(o, sl);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) o[e] = f32_to_bf16(sl[e]);
    }
  } else if (p.slope) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p.slope[(size_t)m * p.N + n + e] = f32_to_bf16(1.f);
  }
  if (p.residual) {
    if (whole && wide_rows(p.residual, p.ldr)) {
      const uint32_t w[4] = {res.x, res.y, res.z, res.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    } else {
      const bf16_t* o = p.residual + m * p.ldr + n;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) v[e] += bf16_to_f32(o[e]);
    }
  }
  bf16_t* o = p.y + m * p.ldy + n;
  if (whole && wide_rows(p.y, p.ldy)) store8(o, v);
  else
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) o[e] = f32_to_bf16(v[e]);
}

// Work-group i of n: the die it runs on is i % 8 (each has its own L2), so die d takes the d-th eighth of the tiles, and neighbours in that
// order share operands: blocks of GROUP tile rows, column by column.
__device__ __forceinline__ void tile_of(unsigned i, unsigned rows, unsigned cols, unsigned& r, unsigned& c) {
  constexpr unsigned GROUP = 8;
  const unsigned n = rows * cols, die = i & 7, at = i >> 3, share = n >> 3, extra = n & 7;
  const unsigned t = die * share + (die < extra ? die : extra) + at;
  const unsigned g = t / (GROUP * cols), r0 = g * GROUP, h = rows - r0 < GROUP ? rows - r0 : GROUP, u = t - g * GROUP * cols;
  c = u / h;
  r = r0 + (u - c * h);
}

// s_waitcnt vmcnt(n), and lgkmcnt(0) with it
constexpr int wait_loads(int n) { return 0x0070 | (n & 15) | (n >> 4) << 14; }

// 16 bytes per lane from memory to LDS, lane i's to lds + 16 i; lds: byte address, the same in all lanes.  Written out because the compiler, which
// knows the builtin as a write to LDS, lets every read that it cannot tell apart from it (ds_read_b64_tr_b16 for one) wait for all of them:
// 416 instead of 200 us for dw of 4096 x 4096 from 8192 rows.  Nothing is returned in registers; who reads has waited (wait_loads, a barrier).
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "m0");
}
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char* at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(at) : "m0");
}

// A barrier that no access to LDS is moved across; what has to be waited for, the caller waits for
__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// BM x BN tile by WM x WN waves; 64 of the contraction per step, STAGES of them in LDS, loaded past the registers.  A stage's row is 128 bytes;
// its 16-byte units are stored in the order unit ^ (row & 7), so that 8 neighbouring rows' reads of one unit fall on all banks.
// A step has two halves of 32.  Among the products of the first, the fragments of the second are read; between the halves comes the step's only
// barrier, behind which the next stage is complete and this one free; among the products of the second half, the loads of a later step
// go out into it and the first fragments of the next step are read.  Issued in one burst instead, these reads and loads kept the matrix
// cores waiting: 213 instead of 200 us at 8192 x 4096 x 4096 (1370 TFLOP/s; 4096 x 8192 x 4096, one tile per CU: 1440).
//
// ROWS: a stage is 64 rows of BM and of BN columns, and ds_read_b64_tr_b16 turns them on the way into the registers: from four rows' 4 x 16
// elements every lane of 16 gets a column's four.  The 32-byte pieces of a row are stored in the order piece ^ f(row), with f over the 16 rows
// of a read such that no more than two of them share banks, and two trips are what 512 bytes take anyway.  dw of 4096 x 4096 from 8192 rows,
// within a backward call: 240 us (dx: 249).  Turned copies of both operands instead were a pass over each before it, 85 us, of which 44 remain
// for dz = dy * slope.
template <int BM, int BN, int WM, int WN, int STAGES, int OUT, bool ROWS>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_mfma(Product p, unsigned tile_rows, unsigned tile_cols, int steps_per_split) {
  constexpr int NT = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, STAGE = (BM + BN) * 64;
  constexpr int LA = BM * 8 / NT, LB = BN * 8 / NT;      // 16-byte units per thread and step
  extern __shared__ __align__(16) bf16_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  unsigned tr, tc;
  tile_of(blockIdx.x, tile_rows, tile_cols, tr, tc);
  const int m0 = (int)tr * BM, n0 = (int)tc * BN;
  const int k_begin = (int)blockIdx.y * steps_per_split, k_all = (p.K + 63) / 64;
  const int steps = (k_all - k_begin < steps_per_split ? k_all - k_begin : steps_per_split);

  // thread: rows tid / 8 + i * NT / 8, unit tid % 8 of the stage, which holds unit (tid ^ row) % 8 of the operand.  Rows behind the last one read
  // the last one; offsets within a tile fit 32 bits (256 rows, 2^22 apart at most).
  const int unit = (tid ^ (tid >> 3)) & 7;
  uint32_t oa[LA], ob[LB];
  // ROWS: thread's unit i is unit i * NT + tid of the stage, rows of W / 8 units; columns behind the last one read the last ones.  Its units are a
  // multiple of 16 rows apart, in the same column, so that one offset serves all.
  auto piece = [](int r, int W) { return W == 64 ? (r >> 1 & 1) | (r >> 3 & 1) << 1 : (r & 3) | (r >> 3 & 1) << 2; };
  static_assert(NT * 8 / BM % 16 == 0 && NT * 8 / BN % 16 == 0, "a thread's units share their column");
  auto at_rows = [&](int W, long ld, int first, int width) {
    const int r = tid / (W / 8), c = tid % (W / 8);
    int col = first + (((c >> 1 ^ piece(r, W)) << 1 | (c & 1)) << 3);
    if (col > width - 8) col = width - 8;
    return (uint32_t)(r * ld + col) * 2u;
  };
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int r = (tid >> 3) + i * (NT / 8), last = p.M - 1 - m0;
    oa[i] = ROWS ? at_rows(BM, p.lda, m0, p.widthA) : (uint32_t)((r < last ? r : last) * p.lda + unit * 8) * 2u;
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int r = (tid >> 3) + i * (NT / 8), last = p.N - 1 - n0;
    ob[i] = ROWS ? at_rows(BN, p.ldb, n0, p.widthB) : (uint32_t)((r < last ? r : last) * p.ldb + unit * 8) * 2u;
  }
  const char* ga = (const char*)(ROWS ? p.A + (long)k_begin * 64 * p.lda : p.A + m0 * p.lda + k_begin * 64);
  const char* gb = (const char*)(ROWS ? p.B + (long)k_begin * 64 * p.ldb : p.B + n0 * p.ldb + k_begin * 64);
  const long step_a = ROWS ? 128 * p.lda : 128, step_b = ROWS ? 128 * p.ldb : 128;        // bytes
  const int k_left = p.K - k_begin * 64;
  const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem) + (uint32_t)wave * 1024u;
  auto load_unit = [&](int step, int i, bool ends) {     // unit i < LA of A, then those of B; ends: the contraction ends within this step
    const uint32_t s = lds0 + (uint32_t)(step % STAGES) * (STAGE * 2) + (uint32_t)i * (NT * 16);      // B's units follow A's
    const bool of_a = i < LA;
    const char* base = of_a ? ga + step * step_a : gb + step * step_b;
    if (ROWS) base += of_a ? i * (NT * 8 / BM) * 2 * p.lda : (i - LA) * (NT * 8 / BN) * 2 * p.ldb;
    const uint32_t offset = of_a ? oa[of_a ? i : 0] : ob[of_a ? 0 : i - LA];
    if (ends && (of_a || ROWS)) {
      const int k = ROWS ? of_a ? (i * NT + tid) / (BM / 8) : ((i - LA) * NT + tid) / (BN / 8) : unit * 8;
      load_to_lds(s, k_left <= step * 64 + k ? (const char*)kZeros : base + offset);
    } else {
      load_to_lds(s, base, offset);
    }
  };
  auto load = [&](int step) {
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) load_unit(step, i, k_left < (step + 1) * 64);
  };

  floatx4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  const int row = lane & 15, q = lane >> 4;
  const int at_a = (wm * (BM / WM) + row) * 64, at_b = BM * 64 + (wn * (BN / WN) + row) * 64;
  const int u0 = ROWS ? 0 : ((q) ^ (row & 7)) * 8, u1 = ROWS ? 32 : ((q + 4) ^ (row & 7)) * 8;
  struct Frags { bf16x8 a[TM], b[TN]; };
  // ROWS: the lane's place in a stage of either operand, its piece not yet taken in
  const int tr_row = q * 8 + (row >> 2), tr_a = tr_row * BM + piece(tr_row, BM) * 16 + (row & 3) * 4, tr_b = tr_row * BN + piece(tr_row, BN) * 16 + (row & 3) * 4;
  auto read_turned = [&](const bf16_t* s, int at, int W) {       // 8 rows of 16 columns
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4 lds_s4;
    struct Pair { s4 lo, hi; } v = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + at)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + at + 4 * W))};
    return __builtin_bit_cast(bf16x8, v);
  };
  auto read_one = [&](Frags& f, int step, int u, int i) {        // u: u0 or u1; ROWS: 0 or 32, the first row of the half
    const bf16_t* s = smem + (step % STAGES) * STAGE;
    if (ROWS) {
      if (i < TN) f.b[i < TN ? i : 0] = read_turned(s + BM * 64 + u * BN, tr_b ^ (wn * (BN / WN) + i * 16), BN);
      else f.a[i < TN ? 0 : i - TN] = read_turned(s + u * BM, tr_a ^ (wm * (BM / WM) + (i - TN) * 16), BM);
      return;
    }
    if (i < TN) f.b[i < TN ? i : 0] = *reinterpret_cast<const bf16x8*>(s + at_b + i * 1024 + u);
    else f.a[i < TN ? 0 : i - TN] = *reinterpret_cast<const bf16x8*>(s + at_a + (i - TN) * 1024 + u);
  };
  auto read = [&](Frags& f, int step, int u) {
#pragma unroll
    for (int i = 0; i < TN + TM; ++i) read_one(f, step, u, i);
  };
  // the products of a half, in TM groups with something else to issue behind each
  auto multiply = [&](const Frags& f, auto behind) {
#pragma unroll
    for (int j = 0; j < TM; ++j) {
#pragma unroll
      for (int i = 0; i < TN; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.b[i], f.a[j], acc[i][j], 0, 0, 0);
      behind(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  constexpr int READS = (TN + TM + TM - 1) / TM, LOADS = (LA + LB + TM - 1) / TM;      // per group
  auto reads = [&](Frags& f, int step, int u, int j) {
#pragma unroll
    for (int i = j * READS; i < (j + 1) * READS; ++i)
      if (i < TN + TM) read_one(f, step, u, i);
  };
  Frags f0, f1;
#pragma unroll
  for (int t = 0; t < STAGES; ++t)
    if (t < steps) load(t);
  if (steps >= STAGES) __builtin_amdgcn_s_waitcnt(wait_loads((STAGES - 1) * (LA + LB)));
  else __builtin_amdgcn_s_waitcnt(wait_loads(0));
  stage_barrier();
  read(f0, 0, u0);
  auto step = [&](int t, auto loads, bool ends) {        // loads: those of step t + STAGES among the products of the second half
    constexpr bool LOAD = decltype(loads)::value;
    __builtin_amdgcn_s_waitcnt(0xc07f);                  // lgkmcnt(0): f0
    __builtin_amdgcn_sched_barrier(0);
    multiply(f0, [&](int j) { reads(f1, t, u1, j); });
    // this thread's units of the next stage are in LDS, and f1 is here
    if (LOAD || t + STAGES == steps) __builtin_amdgcn_s_waitcnt(wait_loads((STAGES - 2) * (LA + LB)));
    else __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();                                     // everybody's are, and everybody has this stage's fragments
    multiply(f1, [&](int j) {
      reads(f0, t + 1, u0, j);
      if (LOAD)
#pragma unroll
        for (int i = j * LOADS; i < (j + 1) * LOADS; ++i)
          if (i < LA + LB) load_unit(t + STAGES, i, ends);
    });
  };
  const int whole = k_left / 64 < steps ? k_left / 64 : steps;      // steps without an end
  int t = 0;
  for (; t + STAGES < whole; ++t) step(t, std::true_type{}, false);
  if (t + STAGES < steps) { step(t, std::true_type{}, true); ++t; }
  for (; t + 1 < steps; ++t) step(t, std::false_type{}, false);
  multiply(f0, [&](int j) { reads(f1, steps - 1, u1, j); });
  multiply(f1, [](int) {});
  __syncthreads();

  // A wave's results go through its own part of LDS, 16 rows at a time, so that a lane ends up with 8 consecutive columns
  constexpr int TS = BN / WN + 4;                        // fp32 row stride: rows shift by 4 banks
  constexpr int LANES = BN / WN / 8, PASS = 64 / LANES;  // lanes per row, rows per pass
  static_assert(16 * TS * 4 * WM * WN <= STAGES * STAGE * 2, "the rows of all waves fit the stages");
  float* mine = reinterpret_cast<float*>(smem) + wave * 16 * TS;
  const int n = n0 + wn * (BN / WN) + (lane % LANES) * 8, m_lane = m0 + wm * (BM / WM) + lane / LANES;
  const Ahead a = ahead<OUT>(p, n);
  uint4 res[TM][16 / PASS];
  if (OUT == OUT_Y && p.residual)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int r = 0; r < 16; r += PASS) res[j][r / PASS] = residual8<OUT>(p, m_lane + j * 16 + r, n);
#pragma unroll
  for (int j = 0; j < TM; ++j) {
#pragma unroll
    for (int i = 0; i < TN; ++i) *reinterpret_cast<floatx4*>(mine + row * TS + i * 16 + q * 4) = acc[i][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < 16; r += PASS) {
      const int m = m_lane + j * 16 + r;
      float v[8];
      load8(mine + (r + lane / LANES) * TS + (lane % LANES) * 8, v);
      if (m < p.M && n < p.N) finish8<OUT>(p, m, n, v, blockIdx.y, a, res[j][r / PASS]);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Up to 16 rows: the product is a reading of the weights.  A wave has 16 columns and an eighth of the work-group's share of the contraction, its
// fragments straight from memory, 256 contiguous bytes of a weight row per round; the eight sums are joined in LDS.  One row of 4096 x 4096:
// 8.6 us (3.9 TB/s; a launch alone takes 3.6).
template <int OUT>
__global__ __launch_bounds__(512) void k_linear_few(Product p, int steps_per_split) {
  __shared__ __align__(16) float part[8][16][20];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16, k_all = round_up64(p.K) / 32;
  const int k_begin = (int)blockIdx.y * steps_per_split, k_end = k_begin + steps_per_split < k_all ? k_begin + steps_per_split : k_all;
  const int share = ((k_end - k_begin + 7) / 8 + 3) & ~3, k0 = k_begin + wave * share, k1 = k0 + share < k_end ? k0 + share : k_end;
  const bf16_t* a = p.A + (row < p.M ? row : p.M - 1) * p.lda + q * 8;
  const bf16_t* b = p.B + (n0 + row < p.N ? n0 + row : p.N - 1) * p.ldb + q * 8;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  auto fragment = [&](const bf16_t* r, int k, bool there) { return *reinterpret_cast<const bf16x8*>(there ? r + k * 32 : (const bf16_t*)kZeros); };
  for (int k = k0; k < k1; k += 8) {
    bf16x8 fa[8], fb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      fb[i] = fragment(b, k + i, k + i < k1);
      fa[i] = fragment(a, k + i, k + i < k1 && (k + i) * 32 + q * 8 < p.K);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[i], fa[i], acc, 0, 0, 0);
  }
  *reinterpret_cast<floatx4*>(&part[wave][row][q * 4]) = acc;        // row: m, columns: n
  __syncthreads();
  if (tid >= 32) return;
  const int m = tid >> 1, n = n0 + (tid & 1) * 8;
  if (m >= p.M || n >= p.N) return;
  float v[8] = {};
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    float t[8];
    load8(&part[w][m][(tid & 1) * 8], t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += t[e];
  }
  finish8<OUT>(p, m, n, v, blockIdx.y, ahead<OUT>(p, n), residual8<OUT>(p, m, n));
}

// y or the sum from the shares of a split contraction (4.3 us of the 14 at 128 x 4096 x 4096, two shares of 128 tiles)
template <int OUT>
__global__ __launch_bounds__(256) void k_linear_join(Product p, const float* __restrict__ slabs, int splits) {
  const int units = (p.N + 7) / 8;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)p.M * units; i += (size_t)gridDim.x * 256) {
    const int m = (int)(i / units), n = (int)(i - (size_t)m * units) * 8;
    const Ahead a = ahead<OUT>(p, n);
    const uint4 res = residual8<OUT>(p, m, n);
    const float* o = slabs + (size_t)m * slab_row(p.N) + n;
    const size_t slab = (size_t)p.M * slab_row(p.N);
    float v[8] = {};
    int s = 0;
    for (; s + 4 <= splits; s += 4) {                    // four shares on their way together
      float w[4][8];
#pragma unroll
      for (int k = 0; k < 4; ++k) load8(o + (s + k) * slab, w[k]);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[k][e];
    }
    for (; s < splits; ++s) {
      float w[8];
      load8(o + s * slab, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
    finish8<OUT>(p, m, n, v, 0, a, res);
  }
}

// dst = src (* slope), rows padded with zeros to ld, and the column sums of each group of rows; either may be missing.  A wave takes 512 columns
// of a row, four rows on their way at a time; its lanes have columns of their own, so sums need no exchange but that of the four waves.  A second
// operand's copy rides along.  dz and its sums at 8192 x 4096: 44 us (4.6 TB/s).
struct Rows {
  const bf16_t* src; long lds;
  const bf16_t* slope;          // dense
  bf16_t* dst; int ld;
  float* sums;                  // [M / group][cols]
  int M, cols;
  int group;                    // rows of a work-group, a multiple of 16
};
__global__ __launch_bounds__(256) void k_linear_rows(Rows first, Rows second, unsigned blocks) {       // blocks: of first
  __shared__ float part[4][512];
  const bool one = blockIdx.x < blocks;
  const Rows p = one ? first : second;
  const unsigned block = one ? blockIdx.x : blockIdx.x - blocks, col_blocks = (unsigned)(p.ld + 511) / 512;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = (int)(block / col_blocks), c0 = (int)(block % col_blocks) * 512, c = c0 + lane * 8;
  float sum[8] = {};
  const int left = p.cols - c;
  auto fetch = [&](const bf16_t* rows, long ld, int m0, uint32_t (&w)[4][4]) {      // four rows; behind the last one: that one
    if (left >= 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(w[i], rows + (m0 + i < p.M ? m0 + i : p.M - 1) * ld + c, 16);      // any multiple of 2 bytes will do
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16_t* r = rows + (m0 + i < p.M ? m0 + i : p.M - 1) * ld + c;
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? r[e] : 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[i][k] = v[2 * k] | v[2 * k + 1] << 16;
      }
    }
  };
  const int each = p.group / 4, m0 = g * p.group + wave * each;
  for (int i0 = 0; i0 < each; i0 += 4) {
    uint32_t r[4][4], s[4][4];
    fetch(p.src, p.lds, m0 + i0, r);
    if (p.slope) fetch(p.slope, p.cols, m0 + i0, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + i0 + i;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (p.slope)            // exact in fp32, then one rounding
          r[i][w] = pack_bf16x2(__uint_as_float(r[i][w] << 16) * __uint_as_float(s[i][w] << 16),
                                __uint_as_float(r[i][w] & 0xffff0000u) * __uint_as_float(s[i][w] & 0xffff0000u));
        if (m >= p.M) r[i][w] = 0;
        sum[2 * w] += __uint_as_float(r[i][w] << 16);
        sum[2 * w + 1] += __uint_as_float(r[i][w] & 0xffff0000u);
      }
      if (p.dst && m < p.M && c < p.ld) *reinterpret_cast<uint4*>(p.dst + (size_t)m * p.ld + c) = make_uint4(r[i][0], r[i][1], r[i][2], r[i][3]);
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) part[wave][lane + 64 * e] = sum[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int n = c0 + (i & 63) * 8 + (i >> 6);
    if (n < p.cols) p.sums[(size_t)g * p.cols + n] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
  }
}
// db from the sums of all groups of rows, one order: 16 shares of the groups, then their sums
__global__ __launch_bounds__(1024) void k_linear_db_join(const float* __restrict__ sums, int groups, float* __restrict__ db, int accumulate, int N) {
  __shared__ float part[16][64];
  const int c = threadIdx.x & 63, w = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
  float s = 0.f;
  if (n < N) {
    int i = w;
    for (; i + 48 < groups; i += 64) {
      const float a = sums[(size_t)i * N + n], b = sums[(size_t)(i + 16) * N + n], d = sums[(size_t)(i + 32) * N + n], e = sums[(size_t)(i + 48) * N + n];
      s += (a + b) + (d + e);
    }
    for (; i < groups; i += 16) s += sums[(size_t)i * N + n];
  }
  part[w][c] = s;
  __syncthreads();
  if (w == 0 && n < N) {
    s = 0.f;
    for (int k = 0; k < 16; ++k) s += part[k][c];
    db[n] = accumulate ? s + db[n] : s;
  }
}

// packed copies of w: blocks of 64 x 64 through LDS, stored 2 bytes at a time (4096 x 4096, 134 MB read and written: 37 us from memory, 3.6 TB/s; 23
// where w is in a cache from the call before)
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

// fp32: dz = dy * slope, rounded once
__global__ __launch_bounds__(256) void k_linear_dz_f32(const float* __restrict__ dy, long lddy, const float* __restrict__ slope, float* __restrict__ dz, int M, int N) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)M * N; i += (size_t)gridDim.x * 256) {
    const size_t m = i / N, n = i - m * N;
    dz[i] = dy[m * lddy + n] * slope[i];
  }
}

// fp32: column sums of dz in double, 64 columns per work-group: 16 shares of the rows, then their sums
__global__ __launch_bounds__(1024) void k_linear_db_f32(const float* __restrict__ dz, long ld, float* __restrict__ db, int accumulate, int M, int N) {
  __shared__ double part[16][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
  double s = 0.0;
  if (n < N) {
    int m = g;
    for (; m + 48 < M; m += 64) s += ((double)dz[m * ld + n] + dz[(m + 16) * ld + n]) + ((double)dz[(m + 32) * ld + n] + dz[(m + 48) * ld + n]);
    for (; m < M; m += 16) s += dz[m * ld + n];
  }
  part[g][c] = s;
  __syncthreads();
  if (g == 0 && n < N) {
    s = 0.0;
    for (int k = 0; k < 16; ++k) s += part[k][c];
    db[n] = (float)(accumulate ? s + db[n] : s);
  }
}

unsigned blocks64(int v) { return (unsigned)((v + 63) / 64); }
unsigned grid_for(size_t n, size_t per, size_t cap) {
  const size_t g = (n + per - 1) / per;
  return (unsigned)(g < 1 ? 1 : g > cap ? cap : g);
}

template <int BM, int BN, int WM, int WN, int STAGES, int OUT, bool ROWS>
hipError_t mfma(const Product& p, const Cut& c, hipStream_t s) {
  constexpr int lds = STAGES * (BM + BN) * 64 * 2;
  const auto kernel = k_linear_mfma<BM, BN, WM, WN, STAGES, OUT, ROWS>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3(c.rows * c.cols, (unsigned)c.splits), 64 * WM * WN, lds, s>>>(p, c.rows, c.cols, c.steps);
  return hipGetLastError();
}
template <int OUT>
hipError_t few(const Product& p, const Cut& c, hipStream_t s) {
  k_linear_few<OUT><<<dim3(c.cols, (unsigned)c.splits), 512, 0, s>>>(p, c.steps);
  return hipGetLastError();
}

// y, or (ROWS) a sum; slabs: room for slab_bytes(c, ...)
template <bool ROWS>
hipError_t product(const Product& p, const Cut& c, float* slabs, hipStream_t s) {
  constexpr int OUT = ROWS ? OUT_SUM : OUT_Y;
  if (c.kind == CUT_LARGE) return mfma<256, 256, 2, 4, 2, OUT, ROWS>(p, c, s);
  if (c.kind == CUT_TILES) return mfma<128, 128, 2, 2, 2, OUT, ROWS>(p, c, s);
  if (c.splits == 1) {
    if constexpr (!ROWS)
      if (c.kind == CUT_FEW) return few<OUT>(p, c, s);
    return mfma<64, 64, 2, 2, 4, OUT, ROWS>(p, c, s);
  }
  Product q = p;
  q.sum = slabs;
  hipError_t e;
  if (!ROWS && c.kind == CUT_FEW) e = few<OUT_SLAB>(q, c, s);
  else e = mfma<64, 64, 2, 2, 4, OUT_SLAB, ROWS>(q, c, s);
  if (e != hipSuccess) return e;
  k_linear_join<OUT><<<grid_for((size_t)p.M * ((p.N + 7) / 8), 256, 2048), 256, 0, s>>>(p, slabs, c.splits);
  return hipGetLastError();
}

// Rows that the tiles read where they are: 16-byte units, and 256 rows within 32-bit offsets
bool direct(const void* p, long ld, int K) { return ((uintptr_t)p & 15) == 0 && (ld & 7) == 0 && (K & 7) == 0 && ld <= 1 << 22; }

unsigned row_blocks(const Rows& r) { return (unsigned)((r.M + r.group - 1) / r.group) * (unsigned)((r.ld + 511) / 512); }
// a copy whose rows start on 16 bytes
Rows copy_of(const void* x, long ldx, int M, int K, char* to) {
  const int Kp = round_up64(K);
  return Rows{(const bf16_t*)x, ldx, nullptr, (bf16_t*)to, Kp, nullptr, M, K, group_of(M, Kp)};
}

hipError_t forward_bf16(const LinearForward& a, char* ws, hipStream_t s) {
  const ForwardSpace at(a.M, a.K, a.N);
  Product p{};
  p.A = (const bf16_t*)a.x; p.lda = a.ldx; p.M = a.M; p.N = a.N; p.K = a.K;
  if (!direct(a.x, a.ldx, a.K)) {
    const Rows r = copy_of(a.x, a.ldx, a.M, a.K, ws);
    k_linear_rows<<<row_blocks(r), 256, 0, s>>>(r, r, row_blocks(r));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.A = r.dst; p.lda = p.K = r.ld;
  }
  p.B = (const bf16_t*)a.weights; p.ldb = round_up64(a.K);
  p.bias = a.bias; p.residual = (const bf16_t*)a.residual; p.ldr = a.ldr; p.y = (bf16_t*)a.y; p.ldy = a.ldy; p.slope = (bf16_t*)a.slope; p.act = a.act;
  return product<false>(p, at.y, (float*)(ws + at.slabs), s);
}

hipError_t backward_bf16(const LinearBackward& a, char* ws, hipStream_t s) {
  const BackwardSpace at(a.M, a.K, a.N);
  const int Np = round_up64(a.N);
  const bool copy = (a.dx || a.dw) && (a.slope || !direct(a.dy, a.lddy, a.N));
  const bf16_t* dz = copy ? (const bf16_t*)(ws + at.dz) : (const bf16_t*)a.dy;
  const long lddz = copy ? Np : a.lddy;
  float* sums = (float*)(ws + at.sums);
  const bool copy_x = a.dw && !direct(a.x, a.ldx, a.K);
  const Rows x = copy_of(a.x, a.ldx, a.M, a.K, ws + at.x);
  hipError_t e = hipSuccess;
  if (copy || a.db || copy_x) {
    const Rows r{(const bf16_t*)a.dy, a.lddy, (const bf16_t*)a.slope, copy ? (bf16_t*)(ws + at.dz) : nullptr, Np, a.db ? sums : nullptr, a.M, a.N, at.group};
    const unsigned blocks = copy || a.db ? row_blocks(r) : 0;
    k_linear_rows<<<blocks + (copy_x ? row_blocks(x) : 0), 256, 0, s>>>(r, x, blocks);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.db) {
    k_linear_db_join<<<blocks64(a.N), 1024, 0, s>>>(sums, at.groups, a.db, a.accumulate, a.N);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.dx) {
    Product p{};
    p.A = dz; p.lda = lddz;
    p.B = (const bf16_t*)a.weights + (size_t)a.N * round_up64(a.K); p.ldb = Np;
    p.M = a.M; p.N = a.K; p.K = copy ? Np : a.N;
    p.y = (bf16_t*)a.dx; p.ldy = a.lddx;
    e = product<false>(p, at.dx, (float*)(ws + at.slabs), s);
  }
  if (e == hipSuccess && a.dw) {
    Product p{};
    p.A = copy_x ? x.dst : (const bf16_t*)a.x; p.lda = copy_x ? x.ld : a.ldx;
    p.widthA = copy_x ? x.ld : a.K;
    p.B = dz; p.ldb = lddz; p.widthB = copy ? Np : a.N;
    p.M = a.K; p.N = a.N; p.K = a.M; p.sum = a.dw; p.accumulate = a.accumulate;
    e = product<true>(p, at.dw, (float*)(ws + at.slabs), s);
  }
  return e;
}

// ---- fp32 (check mode) -----------------------------------------------------------------------------------------------
hipError_t tile(const Operand& A, const Operand& B, const Epilogue& e, int M, int N, int K, hipStream_t s) {
  k_linear_tile_f32<<<(unsigned)((N + 31) / 32) * (unsigned)((M + 31) / 32), 512, 0, s>>>(A, B, e, M, N, K);
  return hipGetLastError();
}

hipError_t forward_f32(const LinearForward& a, hipStream_t s) {
  const Epilogue e{a.bias, (const float*)a.residual, a.ldr, (float*)a.y, a.ldy, (float*)a.slope, nullptr, 0, a.act};
  return tile({(const float*)a.x, a.ldx, 1}, {(const float*)a.weights, 1, a.N}, e, a.M, a.N, a.K, s);
}

hipError_t backward_f32(const LinearBackward& a, float* ws, hipStream_t s) {
  const float* dz = (const float*)a.dy;
  long ld = a.lddy;
  hipError_t err = hipSuccess;
  if (a.slope) {
    k_linear_dz_f32<<<grid_for((size_t)a.M * a.N, 2048, 4096), 256, 0, s>>>(dz, ld, (const float*)a.slope, ws, a.M, a.N);
    dz = ws;
    ld = a.N;
    err = hipGetLastError();
  }
  if (err == hipSuccess && a.db) {
    k_linear_db_f32<<<blocks64(a.N), 1024, 0, s>>>(dz, ld, a.db, a.accumulate, a.M, a.N);
    err = hipGetLastError();
  }
  if (err == hipSuccess && a.dx) {
    Epilogue e{};
    e.y = (float*)a.dx; e.ldy = a.lddx;
    err = tile({dz, ld, 1}, {(const float*)a.weights, a.N, 1}, e, a.M, a.K, a.N, s);
  }
  if (err == hipSuccess && a.dw) {
    Epilogue e{};
    e.sum = a.dw; e.accumulate = a.accumulate;
    err = tile({(const float*)a.x, 1, a.ldx}, {dz, 1, ld}, e, a.K, a.N, a.M, s);
  }
  return err;
}

}  // namespace

hipError_t launch_linear_pack(const float* w, bf16_t* packed, int K, int N, hipStream_t stream) {
  k_linear_pack<<<dim3(blocks64(N), blocks64(K)), 256, 0, stream>>>(w, packed, K, N, round_up64(K), round_up64(N));
  return hipGetLastError();
}

size_t linear_workspace_bytes(int dt, int M, int K, int N) {
  if (dt != DT_BF16) return (size_t)M * N * sizeof(float);
  const size_t f = ForwardSpace(M, K, N).bytes, b = BackwardSpace(M, K, N).bytes;
  return f > b ? f : b;
}

hipError_t launch_linear_forward(int dt, const LinearForward& a, void* workspace, hipStream_t stream) {
  return dt == DT_BF16 ? forward_bf16(a, (char*)workspace, stream) : forward_f32(a, stream);
}
hipError_t launch_linear_backward(int dt, const LinearBackward& a, void* workspace, hipStream_t stream) {
  return dt == DT_BF16 ? backward_bf16(a, (char*)workspace, stream) : backward_f32(a, (float*)workspace, stream);
}

}  // namespace hpf
