// Internal interface of the operators at the answer end of a model: the matrix product with its epilogue
// (kernels_linear.hip) and the row operators on logits (kernels_logits.hip).  Entry points: ops_answer.hip.
// Every launcher only enqueues work on `stream` and returns hipGetLastError().
#pragma once
#include "hpf_kernels.h"
#include "hpf_linear_cut.h"

namespace hpf {

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

// y = act(x W + bias) + residual, slope = act'(x W + bias)
struct LinearForward {
  const void* x; long ldx;
  const void* weights;          // bf16: packed copies; f32: [K][N]
  const float* bias;            // may be null, like residual and slope
  const void* residual; long ldr;
  void* y; long ldy;
  void* slope;                  // [M][N]
  int M, K, N, act;
};
// dz = dy * slope; dx = dz W^T, dw (+)= x^T dz, db (+)= column sums of dz; dx, dw, db may be null
struct LinearBackward {
  const void* dy; long lddy;
  const void* x; long ldx;
  const void* weights;
  const void* slope;            // null: dz = dy
  void* dx; long lddx;
  float* dw;
  float* db;
  int accumulate;               // dw, db: add to what is there
  int M, K, N;
};

// Packed weights: bf16 [N][Kp] (forward operand), then bf16 [K][Np] (operand of dx), rows padded with zeros
inline size_t linear_packed_elems(int K, int N) { return (size_t)N * round_up64(K) + (size_t)K * round_up64(N); }
hipError_t launch_linear_pack(const float* w, bf16_t* packed, int K, int N, hipStream_t stream);

size_t linear_workspace_bytes(int dt, int M, int K, int N);
hipError_t launch_linear_forward(int dt, const LinearForward& a, void* workspace, hipStream_t stream);
hipError_t launch_linear_backward(int dt, const LinearBackward& a, void* workspace, hipStream_t stream);

constexpr int TOP_MAX = 64;     // entries of a list: one per lane
struct LogprobForward {
  const void* logits; long ld;
  const int* labels;            // may be null, like every output
  float *logprob, *entropy; int* rank;
  float* stats;                 // [rows][2]: maximum, log of the sum of exp(logit - maximum)
  int* top_index; float* top_logprob;
  int top, rows, classes;
};
struct LogprobBackward {
  const void* logits; long ld;
  const int* labels;
  const float *stats, *grad_logprob, *entropy, *grad_entropy;   // grad_logprob / grad_entropy may be null
  void* dlogits; long ldd;
  int rows, classes;
};
struct Distill {
  const void* logits; long ld;
  const int* top_index; const float* top_logit;
  const int* labels;
  const float* row_weight;      // null: 1
  float* loss;
  void* dlogits; long ldd;      // null: no gradient
  float temperature, hard_weight;
  int top, rows, classes;
};
size_t logits_workspace_bytes(int dt, int rows, int classes, int top);
hipError_t launch_logprob_forward(int dt, const LogprobForward& a, void* workspace, hipStream_t stream);
// 1024 16-byte units of a row, with the one that a row across a boundary has more: a work-group of 256 threads each.  A launch takes fewer than 2^32
// threads.
inline int64_t logprob_backward_pieces(size_t elem, int classes) {
  const int64_t each = 16 / (int64_t)elem, units = (classes + each - 1) / each + 1;
  return (units + 1023) / 1024;
}
constexpr int64_t LOGPROB_BACKWARD_MOST = (1 << 24) - 1;
hipError_t launch_logprob_backward(int dt, const LogprobBackward& a, hipStream_t stream);
hipError_t launch_distill(int dt, const Distill& a, void* workspace, hipStream_t stream);

}  // namespace hpf
