// Entry points of the operators at the answer end of a model (include/hpf.h): argument checks and launches.
#include "hpf_answer.h"
#include "hpf_error.h"

using namespace hpf;

namespace {

constexpr int MAX_WIDTH = 1 << 20;       // columns of a matrix
constexpr int MAX_CLASSES = 1 << 28;

bool type_of(hpf_dtype dtype, int& dt) {
  dt = dtype == HPF_BF16 ? DT_BF16 : DT_F32;
  return dtype == HPF_BF16 || dtype == HPF_F32;
}
bool rows_ok(int64_t ld, int32_t cols) { return ld >= cols && ld <= (int64_t)1 << 40; }
size_t elem(int dt) { return dt == DT_BF16 ? 2 : 4; }
bool element_aligned(const void* p, int dt) { return (uintptr_t)p % elem(dt) == 0; }
// fp32 or int32 arrays
template <class... P>
bool words_aligned(const P*... p) { return (((uintptr_t)p | ... | (uintptr_t)0) & 3) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + nb && y < x + na;
}
// a [rows, cols] matrix with row stride ld, elements of e bytes; none without an address
struct Matrix {
  const void* p; int64_t rows, cols, ld; size_t e;
  size_t span() const { return p && rows ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * e : 0; }
};
// Columns of one wider matrix, side by side, do not overlap.
bool overlap(const Matrix& a, const Matrix& b) {
  if (!a.span() || !b.span() || !overlap(a.p, a.span(), b.p, b.span())) return false;
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p), e = (int64_t)a.e;
  if (a.ld != b.ld || !a.ld || a.e != b.e || d % e) return true;
  const int64_t at = ((d / e) % a.ld + a.ld) % a.ld;      // b's first column, counted from a's
  return at < a.cols || at + b.cols > a.ld;
}
// `count` numbers of 4 bytes, or `bytes`, in one piece
Matrix words(const void* p, int64_t count) { return Matrix{p, 1, count, 0, 4}; }
Matrix piece(const void* p, size_t bytes) { return Matrix{p, 1, (int64_t)bytes, 0, 1}; }
// Whether an output shares an element with another output or with an input
template <size_t O, size_t I>
bool collide(const Matrix (&out)[O], const Matrix (&in)[I]) {
  for (size_t i = 0; i < O; ++i) {
    for (size_t j = i + 1; j < O; ++j)
      if (overlap(out[i], out[j])) return true;
    for (const Matrix& q : in)
      if (overlap(out[i], q)) return true;
  }
  return false;
}
// The workspace is an output and holds nothing of the call's
template <size_t N>
bool workspace_apart(const void* workspace, size_t need, const Matrix (&of)[N]) {
  for (const Matrix& q : of)
    if (need && overlap(piece(workspace, need), q)) return false;
  return true;
}
hpf_status launched(hipError_t e) { return e == hipSuccess ? HPF_OK : fail(HPF_EDEVICE, "launch failed: %s", hipGetErrorString(e)); }

hpf_status linear_shape(hpf_dtype dtype, int32_t M, int32_t K, int32_t N, int& dt) {
  if (!type_of(dtype, dt)) return fail(HPF_EINVAL, "unknown dtype");
  if (M < 0 || K < 1 || N < 1) return fail(HPF_EINVAL, "M must not be negative, K and N must be positive (%d, %d, %d)", M, K, N);
  if (K > MAX_WIDTH || N > MAX_WIDTH || M > (1 << 21)) return fail(HPF_EUNSUPPORTED, "more than 2^21 rows or 2^20 columns (%d, %d, %d)", M, K, N);
  const int64_t most = (int64_t)1 << 32;
  if ((int64_t)M * N > most || (int64_t)M * K > most || (int64_t)K * N > most)
    return fail(HPF_EUNSUPPORTED, "a matrix of more than 2^32 elements (%d, %d, %d)", M, K, N);
  return HPF_OK;
}
Matrix weights_of(int dt, const void* weights, int32_t K, int32_t N) {
  return dt == DT_BF16 ? piece(weights, linear_packed_elems(K, N) * sizeof(bf16_t)) : words(weights, (int64_t)K * N);
}
hpf_status workspace_ok(const void* workspace, size_t bytes, size_t need) {
  if (!need) return HPF_OK;
  if (!workspace) return fail(HPF_EINVAL, "null workspace");
  if ((uintptr_t)workspace % 256) return fail(HPF_EINVAL, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(HPF_ENOMEM, "workspace has %zu bytes, %zu needed", bytes, need);
  return HPF_OK;
}

}  // namespace

extern "C" {

size_t hpf_op_linear_packed_bytes(int32_t K, int32_t N) {
  int dt;
  return linear_shape(HPF_BF16, 0, K, N, dt) != HPF_OK ? 0 : linear_packed_elems(K, N) * sizeof(bf16_t);
}

hpf_status hpf_op_linear_pack(const float* w, int32_t K, int32_t N, void* packed, size_t packed_bytes, void* hip_stream) {
  int dt;
  const hpf_status st = linear_shape(HPF_BF16, 0, K, N, dt);
  if (st != HPF_OK) return st;
  if (!w || !packed) return fail(HPF_EINVAL, "null tensor");
  if (!words_aligned(w)) return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if ((uintptr_t)packed % 256) return fail(HPF_EINVAL, "packed weights must be 256-byte aligned");
  const size_t need = hpf_op_linear_packed_bytes(K, N);
  if (packed_bytes < need) return fail(HPF_ENOMEM, "packed weights have %zu bytes, %zu needed", packed_bytes, need);
  if (overlap(w, (size_t)K * N * 4, packed, need)) return fail(HPF_EINVAL, "packed weights overlap the weights");
  return launched(launch_linear_pack(w, (bf16_t*)packed, K, N, (hipStream_t)hip_stream));
}

size_t hpf_op_linear_workspace_bytes(hpf_dtype dtype, int32_t M, int32_t K, int32_t N) {
  int dt;
  if (linear_shape(dtype, M, K, N, dt) != HPF_OK || M == 0) return 0;
  return linear_workspace_bytes(dt, M, K, N);
}

hpf_status hpf_op_linear_forward(hpf_dtype dtype, const void* x, int64_t ldx, const void* weights, const float* bias,
                                 const void* residual, int64_t ldr, void* y, int64_t ldy, void* slope, int32_t M, int32_t K,
                                 int32_t N, int32_t activation, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int dt;
  hpf_status st = linear_shape(dtype, M, K, N, dt);
  if (st != HPF_OK) return st;
  if (activation < ACT_NONE || activation > ACT_SILU) return fail(HPF_EINVAL, "unknown activation %d", activation);
  if (M == 0) return HPF_OK;
  if (!x || !weights || !y) return fail(HPF_EINVAL, "null tensor");
  if (!rows_ok(ldx, K) || !rows_ok(ldy, N) || (residual && !rows_ok(ldr, N))) return fail(HPF_EINVAL, "row stride shorter than a row");
  if (!element_aligned(x, dt) || !element_aligned(y, dt) || !element_aligned(residual, dt) || !element_aligned(slope, dt) || !words_aligned(bias) ||
      (dt == DT_F32 && !element_aligned(weights, dt)))
    return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if (dt == DT_BF16 && (uintptr_t)weights % 256) return fail(HPF_EINVAL, "packed weights must be 256-byte aligned");
  const size_t e = elem(dt), need = linear_workspace_bytes(dt, M, K, N);
  const Matrix added{residual, M, N, ldr, e}, in[] = {{x, M, K, ldx, e}, weights_of(dt, weights, K, N), words(bias, N)},
               out[] = {{y, M, N, ldy, e}, {slope, M, N, N, e}};
  if (collide(out, in) || overlap(added, out[1]) || (overlap(added, out[0]) && (residual != y || ldr != ldy)))
    return fail(HPF_EINVAL, "an output overlaps another tensor (only residual and y may be the same)");
  st = workspace_ok(workspace, workspace_bytes, need);
  if (st != HPF_OK) return st;
  const Matrix all[] = {added, in[0], in[1], in[2], out[0], out[1]};
  if (!workspace_apart(workspace, need, all)) return fail(HPF_EINVAL, "the workspace overlaps a tensor");
  const LinearForward a{x, ldx, weights, bias, residual, ldr, y, ldy, slope, M, K, N, activation};
  return launched(launch_linear_forward(dt, a, workspace, (hipStream_t)hip_stream));
}

hpf_status hpf_op_linear_backward(hpf_dtype dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* weights,
                                  const void* slope, void* dx, int64_t lddx, float* dw, float* db, int32_t accumulate, int32_t M,
                                  int32_t K, int32_t N, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int dt;
  hpf_status st = linear_shape(dtype, M, K, N, dt);
  if (st != HPF_OK) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  if (!words_aligned(dw, db)) return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if (M == 0) {
    if (accumulate) return HPF_OK;
    hipError_t e = dw ? launch_zero_f32(dw, (size_t)K * N, s) : hipSuccess;
    if (e == hipSuccess && db) e = launch_zero_f32(db, (size_t)N, s);
    return launched(e);
  }
  if (!dx && !dw && !db) return HPF_OK;
  if (!dy || (dx && !weights) || (dw && !x)) return fail(HPF_EINVAL, "null tensor");
  if (!rows_ok(lddy, N) || (dw && !rows_ok(ldx, K)) || (dx && !rows_ok(lddx, K))) return fail(HPF_EINVAL, "row stride shorter than a row");
  if (!element_aligned(dy, dt) || !element_aligned(x, dt) || !element_aligned(dx, dt) || !element_aligned(slope, dt) ||
      (dt == DT_F32 && !element_aligned(weights, dt)))
    return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if (dx && dt == DT_BF16 && (uintptr_t)weights % 256) return fail(HPF_EINVAL, "packed weights must be 256-byte aligned");
  const size_t e = elem(dt), need = linear_workspace_bytes(dt, M, K, N);
  const Matrix in[] = {{dy, M, N, lddy, e}, {dw ? x : nullptr, M, K, ldx, e}, {slope, M, N, N, e}, weights_of(dt, dx ? weights : nullptr, K, N)};
  const Matrix out[] = {{dx, M, K, lddx, e}, words(dw, (int64_t)K * N), words(db, N)};
  if (collide(out, in)) return fail(HPF_EINVAL, "an output overlaps another tensor");
  st = workspace_ok(workspace, workspace_bytes, need);
  if (st != HPF_OK) return st;
  if (!workspace_apart(workspace, need, in) || !workspace_apart(workspace, need, out)) return fail(HPF_EINVAL, "the workspace overlaps a tensor");
  const LinearBackward a{dy, lddy, x, ldx, weights, slope, dx, lddx, dw, db, accumulate, M, K, N};
  return launched(launch_linear_backward(dt, a, workspace, s));
}

static hpf_status logits_shape(hpf_dtype dtype, const void* logits, int64_t ld, int32_t top, int32_t rows, int32_t classes, int& dt) {
  if (!type_of(dtype, dt)) return fail(HPF_EINVAL, "unknown dtype");
  if (rows < 0 || classes < 1) return fail(HPF_EINVAL, "rows must not be negative, classes must be positive (%d, %d)", rows, classes);
  if (rows > (1 << 21) || classes > MAX_CLASSES || (int64_t)rows * classes > (int64_t)1 << 36)
    return fail(HPF_EUNSUPPORTED, "more than 2^21 rows, 2^28 classes or 2^36 logits (%d, %d)", rows, classes);
  if (top < 0) return fail(HPF_EINVAL, "negative list length");
  if (top > TOP_MAX) return fail(HPF_EUNSUPPORTED, "a list of %d entries, at most %d", top, TOP_MAX);
  if (rows == 0) return HPF_OK;
  if (!logits) return fail(HPF_EINVAL, "null logits");
  if (!rows_ok(ld, classes)) return fail(HPF_EINVAL, "row stride shorter than a row");
  if (!element_aligned(logits, dt)) return fail(HPF_EINVAL, "logits not aligned to their elements");
  return HPF_OK;
}

size_t hpf_op_logits_workspace_bytes(hpf_dtype dtype, int32_t rows, int32_t classes, int32_t top) {
  int dt;
  if (!type_of(dtype, dt) || rows < 1 || rows > (1 << 21) || classes < 1 || classes > MAX_CLASSES || top < 0 || top > TOP_MAX) return 0;
  return logits_workspace_bytes(dt, rows, classes, top);
}

hpf_status hpf_op_logprob_forward(hpf_dtype dtype, const void* logits, int64_t ld, const int32_t* labels, float* logprob,
                                  float* entropy, int32_t* rank, float* stats, int32_t* top_index, float* top_logprob, int32_t top,
                                  int32_t rows, int32_t classes, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int dt;
  hpf_status st = logits_shape(dtype, logits, ld, top, rows, classes, dt);
  if (st != HPF_OK) return st;
  if (rows == 0) return HPF_OK;
  if (top && (!top_index || !top_logprob)) return fail(HPF_EINVAL, "top_index and top_logprob are required with a list");
  if (!words_aligned(labels, logprob, entropy, rank, stats, top_index, top_logprob)) return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if ((logprob || rank) && !labels) return fail(HPF_EINVAL, "labels are required for logprob and rank");
  const Matrix in[] = {{logits, rows, classes, ld, elem(dt)}, words(labels, rows)};
  const int64_t entries = (int64_t)rows * top;
  const Matrix out[] = {words(logprob, rows), words(entropy, rows), words(rank, rows), words(stats, 2 * (int64_t)rows), words(top ? top_index : nullptr, entries),
                        words(top ? top_logprob : nullptr, entries)};
  if (collide(out, in)) return fail(HPF_EINVAL, "an output overlaps another tensor");
  const size_t need = logits_workspace_bytes(dt, rows, classes, top);
  st = workspace_ok(workspace, workspace_bytes, need);
  if (st != HPF_OK) return st;
  if (!workspace_apart(workspace, need, in) || !workspace_apart(workspace, need, out)) return fail(HPF_EINVAL, "the workspace overlaps a tensor");
  const LogprobForward a{logits, ld, labels, logprob, entropy, rank, stats, top_index, top_logprob, top, rows, classes};
  return launched(launch_logprob_forward(dt, a, workspace, (hipStream_t)hip_stream));
}

hpf_status hpf_op_logprob_backward(hpf_dtype dtype, const void* logits, int64_t ld, const int32_t* labels, const float* stats,
                                   const float* grad_logprob, const float* entropy, const float* grad_entropy, void* dlogits,
                                   int64_t ldd, int32_t rows, int32_t classes, void* hip_stream) {
  int dt;
  hpf_status st = logits_shape(dtype, logits, ld, 0, rows, classes, dt);
  if (st != HPF_OK) return st;
  if (rows == 0) return HPF_OK;
  if (rows * logprob_backward_pieces(elem(dt), classes) > LOGPROB_BACKWARD_MOST)
    return fail(HPF_EUNSUPPORTED, "a gradient of 2^24 pieces of 16 KiB or more (%d rows of %d classes)", rows, classes);
  if (!stats || !dlogits) return fail(HPF_EINVAL, "stats and dlogits are required");
  if (grad_logprob && !labels) return fail(HPF_EINVAL, "labels are required with grad_logprob");
  if (grad_entropy && !entropy) return fail(HPF_EINVAL, "entropy is required with grad_entropy");
  if (!rows_ok(ldd, classes)) return fail(HPF_EINVAL, "row stride shorter than a row");
  if (!element_aligned(dlogits, dt)) return fail(HPF_EINVAL, "dlogits not aligned to their elements");
  if (!words_aligned(labels, stats, grad_logprob, entropy, grad_entropy)) return fail(HPF_EINVAL, "tensor not aligned to its elements");
  if (overlap(Matrix{logits, rows, classes, ld, elem(dt)}, Matrix{dlogits, rows, classes, ldd, elem(dt)}) && (logits != dlogits || ld != ldd))
    return fail(HPF_EINVAL, "dlogits overlap the logits (they may be the same tensor)");
  const Matrix in[] = {words(grad_logprob ? labels : nullptr, rows), words(stats, 2 * (int64_t)rows), words(grad_logprob, rows),
                       words(grad_entropy ? entropy : nullptr, rows), words(grad_entropy, rows)};
  const Matrix out[] = {{dlogits, rows, classes, ldd, elem(dt)}};
  if (collide(out, in)) return fail(HPF_EINVAL, "dlogits overlap another tensor (only the logits may be the same)");
  const LogprobBackward a{logits, ld, labels, stats, grad_logprob, entropy, grad_entropy, dlogits, ldd, rows, classes};
  return launched(launch_logprob_backward(dt, a, (hipStream_t)hip_stream));
}

hpf_status hpf_op_distill(hpf_dtype dtype, const void* logits, int64_t ld, const int32_t* top_index, const float* top_logit,
                          int32_t top, const int32_t* labels, float temperature, float hard_weight, const float* row_weight,
                          float* loss, void* dlogits, int64_t ldd, int32_t rows, int32_t classes, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  int dt;
  hpf_status st = logits_shape(dtype, logits, ld, top, rows, classes, dt);
  if (st != HPF_OK) return st;
  if (!(temperature >= 1e-4f && temperature <= 1e4f)) return fail(HPF_EINVAL, "temperature %g outside [1e-4, 1e4]", (double)temperature);
  if (!(hard_weight >= 0.f && hard_weight <= 1.f)) return fail(HPF_EINVAL, "hard_weight %g outside [0, 1]", (double)hard_weight);
  if (rows == 0) return HPF_OK;
  if (!loss) return fail(HPF_EINVAL, "null loss");
  if (top && (!top_index || !top_logit)) return fail(HPF_EINVAL, "top_index and top_logit are required with a list");
  if (hard_weight > 0.f && !labels) return fail(HPF_EINVAL, "labels are required with hard_weight > 0");
  if (dlogits && !rows_ok(ldd, classes)) return fail(HPF_EINVAL, "row stride shorter than a row");
  if (!element_aligned(dlogits, dt)) return fail(HPF_EINVAL, "dlogits not aligned to their elements");
  if (!words_aligned(top_index, top_logit, labels, row_weight, loss)) return fail(HPF_EINVAL, "tensor not aligned to its elements");
  const int64_t entries = (int64_t)rows * top;
  const Matrix in[] = {{logits, rows, classes, ld, elem(dt)}, words(top ? top_index : nullptr, entries), words(top ? top_logit : nullptr, entries),
                       words(labels, rows), words(row_weight, rows)};
  const Matrix out[] = {words(loss, rows), {dlogits, rows, classes, ldd, elem(dt)}};
  if (collide(out, in)) return fail(HPF_EINVAL, "an output overlaps another tensor");
  const size_t need = logits_workspace_bytes(dt, rows, classes, top);
  st = workspace_ok(workspace, workspace_bytes, need);
  if (st != HPF_OK) return st;
  if (!workspace_apart(workspace, need, in) || !workspace_apart(workspace, need, out)) return fail(HPF_EINVAL, "the workspace overlaps a tensor");
  const Distill a{logits, ld, top_index, top_logit, labels, row_weight, loss, dlogits, ldd, temperature, hard_weight, top, rows, classes};
  return launched(launch_distill(dt, a, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
