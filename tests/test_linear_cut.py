"""No-GPU checks of how the products are cut and of the workspace they ask for: the rules of csrc/hpf_linear_cut.h, compiled for the host, walked
over the documented range, and the sizes that the library gives."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1911_05146_amd", "csrc")

COMMON = r'''
#include <cstdio>
#include <initializer_list>
#include <cstddef>
#include "hpf_linear_cut.h"
using namespace hpf;
// The last byte that a launch with this cut writes behind `slabs`, and whether its shares cover the contraction: `k` steps
inline size_t end_of(const Cut& c, int M, int N) { return c.splits > 1 ? (size_t)c.splits * M * slab_row(N) * sizeof(float) : 0; }
inline bool covers(const Cut& c, int K) {
  const int unit = c.kind == CUT_FEW ? 32 : 64, k = (K + unit - 1) / unit;
  return c.splits >= 1 && c.steps >= 1 && (long)c.splits * c.steps >= k && (c.splits == 1 || (long)(c.splits - 1) * c.steps <= k);
}
inline long checked = 0, bad = 0;
inline void look(int M, int K, int N) {
  const ForwardSpace f(M, K, N);
  const BackwardSpace b(M, K, N);
  // a product's operand is read in place, with the contraction as it is, or from a copy whose rows are rounded up to 64
  const int Ks[2] = {K, round_up64(K)}, Ns[2] = {N, round_up64(N)};
  const char* what = nullptr;
  for (int i = 0; i < 2; ++i) {
    const Cut y = cut_of(M, N, Ks[i], false), dx = cut_of(M, K, Ns[i], false);
    if (f.slabs + end_of(y, M, N) > f.bytes) what = "forward";
    if (b.slabs + end_of(dx, M, K) > b.bytes) what = "dx";
    if (!covers(y, Ks[i]) || !covers(dx, Ns[i])) what = "shares";
  }
  const Cut dw = cut_of(K, N, M, true);
  if (b.slabs + end_of(dw, K, N) > b.bytes) what = "dw";
  if (!covers(dw, M)) what = "shares of dw";
  if (f.slabs < (size_t)M * round_up64(K) * 2) what = "copy of x";
  if (b.x < (size_t)M * round_up64(N) * 2 || b.sums < b.x + (size_t)M * round_up64(K) * 2 || b.slabs < b.sums + (size_t)b.groups * N * 4) what = "regions";
  if ((f.slabs | f.bytes | b.x | b.sums | b.slabs | b.bytes) & 255) what = "alignment";
  ++checked;
  if (what && bad++ < 20) std::printf("%d x %d x %d: %s\n", M, K, N, what);
}
'''


def run_cpp(tmp_path, source):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(COMMON + source)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout.split()


def test_no_product_writes_behind_its_workspace(tmp_path):
    """Few rows and long contractions of every remainder, where the number of shares is not monotonic in the contraction; then sizes spread over
    the documented range."""
    out = run_cpp(tmp_path, r'''
int main() {
  for (int M : {1, 2, 5, 15, 16, 17})
    for (int N = 1; N <= 160; N += N < 40 ? 13 : 1)
      for (int K = 8; K < 200000; K += 8 * (1 + (K / 8) % 3)) { look(M, K, N); if (M < 3) look(M, N, K); }
  unsigned long long r = 88172645463325252ull;
  auto below = [&](int bits) {       // spread over the logarithm
    r ^= r << 13; r ^= r >> 7; r ^= r << 17;
    const int b = (int)(r % (bits + 1));
    return (int)(1 + (r >> 20) % (1ull << b));
  };
  for (int i = 0; i < 2000000; ++i) {
    const int M = below(21), K = below(20), N = below(20);
    if ((long)M * N <= 1l << 32 && (long)M * K <= 1l << 32 && (long)K * N <= 1l << 32) look(M, K, N);
  }
  for (int M : {1, 16, 17, 1 << 21}) for (int K : {1, 1 << 10, 1 << 20}) for (int N : {1, 1 << 11, 1 << 20})
    if ((long)M * N <= 1l << 32 && (long)M * K <= 1l << 32 && (long)K * N <= 1l << 32) look(M, K, N);
  std::printf("%ld\n", checked);
  return bad != 0;
}
''')
    assert int(out[0]) > 3_000_000


SIZES = [(16, 89760, 40), (16, 89760, 48), (1, 53856, 65), (5, 53856, 65), (1, 40, 89760), (16, 40, 89760), (1, 1, 1), (16, 4096, 4096), (128, 4096, 4096),
         (1021, 2049, 1000), (2560, 4096, 4096)]


def test_the_library_asks_for_what_these_rules_say(tmp_path):
    from paper_1911_05146_amd import hpf
    out = run_cpp(tmp_path, "int main() {\n" + "".join(
        "  { const size_t f = ForwardSpace(%d, %d, %d).bytes, b = BackwardSpace(%d, %d, %d).bytes; std::printf(\"%%zu\\n\", f > b ? f : b); }\n" % (s + s) for s in SIZES) + "}\n")
    assert [int(v) for v in out] == [hpf.hpf_op_linear_workspace_bytes(hpf.HPF_BF16, *s) for s in SIZES]


@pytest.mark.parametrize("M,K,N", [(16, 89760, 40), (16, 89760, 48), (1, 53856, 65)])
def test_a_contraction_is_cut_alike_in_place_and_padded(tmp_path, M, K, N):
    out = run_cpp(tmp_path, "int main() { const Cut a = cut_of(%d, %d, %d, false), b = cut_of(%d, %d, round_up64(%d), false);\n"
                  "  std::printf(\"%%d %%d %%d\\n%%d %%d %%d\\n\", a.kind, a.splits, a.steps, b.kind, b.splits, b.steps); }" % (M, N, K, M, N, K))
    assert out[:3] == out[3:]
