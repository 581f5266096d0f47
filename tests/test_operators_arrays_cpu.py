"""Which arrays the operators' entry points take together, which needs no GPU: calls
that they refuse return before anything is launched, and the rule itself
(csrc_ops/ops_common.h) is checked against sets of bytes."""

import itertools
import os
import subprocess

import pytest

from paper_1902_06714_amd import build, nf

from .test_operators_cpu import E, GRAD, LOGP, MUON, ORTH, P, S, TRAIN, _call

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# d_out over d_x with another pitch or stride, shifted, or a stack that begins at its one input
@pytest.mark.parametrize("change", [
    {"x": P, "out": P, "ld": 9},                                                    # the rows move
    {"x": P, "out": P + 4}, {"x": P + 32, "out": P}, {"x": P, "out": P + 4 * 48},    # shifted
    {"x": P, "out": P, "stride": 0},                                                # one input of a stack
    {"x": P, "out": P, "stride": 49},
    {"x": P, "out": P + 4 * 4, "ld": 16, "ldo": 16, "stride": 96, "so": 96},         # half of the columns
    {"x": P, "out": P + 4 * 8, "ld": 16, "ldo": 17, "stride": 96, "so": 102},
    {"x": P, "out": P, "count": 1, "rows": 40, "cols": 70, "ld": 77, "ldo": 70},
    {"x": P, "out": P, "count": 1, "rows": 300, "cols": 400, "ld": 410, "ldo": 400}])
def test_orthogonalize_refuses_a_result_over_its_matrices(change):
    assert _call("nf_orthogonalize", ORTH, change) == E, nf.nf_last_error()
    assert "overlaps" in nf.nf_last_error()


@pytest.mark.parametrize("change", [
    {"so": 7, "ldo": 40}, {"so": 20, "ldo": 27}, {"so": 0, "ldo": 40}, {"so": -8, "ldo": 40}, {"so": 13, "ldo": 40, "count": 4},
    {"so": 47, "count": 3}])
def test_orthogonalize_refuses_results_over_one_another(change):
    assert _call("nf_orthogonalize", ORTH, {"out": 99 * P, **change}) == S, nf.nf_last_error()
    assert "overlap" in nf.nf_last_error()


# new weights shifted on the gradient, or in its place with fp32 for bf16
@pytest.mark.parametrize("change", [
    {"wo": 3 * P + 4}, {"wo": 3 * P - 32}, {"wo": 3 * P, "gd": nf.NF_BF16}, {"wo": 3 * P - 128, "gd": nf.NF_BF16},
    {"wo": 3 * P + 400, "rows": 100, "cols": 120}])
def test_muon_step_refuses_new_weights_over_the_gradient(change):
    assert _call("nf_muon_step", MUON, change) == E, nf.nf_last_error()
    assert "gradient" in nf.nf_last_error()


# each array of a call on its own, a megabyte from the next
APART = {name: {k: (i + 1) * P for i, k in enumerate(k for k in base if base[k] in (P, 2 * P))}
         for name, base in (("nf_logprobs", LOGP), ("nf_logprobs_train", TRAIN), ("nf_logprobs_grad", GRAD))}


@pytest.mark.parametrize("name,base,out,inputs", [
    ("nf_logprobs", LOGP, ("logp", "ent", "stat", "ids", "alt"), ("x", "t")),
    ("nf_logprobs_train", TRAIN, ("logp", "ent", "stat"), ("x", "t", "g", "h")),
    ("nf_logprobs_train", TRAIN, ("dx",), ("t", "g", "h", "logp", "ent", "stat")),
    ("nf_logprobs_grad", GRAD, ("dx",), ("t", "stat", "ent", "g", "h"))])
def test_logprobs_refuse_outputs_over_their_inputs(name, base, out, inputs):
    apart = APART[name]
    for o, i in itertools.product(out, inputs):
        assert _call(name, base, {**apart, o: apart[i] + 8}) == E, (o, i, nf.nf_last_error())
        assert "overlaps" in nf.nf_last_error(), (o, i)


def test_workspaces_of_sizes_that_are_refused():
    lib = nf.raw()
    for rows, classes, top in ((1 << 31, 10, 0), (1 << 40, 131072, 5), (4, 6, 7), (0, 6, 7), (1, (1 << 30) + 1, 0)):
        assert lib.nf_logprobs_work(nf.NF_F32, rows, classes, top, 0) == -1 and nf.nf_last_error() != ""
        with pytest.raises(nf.NfError):
            nf.nf_logprobs_work(nf.NF_F32, rows, classes, top)
    assert lib.nf_logprobs_work(nf.NF_F32, 1 << 31, 10, 0, 1) == -1
    assert lib.nf_logprobs_work(nf.NF_F32, (1 << 31) - 1, 10, 10, 0) == 0
    assert lib.nf_logprobs_work(nf.NF_F32, 4, 6, 0, 1) == 0


RULE = r"""
#include <cstdio>
#include "ops_common.h"
int main() {
  long long v[2][6];
  for (;;) {
    for (auto& r : v)
      for (auto& x : r)
        if (std::scanf("%lld", &x) != 1) return 0;
    auto of = [](const long long* q) {
      return nf::OpArray{reinterpret_cast<const void*>(q[0]), q[1], q[2], q[3], q[4], q[5]};
    };
    std::printf("%d %d\n", (int)nf::op_share(of(v[0]), of(v[1])), (int)nf::op_same(of(v[0]), of(v[1])));
  }
}
"""


def _bytes(p, count, stride, rows, pitch, width):
    return {p + k * stride + r * pitch + c for k in range(count) for r in range(rows) for c in range(width)}


def _program(d, text):
    """A host program of the operators' sources: lines of numbers in, lines of numbers out."""
    (d / "rule.hip").write_text(text)
    subprocess.run([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                    "-I", build.CSRC, "-I", build.OPS, str(d / "rule.hip"), "-o", str(d / "rule")], check=True)

    def ask(lines):
        text = "\n".join(" ".join(str(v) for v in line) for line in lines)
        out = subprocess.run([str(d / "rule")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    ask = _program(tmp_path_factory.mktemp("rule"), RULE)
    return lambda pairs: ask([a + b for a, b in pairs])


def test_arrays_that_share_bytes_are_found(rule):
    """No two arrays with a common byte pass, and those that lie side by side in a
    buffer's rows, or by turns in a stack, do."""
    firsts = [(1000, c, s, r, p, w) for c, s in ((1, 0), (2, 0), (2, 64), (3, 70), (3, 64)) for r in (1, 3) for p in (8, 16)
              for w in (3, 8)]
    pairs = [((q, *a[1:]), (1000 + off, *b[1:])) for a, b in itertools.product(firsts, firsts)
             for off, q in ((-20, 1000), (0, 1000), (3, 1000), (4, 1000), (8, 1000), (24, 1000), (32, 1000), (200, 1000))]
    for (a, b), (share, same) in zip(pairs, rule(pairs)):
        common = _bytes(*a) & _bytes(*b)
        assert share or not common, (a, b)
        if same:
            assert _bytes(*a) == _bytes(*b), (a, b)
    apart = [((1000, 1, 0, 9, 32, 16), (1016, 1, 0, 9, 32, 16)),           # halves of rows
             ((1016, 1, 0, 9, 32, 16), (1000, 1, 0, 4, 32, 16)),
             ((1000, 4, 320, 5, 32, 12), (1012, 4, 640, 5, 32, 20)),       # of a stack's rows
             ((1000, 4, 320, 10, 16, 16), (1160, 4, 320, 10, 16, 16)),     # matrices by turns
             ((1000, 4, 64, 1, 7, 32), (1032, 4, 64, 1, 9, 32)),
             ((1000, 1, 0, 9, 100, 20), (1020, 1, 0, 1, 0, 80)),           # between two rows
             ((1340, 1, 0, 2, 8, 4), (1000, 2, 500, 5, 100, 40)),
             ((1000, 1, 0, 2, 50, 50), (1100, 1, 0, 2, 60, 50))]
    assert all(r == (0, 0) for r in rule(apart))
    one = (1000, 1, 5, 1, 99, 16)
    assert rule([(one, (1000, 1, 7, 1, 16, 16))]) == [(1, 1)]


LAUNCHES = r"""
#include <cstdio>
#include "ops_common.h"
int main() {
  long long rows, block, per_block, per_row;
  while (std::scanf("%lld %lld %lld %lld", &rows, &block, &per_block, &per_row) == 4) {
    long long next = 0, launches = 0, most = 0;
    const hipError_t e = nf::op_each_launch(rows, block, per_block, per_row, [&](int64_t first, int64_t n) {
      if (first != next || n < 1) return hipErrorInvalidValue;
      next += n;
      ++launches;
      const long long threads = ((n * per_row + per_block - 1) / per_block + 7) / 8 * 8 * block;
      if (threads > most) most = threads;
      return hipSuccess;
    });
    std::printf("%d %lld %lld %d\n", (int)(e == hipSuccess), next, launches, (int)(most < (1ll << 32)));
  }
}
"""


def test_rows_past_a_grid_take_several_launches(tmp_path):
    """Rows up to 2^31 - 1 by every kernel's workgroups: whole, in order, each grid below
    2^32 threads, and one launch where one holds them."""
    ways = [(256, 32, 1), (256, 4, 1), (64, 1, 1), (256, 1, 1), (512, 1, 1), (1024, 1, 1), (256, 1, 3), (256, 1, 1 << 19),
            (512, 1, 1024)]
    asked = [(rows, *w) for rows in (1, 1000, (1 << 22) - 8, 1 << 22, 1 << 24, (1 << 26) + 9, (1 << 31) - 1) for w in ways]
    for (rows, block, per_block, per_row), got in zip(asked, _program(tmp_path, LAUNCHES)(asked)):
        assert got[0] == 1 and got[1] == rows and got[3] == 1, (rows, block, per_block, per_row, got)
        blocks = (rows * per_row + per_block - 1) // per_block
        if (blocks + 8 * per_row) * block < 1 << 32:
            assert got[2] == 1, (rows, block, per_block, per_row, got)
