"""Which kernels some tests on the GPU take (CPU only): the library's own
plan for their sizes, so that a change of its rules cannot take a kernel out of the tests
unnoticed."""
import os
import subprocess

import pytest

from paper_2506_12035_amd import build

import test_gpu_paged_append_many as appends
import test_gpu_paged_joins as joins
import test_gpu_paged_many_rows as many
import test_gpu_paged_window_limits as limits
from test_abi_paged import built_library  # noqa: F401

LOOK = {"all": 0, "window": 2, "tree": 3}
PROGRAM = r"""
#include <cstdio>
#include "marche_internal.h"
using namespace marche;
int main(int argc, char **) {
  if (argc > 1) {  // appends
    int f32, dh, rows, q_heads, heads;
    while (std::scanf("%d %d %d %d %d", &f32, &dh, &rows, &q_heads, &heads) == 5) {
      const PagedAppendPlan p = paged_append_plan(f32 ? DType::F32 : DType::BF16, dh, rows, q_heads, heads);
      std::printf("%d %d\n", p.heads, (int)p.stream);
    }
    return 0;
  }
  int f32, bits8, dh, seqs, total, most, heads, group, len, look, window, sinks;
  while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d %d", &f32, &bits8, &dh, &seqs, &total, &most, &heads, &group, &len, &look, &window,
                    &sinks) == 12) {
    PagedAttnArgs a{};
    a.n_pages = 1 << 20;
    a.n_heads = heads;
    a.page_log2 = 6;
    a.max_pages = 1 << 20;
    a.n_seqs = seqs;
    a.q_total = total;
    a.q_max = most;
    a.group = group;
    a.len_max = len;
    a.look = look;
    a.bits8 = bits8;
    a.window = window;
    a.sinks = sinks;
    paged_plan(f32 ? DType::F32 : DType::BF16, dh, a);
    std::printf("%d %d %d %d\n", a.row_waves, a.splits, a.budget, paged_join_turns(dh, a));
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory, built_library):  # noqa: F811
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    r = subprocess.run([build.hipcc(), "-std=c++17", "-O1", f"--offload-arch={build.ARCH}", "-x", "hip", "-I", build.CSRC, "-I",
                        os.path.join(build.ROOT, "include"), str(d / "plan.cpp"), "-x", "none", build.LIB,
                        f"-Wl,-rpath,{build.PKG}", "-o", str(d / "plan")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(sizes, *args):
        r = subprocess.run([str(d / "plan"), *args], input=" ".join(map(str, sizes)), capture_output=True, text=True, check=True)
        return list(map(int, r.stdout.split()))
    return run


@pytest.fixture(scope="module")
def plan(program):
    """(dtype, format, dh, seqs, rows in all, rows of a sequence, heads, group, len_max, look, window, sinks) ->
    dict of row_waves, splits, budget, turns (of the join)"""
    def ask(dtype, fmt, dh, seqs, total, most, heads, group, len_max, look, window=1, sinks=0):
        sizes = [int(dtype == "f32"), int(fmt != "bf16"), dh, seqs, total, most, heads, group, len_max, LOOK[look], window, sinks]
        return dict(zip(("row_waves", "splits", "budget", "turns"), program(sizes)))
    return ask


@pytest.mark.parametrize("case", many.by_blocks() + limits.by_blocks(), ids=lambda c: "-".join(str(c[k]) for k in (
    "look", "fmt", "dh", "heads", "most", "group", "len_max", "window")))
def test_many_rows_go_by_blocks(plan, case):
    assert plan(**case)["row_waves"] > 0


@pytest.mark.parametrize("case,many_rows,turns", joins.plans(), ids=[joins._name(c) for c in joins.CASES])
def test_joins_are_reached(plan, case, many_rows, turns):
    p = plan(**case)
    assert (p["row_waves"] > 0, p["splits"] > 1, p["turns"]) == (many_rows, True, turns)


@pytest.mark.parametrize("sizes,heads,stream", appends.plans(), ids=lambda x: "-".join(map(str, x)) if isinstance(x, tuple) else str(x))
def test_appends_take_four_heads(program, sizes, heads, stream):
    assert program([int(sizes[0] == "f32"), *sizes[1:]], "append") == [heads, stream]
