"""The forms that attention's launches take, compiled for the host: the batches that the GPU tests run
reach the forms they are meant for."""
import os
import subprocess

from tests.update_forms import FORMS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_28166_amd", "csrc")

SOURCE = r"""
#include <cstdio>
#include "update_plan.h"
using namespace tandem;
int main() {
  int N, s, nq, nkv, hd, b;
  while (scanf("%d %d %d %d %d %d", &N, &s, &nq, &nkv, &hd, &b) == 6)
    printf("%d %d\n", few_queries(N, s, nq, nkv, hd, b), flash_parts(N, s, nq, nkv, hd, b));
}
"""


def test_batches_reach_their_forms(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    # the GPU tests put 9 rows of no sequence around the batch
    ask = "\n".join(f"{sum(n) + 9} {len(n)} {nq} {nkv} {hd} {int(b)}" for n, nq, nkv, hd, b, _, _ in FORMS.values())
    out = subprocess.run([str(exe)], input=ask, capture_output=True, text=True, check=True).stdout.splitlines()
    got = {name: (line.split()[0] == "1", int(line.split()[1]) > 1) for name, line in zip(FORMS, out)}
    assert len(out) == len(FORMS) and got == {name: f[5:] for name, f in FORMS.items()}
    # every kernel of a type and head size: ordinary and shared keys, whole and in parts
    assert {f[5:] for f in FORMS.values()} == {(a, b) for a in (False, True) for b in (False, True)}
