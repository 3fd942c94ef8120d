"""The GPU parity tests of the E4M3 products reach every kernel form that the library's choice gives to a call: the choice
(host code) is compiled alone and asked for each of the tests' sizes, with the 256 CUs of the device. And the kernels of
these forms, like the gates', keep their state in registers."""
import os
import re
import shutil
import subprocess

import pytest

import test_gpu_fp8 as t
from test_built_code import READELF, objects  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["split12", "split22", "split24", "split44", "low", "deep", "mid", "big"]
CUS, B = 256, 128

MAIN = """
#include <cstdio>
#include "xs_gemm_fp8_form.hpp"
int main() {
  int M, N, K, n, swiglu, f32;
  while (scanf("%d %d %d %d %d %d", &M, &N, &K, &n, &swiglu, &f32) == 6)
    printf("%d\\n", static_cast<int>(xs::f8::choose_form(CUS, M, N, K, (K / 128 + 3) / 4 * 4, n, swiglu, f32)));
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("forms")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run([gxx, "-std=c++17", f"-DCUS={CUS}", "-I", os.path.join(ROOT, "paper_2607_23264_amd", "csrc"), "-o", str(d / "main"),
                    str(d / "main.cpp")], check=True)

    def ask(calls):
        text = "\n".join(" ".join(map(str, c)) for c in calls)
        out = subprocess.run([str(d / "main")], input=text, text=True, capture_output=True, check=True).stdout.split()
        assert len(out) == len(calls)
        return [NAMES[int(i)] for i in out]
    return ask


def test_plain_products_of_every_form(forms):
    sizes = t.GEMMS + t.FORM_GEMMS
    assert set(forms([(*s, 0, 0, 1) for s in sizes])) == {"split12", "split22", "split24", "split44", "mid"}
    tiles = [(M, N, b * B) for M, N, b in t.test_gemm_of_about_a_tile_to_a_cu.pytestmark[1].args[1]]
    assert set(forms([(*s, 0, 0, 0) for s in sizes + tiles + t.LARGE_GEMMS])) == set(NAMES)
    assert set(forms([(*s, 0, 0, 0) for s in t.LARGE_GEMMS])) == {"big"}
    # more than a tile to a workgroup, and more than the eight row blocks of a group of tiles
    assert any(-(-M // 256) * -(-N // 256) > CUS and M > 8 * 256 for M, N, _ in t.LARGE_GEMMS)


def test_grouped_products_of_every_form(forms):
    calls = [(t.large_layout(rows)[1], N, K, len(rows)) for rows, N, K in t.LARGE_GROUPS]
    store, swiglu = forms([(*c, 0, 0) for c in calls]), forms([(*c, 1, 0) for c in calls])
    small = [(sum(rows) + 2 * len(rows), N, K, len(rows), int(epi == "swiglu"), 0) for rows in t.SEGMENTS
             for N, K, epi in t.test_grouped_gemm.pytestmark[0].args[1]]
    of = dict(zip(small, forms(small)))
    assert set(store) | {f for c, f in of.items() if not c[4]} == set(NAMES)
    assert set(swiglu) | {f for c, f in of.items() if c[4]} == set(NAMES)
    assert {"big", "deep", "mid"} <= set(store) and {"big", "deep", "mid"} <= set(swiglu)
    assert any(f == "big" and sum(-(-r // 256) for r in rows) * -(-N // 256) > CUS
               for (rows, N, _), f in zip(t.LARGE_GROUPS, store))


def test_overlapping_segments_in_split_forms_and_tiles(forms):
    cases = t.test_overlapping_segments_compute_all_their_rows.pytestmark[1].args[1]
    got = forms([(max(o + r for o, r in spans) + 3, N, K, len(spans), 0, 0) for spans, N, K in cases])
    assert {f[:5] for f in got} >= {"split"} and set(got) & {"low", "deep", "mid", "big"}
    assert any(f.startswith("split") and len(c[0]) > 64 for f, c in zip(got, cases))


def test_the_kernels_stay_in_registers(objects):  # noqa: F811
    """Spilled vector registers: only the 256-tile's, where 256 registers hold the sums and scales by rows or SwiGLU's halves
    come on top, and no more of them than what the forms' measured times contain."""
    spills = {}
    for path in objects:
        r = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True)
        names = re.findall(r"^\s+\.name:\s+(_Z\w+)$", r.stdout, flags=re.M)
        counts = re.findall(r"^\s+\.vgpr_spill_count:\s+(\d+)$", r.stdout, flags=re.M)
        assert len(names) == len(counts)
        spills.update((n, int(c)) for n, c in zip(names, counts) if "N2xs2f8" in n or "gate_" in n)
    assert len(spills) > 100
    big = "4TileILi256ELi256ELi2ELi4ELi2EEE"
    allowed = {big + "Lb1ELb0ELb0E": 9, big + "Lb0ELb1ELb0E": 2}
    for name, n in spills.items():
        assert n <= max([v for k, v in allowed.items() if k in name], default=0), name
