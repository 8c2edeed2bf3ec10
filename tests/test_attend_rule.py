"""The form that md_attend_cache's estimate takes for a launch, and its split of the rows (no GPU needed)."""
import os
import random
import shutil
import subprocess

import pytest

from tests.attend_forms import FORMS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ALL = (1 << 31) - 1


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    """Runs the library's rule on launches: kind, layers, KV heads, workspace, tokens, window, sinks."""
    nvcc = shutil.which("nvcc") or pytest.skip("no nvcc")
    exe = str(tmp_path_factory.mktemp("rule") / "attend_rule")
    r = subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-O1", "--expt-relaxed-constexpr", "-I",
                        os.path.join(ROOT, "include"), "-o", exe, os.path.join(ROOT, "tests", "c", "attend_rule.cu")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(launches):
        lines = [" ".join(map(str, (int(k == "e4m3"), L, h, w, s, ws, len(n), *n))) for k, L, h, ws, n, w, s in launches]
        r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r                       # 2, 3: the parts do not fit their places; 4: a warp for a part
        return [tuple(map(int, x.split())) for x in r.stdout.splitlines()]

    return ask


def test_the_shapes_of_the_gpu_tests_take_their_forms(rule):
    got = rule([f[:5] + (ALL, 0) for f in FORMS])
    assert [(c, w, p > 1) for c, w, p in got] == [f[5] for f in FORMS]


def test_any_launch_has_a_form_and_its_parts_have_places(rule):
    """From one token to the largest batch and the longest sequence, all empty, with windows: rows are split
    only with a workspace, and the parts fit it."""
    r = random.Random(3)
    launches = [("e4m3", 255, 64, 1, [1 << 18] * 256, ALL, 0), ("bf16", 1, 1, 1, [1 << 18], ALL, 0), ("e4m3", 1, 1, 1, [0], ALL, 0),
                ("bf16", 36, 8, 1, [0] * 256, ALL, 5), ("e4m3", 1, 1, 1, [1 << 18], 0, 0), ("e4m3", 1, 1, 1, [1 << 18], 0, 1 << 18),
                ("e4m3", 255, 1024, 0, [1 << 18] * 256, ALL, 0), ("e4m3", 1, 1, 1, [1 << 18] + [1] * 255, ALL, 0)]
    for _ in range(3000):
        n = [r.choice((0, 1, int(2 ** r.uniform(0, 18)), int(2 ** r.uniform(0, 12)))) for _ in range(r.choice((1, 1, 2, 5, 17, 64, 256)))]
        launches.append((r.choice(("e4m3", "bf16")), r.choice((1, 2, 36, 255)), r.choice((1, 2, 8, 40)), r.choice((0, 1)), n,
                         r.choice((ALL, ALL, 0, 1, 100, 5000)), r.choice((0, 0, 4, 1000, 1 << 20))))
    for launch, (C, warps, parts) in zip(launches, rule(launches)):
        assert C in (0, 1, 2, 4, 8, 16) and warps in (4, 8) and 1 <= parts <= 32 and (parts == 1 or launch[3]), launch
