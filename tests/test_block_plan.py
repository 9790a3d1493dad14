"""How residual borders share out their rows, and what products in 4 bits launch (no GPU needed)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "block_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "block_plan.cpp"), "-o", exe], check=True)

    def ask(units, products):
        text = "".join("%d %d %d %d\n" % c for c in units) + "0 0 0 0\n" + "".join("%d %d %d %d\n" % c for c in products)
        return subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    return ask


def test_every_row_belongs_to_one_unit(plans):
    calls = []
    for n in (1, 64, 65, 300, 512, 1000, 2048, 4096, 4097, 16384):
        for m in (0, 1, 2, 3, 255, 256, 257, 512, 513, 1000, 1024, 4097, 16384, 100003):
            calls.append((m, n, 0, 1))
            calls += [(m, n, 1, div) for div in {1, 2, 3, 7, 64, 100, 1024, m} if div and m % div == 0]
    calls += [(1 << 30, n, 1, div) for n in (8, 16384) for div in (1, 2, 1 << 20, 1 << 30)]
    said = plans(calls, [])
    assert len(said) == len(calls)
    assert [(c, s) for c, s in zip(calls, said) if not s.startswith("ok")] == []


def test_products_launch_what_their_kernels_assume(plans):
    calls = [(codes, m, n, k) for codes in (0, 1) for m in (1, 2, 16, 17, 32, 33, 64, 65, 300, 1000, 8192, (1 << 31) - 2000)
             for n in (1, 16, 100, 1024, 8192, 1 << 26, (1 << 26) + 1, 1 << 27) for k in (1, 128, 129, 1000, 8192, 1 << 24)
             if -(-m // 128) * -(-n // 128) <= 1 << 20]
    said = plans([], calls)
    assert len(said) == len(calls)
    assert [(c, s) for c, s in zip(calls, said) if not s.startswith("ok")] == []
    kinds = {s.split()[1] for s in said}
    assert kinds == {"0", "1", "2", "3"} and {s.split()[2] for s in said} == {"0", "1"} and len({s.split()[3] for s in said}) > 3
