"""The backward call's plan of residual borders for each set of operands and wanted gradients (no GPU needed)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_plans_of_every_set_of_gradients(tmp_path):
    exe = str(tmp_path / "block_wanted_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "block_wanted_plan.cpp"), "-o", exe], check=True)
    calls = [(m, n, shared, div) for n in (8, 100, 512, 2048, 4096, 4097, 8192, 8193, 16384) for m in (1, 6, 600, 16384)
             for shared, div in [(0, 1), (1, 1)] + [(1, d) for d in (2, 3, 100, 600, 1024) if m % d == 0]]
    said = subprocess.run([exe], input="".join("%d %d %d %d\n" % c for c in calls), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(said) == len(calls)
    assert [(c, s) for c, s in zip(calls, said) if not s.startswith("ok")] == []
    assert all(int(s.split()[1]) > 200 for s in said)
