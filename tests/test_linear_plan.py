"""Which kernels the channel products choose, and what their kernels assume of the operands (no GPU needed)."""
import itertools
import os
import subprocess

import pytest

import paper_2204_03643_amd as tv

HERE = os.path.dirname(os.path.abspath(__file__))
# the kernels' kinds, in their order, and the outputs of a workgroup's tile
FEW, TILE256, TILE128, TILE128DEEP, TILE64, SPLIT256, SPLIT128, SPLIT64 = range(8)
TILES = {TILE256: (256, 256), TILE128: (128, 128), TILE128DEEP: (128, 128), TILE64: (64, 128), SPLIT256: (256, 256),
         SPLIT128: (128, 128), SPLIT64: (64, 128)}
DIRECT = (TILE256, TILE128, TILE128DEEP, TILE64)          # bf16 straight from memory to LDS, 32-bit offsets within a tile


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """calls -> for each a dict of its products (y, dx, dw) and workspaces."""
    exe = str(tmp_path_factory.mktemp("plan") / "linear_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "linear_plan.cpp"), "-o", exe], check=True)

    def ask(calls):
        text = "".join("%d %d %d %d %d %d %d %d %d %d %d %d\n" % c for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(calls)
        names = ("kind", "splits", "k_per", "copy_a", "copy_b", "lda", "ldb")
        made = []
        for line in out:
            v = [int(t) for t in line.split()]
            made.append({p: dict(zip(names, v[7 * i:7 * i + 7])) for i, p in enumerate(("y", "dx", "dw"))})
            made[-1]["fwd_bytes"], made[-1]["bwd_bytes"] = v[21:]
        return made
    return ask


def call(m, k, n, dtype=tv.TV_BF16, act=tv.TV_ACT_NONE, x8=0, ldg=None, ldx=None, ldw=None, on16=(1, 1, 1)):
    return (dtype, act, x8, m, k, n, ldg or n, ldx or k, ldw or k) + tuple(on16)


def tiles_fit(a, b):
    return -(-a // 128) * -(-b // 128) <= 1048576


def farthest(rows, ld, tile, transposed):
    """Bytes from a tile's origin to the end of what a lane may load there: a row of the tile and 64 contraction indices,
    or a contraction index of a step and the tile's columns."""
    return ((63 * ld + tile) if transposed else ((min(tile, rows) - 1) * ld + 64)) * 2


@pytest.mark.parametrize("what,act,x8,on16", [("tensors as they are", tv.TV_ACT_NONE, 0, (1, 1, 1)), ("dz", tv.TV_ACT_RELU, 0, (1, 1, 1)),
                                              ("codes", tv.TV_ACT_NONE, 1, (1, 1, 1)), ("copies of all", tv.TV_ACT_NONE, 0, (0, 0, 0)),
                                              ("a copy of x", tv.TV_ACT_GELU, 0, (1, 0, 1)), ("a copy of W", tv.TV_ACT_GELU, 1, (1, 1, 0))])
def test_offsets_within_a_tile_fit_32_bits(plans, what, act, x8, on16):
    """Long rows: of the caller's tensors, of dz, of an input restored from codes, and of copies."""
    small = (1, 8, 20, 64, 250, 1024, 1800)
    large = (1 << 22, (1 << 22) + 8, 8_500_001, 8_500_008, 17_000_000, 36_000_000, 100_000_000)
    shapes = [s for s in itertools.chain(itertools.product(small, small, large), itertools.product(small, large, small),
                                         itertools.product(large, small, small))
              if tiles_fit(s[0], s[2]) and tiles_fit(s[0], s[1]) and tiles_fit(s[1], s[2])]
    calls = [call(m, k, n, act=act, x8=x8, on16=on16) for m, k, n in shapes]
    taken = set()
    for c, p in zip(calls, plans(calls)):
        m, k, n = c[3:6]
        for name, M, N, at, bt in (("y", m, n, False, False), ("dx", m, k, False, True), ("dw", n, k, True, True)):
            q = p[name]
            taken.add(q["kind"])
            if q["kind"] in DIRECT:
                tile = TILES[q["kind"]]
                assert farthest(M, q["lda"], tile[0], at) < 1 << 32, (c, name, q)
                assert farthest(N, q["ldb"], tile[1], bt) < 1 << 32, (c, name, q)
    assert {TILE256, SPLIT64} <= taken


FAKE = 1 << 20


@pytest.mark.parametrize("dtype", (tv.TV_F32, tv.TV_BF16))
@pytest.mark.parametrize("act", (tv.TV_ACT_NONE, tv.TV_ACT_GELU))
def test_workspaces_of_pointers(dtype, act):
    """What is enough everywhere is what the neediest pointers need (or more, where rows cannot all start on 16-byte
    boundaries), and nobody is asked for more than that."""
    size = 2 if dtype == tv.TV_BF16 else 4
    for m, k, n in ((1, 64, 64), (64, 8192, 256), (300, 1001, 777), (8192, 2048, 8192), (4096, 8192, 2048), (0, 8, 8)):
        d = tv.tv_linear_desc(m, k, n, k, k, n, n, dtype, act)
        places = list(itertools.product((FAKE, FAKE + size), repeat=3))
        have = [tv.tv_linear_fwd_workspace_bytes_at(x, w, d) for x, w, _ in places]
        even = k % 8 == 0 and n % 8 == 0
        query = tv.tv_linear_fwd_workspace_bytes(d)
        assert max(have) == query if even else max(have) <= query
        for x8 in (False, True):
            def at(p, dx=FAKE, dw=FAKE, db=FAKE):
                return tv.tv_linear_bwd_workspace_bytes_at(p[0], p[1], FAKE if x8 else None, p[2], dx, dw, db, d)
            have = [at(p) for p in places]
            query = tv.tv_linear_bwd_workspace_bytes(d, x8)
            assert max(have) == query if even else max(have) <= query
            for p in places:
                for wanted in itertools.product((FAKE, None), repeat=3):
                    assert at(p, *wanted) <= at(p)
                assert at(p, None, None, None) == 0


def test_no_workspace_for_copies_that_are_not_made():
    """8192 x 2048 -> 8192 in bf16 on 16-byte boundaries: nothing forward, dz and the column sums' groups backward."""
    m, k, n = 8192, 2048, 8192
    d = tv.tv_linear_desc(m, k, n, k, k, n, n, tv.TV_BF16, tv.TV_ACT_GELU)
    assert tv.tv_linear_fwd_workspace_bytes_at(FAKE, FAKE, d) == 0
    full = tv.tv_linear_bwd_workspace_bytes_at(FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, d)
    assert 2 * m * n < full < 2.1 * m * n
    assert tv.tv_linear_bwd_workspace_bytes_at(FAKE, FAKE, None, FAKE, None, None, FAKE, d) < 1 << 22     # db alone
    bad = tv.tv_linear_desc(m, k, n, k - 1, k, n, n, tv.TV_BF16, tv.TV_ACT_GELU)
    assert tv.tv_linear_fwd_workspace_bytes_at(FAKE, FAKE, bad) == 0
    assert tv.tv_linear_bwd_workspace_bytes_at(FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, bad) == 0


def test_a_call_takes_the_workspace_of_its_pointers():
    """A byte less is refused, before any launch."""
    nothing = tv.tv_held(None, None, tv.TV_HELD_NONE)
    d = tv.tv_linear_desc(64, 8192, 256, 8192, 8192, 256, 256, tv.TV_BF16, tv.TV_ACT_NONE)
    need = tv.tv_linear_fwd_workspace_bytes_at(FAKE, FAKE, d)
    assert need > 0
    assert tv.lib().tv_linear_fwd(FAKE, FAKE, None, None, FAKE, nothing, d, FAKE, need - 1, None) == 5
    d.act = tv.TV_ACT_GELU                                                  # dz has a place of its own
    held = tv.tv_held(FAKE, None, tv.TV_HELD_PLAIN)
    for dx, dw, db in ((FAKE, None, None), (None, FAKE, None), (None, None, FAKE)):
        need = tv.tv_linear_bwd_workspace_bytes_at(FAKE, FAKE + 2, None, FAKE, dx, dw, db, d)
        assert need > 0
        assert tv.lib().tv_linear_bwd(FAKE, FAKE + 2, None, held, FAKE, dx, dw, db, d, FAKE, need - 1, None) == 5


def test_split_sums_of_a_moved_tile_promise_no_alignment(plans):
    """f32 dx of 1001 columns: the last tile starts at column 873 (1001 - 128), and its sums go to the workspace from there on;
    the store must not promise 16 bytes (the hardware takes it, the compiler need not)."""
    (p,) = plans([call(1024, 1001, 1024, dtype=tv.TV_F32)])
    q = p["dx"]
    assert q["splits"] > 1 and (1001 - TILES[q["kind"]][1]) % 4 != 0
    source = open(os.path.join(HERE, "..", "paper_2204_03643_amd", "csrc", "tv_gemm.hpp")).read()
    body = source[source.index("if (g.splits > 1) {"):source.index("if (!whole) {")]
    stores = [line.strip() for line in body.splitlines() if line.strip().startswith(("*(", "put16("))]
    assert stores and all(s.startswith("put16(") for s in stores), stores
