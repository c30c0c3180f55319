"""Which kernels the orthogonalisation launches for plans of many shapes, against a stand-in for the HIP runtime
(ortho_launches.cpp), without a GPU: what the GPU tests of those plans reach."""
import os
import shutil
import subprocess

import pytest

from ortho_plans import PLANS, name

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_1905_05957_amd")
TYPES = range(3)                                          # fp32, bf16, into the model
G, B, X, LAST = range(4)


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """(one half, matrices, type) -> bytes of the plan's allocation, {(kernel, side, halves, product, output)}, of many at once."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    binary = str(tmp_path_factory.mktemp("launches") / "ortho_launches")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(HERE, "ortho_launches.cpp"), "-o", binary,
                    "-rdynamic", "-L" + PKG, "-lds_hip", "-Wl,--unresolved-symbols=ignore-in-shared-libs",
                    f"-Wl,-rpath,{PKG}:{rocm}/lib"], check=True)

    def run(plans):
        text = "".join("%d %d %d %s\n" % (2 if half else 0, kind, len(mats), " ".join("%d %d" % m for m in mats)) for half, mats, kind in plans)
        r = subprocess.run([binary], input=text, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for block in r.stdout.split(".\n")[:-1]:
            lines = block.split("\n")[:-1]
            tiles = set()
            for words in (line.split() for line in lines[1:]):
                if words[0] in ("k_ortho_product", "k_ortho_join"):      # side first, then halves, product and output at the end
                    two, product, output = (int(w) for w in words[-3:])
                    tiles.add((words[0][8:], int(words[1]), two, product, output))
            out.append((int(lines[0]), tiles))
        assert len(out) == len(plans)
        return out

    return run


def expected(plan, kind):
    half, _, tiles = plan
    out = set()
    for product, text in enumerate(tiles.split()):
        side = int(text.rstrip("c"))
        for p in (X, LAST) if product == X else (product,):
            for kernel in ("product", "join") if text.endswith("c") else ("product",):
                out.add((kernel, side, int(not half), p, kind if p == LAST else 0))
    return out


def test_the_listed_plans_launch_what_is_listed(launches):
    calls = [(plan, kind) for plan in PLANS for kind in TYPES]
    for (plan, kind), (_, got) in zip(calls, launches([(half, mats, kind) for (half, mats, _), kind in calls])):
        assert got == expected(plan, kind), (name(plan), kind)


def test_together_they_launch_every_kernel_of_tiles():
    reached = set().union(*(expected(plan, kind) for plan in PLANS for kind in TYPES))
    outputs = {G: (0,), B: (0,), X: (0,), LAST: TYPES}
    for two in (0, 1):
        for product, kinds in outputs.items():
            for kind in kinds:
                for side in (64, 128, 256):
                    assert ("product", side, two, product, kind) in reached
                    if side > 64 or product == G:
                        assert ("join", side, two, product, kind) in reached


def test_the_memory_is_what_the_header_says(launches):
    up = lambda v: (v + 63) // 64 * 64                    # noqa: E731
    for (half, mats, tiles), (got, _) in zip(PLANS, launches([(half, mats, 0) for half, mats, _ in PLANS])):
        d = sum(r * c for r, c in mats)
        sides = [(up(min(m)), up(max(m))) for m in mats]
        least = 4 * d + sum((4 if half else 8) * m * (m + n) for m, n in sides)
        most = 4.2 * d + sum((4 if half else 8) * m * (m + n) + 0.3 * m * n for m, n in sides) + (1e8 if "c" in tiles else 0) + 65536
        assert least <= got <= most, (mats[0], got, least, most)
    small = [(64, 512)] * 100 + [(100, 128)] * 50
    (got, _), = launches([(False, small, 0)])
    assert got <= 4.2 * sum(r * c for r, c in small) + 65536
