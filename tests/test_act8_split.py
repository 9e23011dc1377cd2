"""How the weight gradient from 8 bits is cut, on the host: every k-block of every tile once, every part its own slot within the workspace,
and workers left over are used only where the longest of them is done sooner."""
import math
import os
import random
import subprocess

import pytest

from paper_2609_09821_b200 import binding as B
from paper_2609_09821_b200 import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))
SIZES = [(R, Mo, No, 148) for Mo, No in ((512, 1024), (1024, 1024), (1280, 1280), (1280, 1024), (1024, 768), (2048, 1280), (2048, 2048), (300, 700), (64, 1100),
                                          (64, 9600), (64, 12800), (128, 4800), (69, 512), (28, 512), (1, 1), (300, 129), (128, 65536))
         for R in (1, 64, 300, 2048, 4096, 8192, 16000, 20000, 40000, 131072)]


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("split") / "split")
    subprocess.run([lib_build._nvcc()] + lib_build.NVCC_FLAGS + ["-I", lib_build.CSRC, os.path.join(HERE, "act8_split_host.cu"), "-o", exe], check=True)
    rng = random.Random(5)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    sizes = SIZES + [(log(1, 300000), log(1, 4096), log(1, 8192), rng.choice([148, 148, 148, 132, 80, 18])) for _ in range(400)]
    text = subprocess.run([exe], input="\n".join("%d %d %d %d" % s for s in sizes), capture_output=True, text=True, check=True).stdout
    out = []
    for line in text.splitlines():
        kind, *v = line.split()
        if kind == "split":
            out.append((dict(zip(("block_n", "pair", "tiles", "kb", "workers", "slices", "slice_kb", "helpers"), map(int, v))), []))
        elif kind == "part":
            out[-1][1].append(tuple(map(int, v)))
    assert len(out) == len(sizes)
    return list(zip(sizes, out))


def test_every_block_once_and_slots_within_the_workspace(split):
    lib_build.build()
    lib = B.load()
    for (R, Mo, No, _), (s, parts) in split:
        tiles = {}
        for _, tile, k0, n, _ in parts:
            assert n >= 1
            tiles.setdefault(tile, []).append((k0, n))
        assert sorted(tiles) == list(range(s["tiles"]))
        for ranges in tiles.values():
            at = 0
            for k0, n in sorted(ranges):
                assert k0 == at
                at += n
            assert at == s["kb"]
        if s["slices"] == 1 and not s["helpers"]:
            continue                                                     # whole tiles: no slots
        slots = [p[4] for p in parts]
        assert len(set(slots)) == len(slots)
        assert (max(slots) + 1) * s["block_n"] * (256 if s["pair"] else 128) * 4 <= lib.im_gemm_act8_tn_workspace_bytes(R, Mo, No), (R, Mo, No)


def test_helpers_are_done_sooner(split):
    """A worker's k-blocks, and what the ends of its parts behind the first cost (measured: 12 k-blocks of a pair, 3 of a lone CTA): with
    helpers the longest is shorter than without, also where the sum of partial tiles has to be paid for first (24 and 9)."""
    helped = 0
    for size, (s, parts) in split:
        if not s["helpers"]:
            continue
        helped += 1
        cost, total = (12, 24) if s["pair"] else (3, 9)
        work = {}
        for w, _, _, n, _ in parts:
            work[w] = work[w] + n + cost if w in work else n
        without = -(-s["kb"] // s["slices"])
        assert max(work.values()) + (total if s["slices"] == 1 else 0) < without, (size, s)
        # and nobody waits long for the rest: the mains are within a part's cost and rounding of an even share
        assert s["slice_kb"] <= (s["kb"] * s["tiles"] + sum(cost for p in parts[s["tiles"] * s["slices"]:])) / s["workers"] + cost
    assert helped >= 40
