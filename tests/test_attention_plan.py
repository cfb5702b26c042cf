"""What sizes the attention blocks are cut into (csrc/psgd_attention_plan.h), compiled for the CPU: every sequence's tiles have places of their own, every part's sums
a slot, and the sizes that the kernels' tests count on have several parts."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LDS = 160 * 1024


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    gxx = shutil.which("g++") or shutil.which("c++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "attention_plan_check")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2002_01119_amd", "csrc"),
                    os.path.join(ROOT, "tests", "attention_plan_check.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True).stdout.strip().split("\n")
        assert len(out) == len(lines)
        return [[int(w) for w in line.split()] for line in out]
    return run


def shape(ask, size, head):
    return dict(zip(("held", "lds", "own", "walked", "queries", "waves"), ask(["shape %d %d" % (size, head)])[0]))


@pytest.mark.parametrize("size", [2, 4])
def test_tiles_fit_the_local_memory(ask, size):
    for head in range(1, 257):
        s = shape(ask, size, head)
        row = s["lds"] * size
        assert s["held"] >= head and s["held"] % 32 == 0 and s["lds"] >= s["held"] and row & (row - 1) == 0
        assert s["walked"] % 32 == 0 and s["queries"] % 32 == 0 and s["own"] % 64 == 0
        assert 4 * s["walked"] * row <= LDS and 4 * s["queries"] * row + (s["own"] * row if s["queries"] != s["walked"] else 0) + 16 * s["queries"] <= LDS
        assert s["waves"] * 2 * 2 * 32 * row <= LDS and s["waves"] * 16 * (s["held"] + 2) * 4 <= LDS


def test_sequences_have_places_of_their_own():
    """The rule by which a workgroup finds its tile: sequence s has places from starts[s] / rows + s on."""
    rng = random.Random(2)
    for _ in range(300):
        t, rows = rng.randint(1, 2000), rng.choice([64, 128])
        starts = sorted(rng.randint(0, t) for _ in range(rng.randint(2, 40)))
        taken = []
        for s, (a, b) in enumerate(zip(starts, starts[1:])):
            taken += [a // rows + s + tile for tile in range(-(-(b - a) // rows))]
        assert len(taken) == len(set(taken)) and all(0 <= p < t // rows + len(starts) - 1 for p in taken)
        for place in range(t // rows + len(starts) - 1):          # and finds it: the last sequence that begins at the place or before
            found = [s for s in range(len(starts) - 1) if starts[s] // rows + s <= place]
            tile = place - (starts[found[-1]] // rows + found[-1]) if found else -1
            there = bool(found) and 0 <= tile and tile * rows < starts[found[-1] + 1] - starts[found[-1]]
            assert there == (place in taken)


@pytest.mark.parametrize("size", [2, 4])
def test_every_part_has_a_slot(ask, size):
    """The parts that the kernel makes of a tile, by its own arithmetic, against the slots that the workspace has."""
    rng = random.Random(size)
    lines, calls = [], []
    for _ in range(400):
        kv = rng.choice([1, 2, 3, 8])
        heads, head, n, t = kv * rng.choice([1, 2, 4, 16]), rng.choice([16, 64, 80, 128, 200, 256]), rng.choice([1, 2, 8, 64]), rng.choice([1, 70, 300, 1000, 5000, 40000])
        window = rng.choice([0, 0, 1, 33, 500, 4096, 10 ** 6])
        calls.append((heads, kv, head, window, rng.choice([0, 1, 4, 300]) if window else 0, rng.choice([0, 1, 3, 40]), n, t))
        lines.append("grad %d %s" % (size, " ".join(map(str, calls[-1]))))
    several = first = 0
    for (heads, kv, head, window, sinks, seqs, n, t), (most, steps, first_tiles, first_most, first_steps, slots, first_slots, slot_bytes, total) in zip(calls, ask(lines)):
        s = shape(ask, size, head)
        own, rows, members = s["own"], s["queries"], heads // kv
        places = t // own + max(1, seqs)
        assert most >= 1 and first_most >= 1 and slots == (places * most if most > 1 else 0) and first_slots == max(1, seqs) * first_tiles * first_most
        assert slot_bytes == 2 * own * s["held"] * 4 and total >= (slots + first_slots) * n * kv * slot_bytes
        assert (slots + first_slots) * n * kv * slot_bytes <= (5 << 30)
        seen = window if 0 < window < t else t + 1
        for tile in {0, 1, first_tiles, (t - 1) // own}:                             # of one sequence of all rows, the longest there is
            key0 = tile * own
            if key0 >= t:
                continue
            behind = t if key0 < sinks and seen <= t else min(t, min(key0 + own, t) - 1 + seen)
            count = (-(-behind // rows) - key0 // rows) * members
            cap, least = (first_most, first_steps) if tile < first_tiles else (most, steps)
            parts = min(cap, (count - 1) // least + 1)
            each = -(-count // parts)
            parts = -(-count // each)
            assert 1 <= parts <= cap and (parts - 1) * each < count <= parts * each
            several += parts > 1 and tile >= first_tiles
            first += parts > 1 and tile < first_tiles
    assert several > 20 and first > 20


def test_sizes_of_the_kernels_tests_have_parts(ask):
    grad = lambda *a: ask(["grad " + " ".join(map(str, a))])[0]  # noqa: E731
    assert grad(2, 2, 1, 64, 0, 0, 0, 1, 257)[0] > 1                                 # all tiles, each length of a few tiles
    assert grad(4, 2, 1, 64, 0, 0, 0, 1, 257)[0] > 1
    assert grad(2, 2, 1, 64, 129, 3, 0, 1, 2100)[3] > 1                              # the first tokens' tile
    assert grad(2, 32, 8, 128, 0, 0, 5, 4, 4096)[0] == 1                             # a training batch fills the chip with whole tiles
    assert grad(2, 32, 8, 128, 512, 4, 5, 4, 4096)[:1] + grad(2, 32, 8, 128, 512, 4, 5, 4, 4096)[3:4] == [1, grad(2, 32, 8, 128, 512, 4, 5, 4, 4096)[3]]


def test_a_steps_parts(ask):
    parts = lambda *a: ask(["step " + " ".join(map(str, a))])[0][0]  # noqa: E731
    assert parts(2, 8, 131072, 128) == 32 and parts(2, 768, 4100, 128) == 1 and parts(2, 1, 1, 64) == 1 and parts(2, 1, 256, 64) == 1 and parts(2, 1, 257, 64) == 2
    assert parts(2, 10 ** 6, 1 << 30, 128) == 1 and parts(4, 1, 1 << 30, 256) == 256 and parts(2, 1, 1 << 30, 16) == 512


def test_heights_of_forward_tiles(ask):
    blocks = lambda *a: ask(["forward %d %d %d %d" % a])[0][0]  # noqa: E731
    assert [blocks(2, h, 260, 15 * 16) for h in (24, 64, 80, 128, 144)] == [1, 1, 1, 1, 1] and [blocks(2, h, 260, 256) for h in (24, 64, 80, 128, 144)] == [2, 2, 2, 2, 1]
    assert blocks(4, 64, 4096, 128) == 1
