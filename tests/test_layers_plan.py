"""What sizes run which kernel: the launch rules of the layers and losses (csrc/psgd_layers_plan.h), compiled for the CPU, against what the tests of the
kernels count on."""
import os
import shutil
import subprocess

import pytest

import layers_shapes as shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    gxx = shutil.which("g++") or shutil.which("c++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "layers_plan_check")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2002_01119_amd", "csrc"),
                    os.path.join(ROOT, "tests", "layers_plan_check.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True).stdout.strip().split("\n")
        assert len(out) == len(lines)
        return [line.split(None, 1)[1] for line in out]
    return run


def question(kind, size, shape):
    return " ".join(map(str, (kind, size, *shape, *([0] if len(shape) == 3 else []), CUS)))


TABLES = dict(linear=shapes.LINEAR, grad=shapes.GRAD, logprobs=shapes.LOGPROBS, distill=shapes.DISTILL)


@pytest.mark.parametrize("kind", sorted(TABLES))
@pytest.mark.parametrize("size", [2, 4])
def test_sizes_run_what_their_tests_say(ask, kind, size):
    rows = TABLES[kind][size]
    got = ask([question(kind, size, shape) for shape, _ in rows])
    assert [(shape, g) for (shape, _), g in zip(rows, got)] == rows


TILES = {2: ["64x64", "128x128", "256x256"], 4: ["32x128", "64x64", "128x32", "256x256"]}


def test_a_workgroup_more_is_counted_only_where_its_registers_fit(ask):
    """dx's 128 x 128 tiles hold two workgroups to a compute unit whatever the sum's length; counted as three they were chosen over faster ones."""
    for n, t, i, o in ((8, 2048, 2048, 40), (4, 2048, 8192, 100), (4, 2048, 8192, 16), (8, 2048, 2048, 100)):
        assert ask(["grad 2 %d %d %d %d %d" % (n, t, i, o, CUS)])[0].startswith("dx=256x256/short")


def test_rows_of_three_to_eight_a_compute_unit_are_held_by_fewer_lanes(ask):
    for size, v in ((4, 10007), (4, 16384), (2, 20000), (2, 32768)):
        got = ask(["distill %d %d %d 1 0 %d" % (size, rows, v, CUS) for rows in (512, 513, 1024, 1025, 1600, 2048, 2049)])
        assert got == ["lanes=1024 held=4"] + ["lanes=256 held=16"] * 5 + ["lanes=1024 held=4"]


def words(table, size):
    return {word for _, said in table[size] for word in said.split()}


@pytest.mark.parametrize("size", [2, 4])
def test_every_kernel_of_the_products_is_reached(size):
    """Each tile in each orientation with whole sums, parts of them and short ones, but what next to no size chooses: parts of 256 x 256 in bf16 other than
    dx's, and 128 x 128 of floats other than with short sums."""
    y, g = words(shapes.LINEAR, size), words(shapes.GRAD, size)
    wanted_y = {"y=" + tile + how for tile in TILES[size] for how in ("", "/short")} | {"y=%s/parts" % tile for tile in TILES[size] if (size, tile) != (2, "256x256")}
    wanted_g = {product + "=" + tile + how for product in ("dx", "dw") for tile in TILES[size] for how in ("", "/short")}
    wanted_y |= {"few=%d/%d" % (tokens, outputs) for tokens in (1, 2, 4) for outputs in (1, 4)} | ({"few=8/1"} if size == 4 else set())
    wanted_g |= {"dwfew=%d/%d" % (tokens, rows) for tokens in ((2, 4, 8) if size == 2 else (2, 4, 8, 16)) for rows in (4, 16, 64)}
    wanted_g |= {"pair=64"} | ({"pair=128", "dx=256x256/parts", "dx=128x128/parts", "dw=128x128/parts"} if size == 2 else {"dw=128x128/short"})
    assert not wanted_y - y and not wanted_g - g, (sorted(wanted_y - y), sorted(wanted_g - g))


def test_every_form_of_the_losses_is_reached():
    said = {" ".join(word for word in s.split()) for size in (2, 4) for _, s in shapes.LOGPROBS[size]}
    for lanes, batches, kept in ((64, "several", 1), (256, "one", 1), (256, "several", 1), (256, "several", 0), (1024, "several", 1), (1024, "several", 0)):
        assert "lanes=%d batches=%s kept=%d" % (lanes, batches, kept) in said
    said = words(shapes.DISTILL, 2) | words(shapes.DISTILL, 4)
    assert {"held=%d" % held for held in (0, 1, 2, 4, 8, 16)} <= said
    forms = {s for size in (2, 4) for _, s in shapes.DISTILL[size]}
    assert {"lanes=%d held=%d" % f for f in ((64, 1), (64, 2), (64, 4), (256, 2), (256, 4), (256, 8), (256, 16), (1024, 4), (1024, 8), (1024, 16), (1024, 0),
                                             (64, 0), (256, 0))} <= forms
