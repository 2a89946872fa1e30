"""The sizes of tests/token_sizes.py reach every form that the calls from tokens to the loss can take."""
import re
import shutil
import subprocess

import pytest

from paper_2603_28845_amd import binding
from token_shapes import TILES, ask
from token_sizes import LAYER, LOSS, TABLE

ALL = set(TILES)


@pytest.mark.parametrize("dtype,esz", [("bf16", 2), ("f32", 4)])
def test_loss(tmp_path, dtype, esz):
    sizes = LOSS[dtype]
    first = ask(tmp_path, [q for n, d, v in sizes for q in (("few", n, v, esz), ("tiles", n, v, d, esz), ("columns", n, v, esz))])
    seen = {k: set() for k in ("few", "logits", "grads", "rows", "weight")}
    for i, (n, d, v) in enumerate(sizes):
        few, tiles, columns = first[3 * i:3 * i + 3]
        seen["few" if few else "logits"].add(-(-n // 16) if few else TILES[tiles])
        wide = min(columns, v)
        grads, rows, weight = ask(tmp_path, [("tiles", n, wide, d, esz), ("rows", n, d, columns, esz), ("tiles", wide, d, n, esz)])
        seen["grads"].add(TILES[grads])
        seen["rows"].add(TILES[rows])
        seen["weight"].add(TILES[weight])
    products = ALL if esz == 2 else {"HALF", "SMALL", "SMALL_SPLIT"}
    assert seen["logits"] == seen["grads"] == seen["weight"] == products
    assert seen["rows"] == ALL - {"SMALL_SPLIT"}
    assert seen["few"] >= ({1, 2} if esz == 2 else {1, 2, 3, 4})


def test_fp32_takes_small_tiles(tmp_path):
    """What is not built for fp32 is never asked for."""
    sizes = [(m, n, k, 4) for m in (1, 63, 200, 1000, 9000, 1 << 20) for n in (1, 100, 3000, 50000, 1 << 20) for k in (4, 64, 500, 5000, 1 << 20) if m * n < 1 << 35]
    assert {TILES[t] for t in ask(tmp_path, [("tiles", *s) for s in sizes])} == {"HALF", "SMALL", "SMALL_SPLIT"}


def test_layers(tmp_path):
    answers = ask(tmp_path, [q for n, d, m in LAYER for q in (("few", n, m, 1), ("tiles", n, m, d, 1))])
    few, tiles = set(), set()
    for i, (n, d, m) in enumerate(LAYER):
        if answers[2 * i]:
            few.add((2, 1) if m > 8192 else (1, 1 if n <= 16 else 2 if n <= 32 else 4))
        else:
            tiles.add(TILES[answers[2 * i + 1]])
    assert tiles == ALL and few == {(2, 1), (1, 1), (1, 2), (1, 4)}


def test_table(tmp_path):
    assert set(ask(tmp_path, [("segment", n, d) for n, d, _ in TABLE])) == {16, 32, 64}


def test_nothing_is_built_that_no_size_takes():
    """The kernels' launch stubs in the built library: bf16 (of layers: both) with each shape, fp32 with 64 x 64 and 128 x 64 tiles, but
    for the gradient of the rows, whose tiles are chosen with their shares; no waves that share k there."""
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    said = subprocess.run([nm, "-C", binding.LIB_PATH], check=True, capture_output=True, text=True).stdout
    shapes = {"2, 2, 4, 4": "BIG", "2, 2, 2, 2": "MID", "2, 2, 2, 1": "HALF"}
    built = {}
    for kernel, kind, waves, split in re.findall(r"__device_stub__(\w+)<([\w:() ]+), onecomp::product::Shape<(\d, \d, \d, \d), \d+, (\d), \d>", said):
        built.setdefault((kernel, kind.split("::")[-1]), set()).add(shapes.get(waves, "SMALL_SPLIT" if split == "4" else "SMALL"))
    if not built:
        pytest.skip("the library has no symbols")
    small = {"HALF", "SMALL", "SMALL_SPLIT"}
    want = {("linear_kernel", t): ALL for t in ("float", "unsigned short")}
    want.update({("grad_rows_kernel", t): ALL - {"SMALL_SPLIT"} for t in ("Bf16", "F32")})
    for kernel in ("logits_kernel", "logit_grads_kernel", "grad_weight_kernel"):
        want[kernel, "Bf16"], want[kernel, "F32"] = ALL, small
    assert built == want
