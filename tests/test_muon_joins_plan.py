"""Which products of the orthogonalised matrices are cut along their sums and joined, on the CPU:
a Muon step's launches are written down instead of made (launches.c)."""
import json
import os
import re
import subprocess
import sys

import pytest

h2 = pytest.importorskip("paper_1907_11210_amd.huge2")
from test_train_plan import HERE  # noqa: E402

# Lists of matrices, and which of them (if any) has no gradient.  By the rule that chooses the
# tiles and cuts their sums, together they take every kernel that it ever takes.
JOINED = {
    "f32": [([(1454, 67)], None), ([(1166, 1191)], None), ([(1536, 1536)], None),
            ([(132, 4968)] * 6, None), ([(1569, 1892)] * 6, 2), ([(8922, 450)], None),
            ([(497, 121), (7018, 145), (275, 993), (3575, 334), (64, 925), (240, 1243)], 4),
            ([(939, 1135), (672, 94), (1081, 3774)], 1),
            ([(157, 445), (882, 3615), (1351, 1654)], 0)],
    "f16": [([(3035, 64)], None), ([(136, 8985)] * 6, None), ([(1572, 2008)] * 6, 5),
            ([(934, 822)] * 6, 0), ([(2947, 776)], None), ([(4309, 2061)], None),
            ([(4205, 976)], None),
            ([(2488, 2966), (180, 5725), (77, 983), (2973, 1995), (450, 1352), (776, 227)], 2)],
}
# Products: A = X X^T, A A, B X, B X of the last step; tiles: 64x64, 128x128, 256x128.  (The rule
# takes small tiles for short sums alone, which are not cut but in the first product.)
EVERY = {(product, size) for product in range(4) for size in range(3) if product == 0 or size}

SCRIPT = """
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2], ctypes.RTLD_GLOBAL)
L.launch_name.restype = ctypes.c_char_p
from paper_1907_11210_amd import train as tr
done = []
for shapes, products in json.load(sys.stdin):
    tensors, at = [], 1 << 20
    for rows, cols in shapes:
        room = (4 * rows * cols + 255) // 256 * 256
        tensors.append(tr.MuonTensor(param=at, m=at + room, rows=rows, cols=cols, scale=1.0))
        at += 2 * room
    plan = tr.huge2_muon_plan_create(tensors, tr.newton_schulz(products=products))
    grads = (ctypes.c_void_p * len(shapes))(*[at] * len(shapes))
    tr.huge2_muon_step(plan, ctypes.addressof(grads), tr.MuonOptions(0.1, 0.9, 1))
    tr.huge2_muon_plan_destroy(plan)
    done.append([(L.launch_name(i).decode(), L.launch_grid(i, 0), L.launch_grid(i, 1))
                 for i in range(L.launch_total())])
    L.launch_forget()
json.dump(done, sys.stdout)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(h2.LIB_PATH):
        from paper_1907_11210_amd import _build
        _build.build()
    libs = []
    for name in ("allocations", "launches"):
        libs.append(str(tmp_path_factory.mktemp("plan") / (name + ".so")))
        subprocess.run(["gcc", "-shared", "-fPIC", "-o", libs[-1], os.path.join(HERE, name + ".c")],
                       check=True)

    def run(calls):
        done = subprocess.run([sys.executable, "-c", SCRIPT, *libs], input=json.dumps(calls),
                              text=True, capture_output=True, cwd=os.path.dirname(HERE), timeout=120)
        assert done.returncode == 0, done.stderr
        return json.loads(done.stdout)
    return run


def _products(launched):
    """(kernel, parts, product, size of tiles) of each launch, its works and blocks."""
    found = []
    for name, works, blocks in launched:
        m = re.search(r"ns_(product|join)_kernelILi(\d)ELi(\d)ELi(\d)E", name)
        if m:
            found.append((m[1], *(int(n) for n in m.groups()[1:]), works, blocks))
    return found


def _tiles(shapes, product, size):
    """Tiles of a product, of symmetric ones those that hold a block on or over the diagonal."""
    high, wide = ((64, 64), (128, 128), (256, 128))[size]
    total = 0
    for rows, cols in shapes:
        m, n = (-(-s // 64) * 64 for s in sorted((rows, cols)))
        turned = product == 3 and rows > cols
        down = -(-(n if turned else m) // high)
        right = -(-(m if turned or product < 2 else n) // wide)
        total += sum(right - (r * high // wide if product < 2 else 0) for r in range(down))
    return total


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_every_product_is_cut_and_joined(launches, products):
    cut, whole, mixed = set(), set(), set()
    lists = [shapes for shapes, _ in JOINED[products]]
    for shapes, launched in zip(lists, launches([(s, products) for s in lists])):
        found = _products(launched)
        assert {p[1] for p in found} == {2 if products == "f32" else 1}
        for i, (kernel, _, product, size, works, blocks) in enumerate(found):
            if kernel == "join":
                assert found[i - 1][:4] == ("product", *found[i][1:4])  # right behind it
                assert blocks == (1, 4, 8)[size]
                cut.add((product, size))
                pieces, tiles = found[i - 1][4], _tiles(shapes, product, size)
                assert pieces >= tiles + works  # two pieces or more of each that is cut
                if works < tiles:
                    mixed.add((product, size))
            elif i + 1 == len(found) or found[i + 1][0] == "product":
                assert works == _tiles(shapes, product, size)
                whole.add((product, size))
    assert cut == EVERY
    assert whole >= {(p, 0) for p in range(1, 4)}
    assert {p for p, _ in mixed} == set(range(4)) and {s for _, s in mixed} >= {1, 2}


def test_the_lists_with_whole_rounds_and_a_cut_rest(launches):
    """A round of 256 tiles that stay whole, and the others cut: a large matrix in f16."""
    found = _products(launches([([(4096, 8192)], "f16")])[0])
    gram = [f for f in found if f[2] == 0][:2]
    assert gram[0] == ("product", 1, 0, 2, 512, 1) and gram[1] == ("join", 1, 0, 2, 16, 8)
    assert _tiles([(4096, 8192)], 0, 2) == 256 + 16


@pytest.mark.parametrize("tile", ["-2147483648", "-1", "0", "2", "2147483647", "x"])
def test_sizes_of_tiles_by_the_environment(launches, monkeypatch, tile):
    """Any number chooses one of the three."""
    monkeypatch.setenv("HUGE2_NS_TILE", tile)
    for found in _products(launches([([(2000, 90)], "f32")])[0]):
        assert found[3] in (0, 1, 2)
        if found[2] >= 2:  # (whole tiles, with sums of 128)
            assert found[4] == _tiles([(2000, 90)], *found[2:4])
        if tile in ("0", "2"):
            assert found[3] == int(tile)
