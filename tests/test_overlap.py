"""Outputs that share part of their memory with an input or another output are refused; those that lie beside them, or between
their rows, are not."""
from __future__ import annotations

import ctypes
import os
import random
import shutil
import subprocess

import pytest
import torch

import paper_2607_20538_gb300 as cg
from paper_2607_20538_gb300 import build
from test_block8_abi import _encode, _matmul, lib  # noqa: F401  (a fixture)
from test_tree_abi import GOOD, _commit, _plan

E4M3, BF16, I32 = torch.float8_e4m3fn, torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    where = tmp_path_factory.mktemp("overlap")
    src, so = where / "o.cpp", where / "o.so"
    src.write_text(f'#include "{os.path.join(build.CSRC, "cg_overlap.h")}"\n'
                   'extern "C" int o(int64_t a, int64_t an, int64_t ab, int64_t as, int64_t b, int64_t bn, int64_t bb, int64_t bs) {\n'
                   "    return cg::overlap(cg::Rows{(const void*)a, an, ab, as}, cg::Rows{(const void*)b, bn, bb, bs});\n}\n")
    subprocess.check_call([gxx, "-O1", "-std=c++17", "-shared", "-fPIC", str(src), "-o", str(so)])
    fn = ctypes.CDLL(str(so)).o
    fn.argtypes = [ctypes.c_int64] * 8
    return lambda a, b: bool(fn(*a, *b))


def test_against_sets_of_bytes(overlap):
    rng, hits = random.Random(1), 0
    for _ in range(20000):
        rows = []
        for _ in range(2):
            n, width = rng.choice([1, 1, 2, 3, 7, 20]), rng.randint(1, 12)
            rows.append([1000 + rng.randint(0, 90), n, width, width + rng.choice([0, 0, 1, 5, 12, 20])])
        if rng.random() < 0.5:
            rows[1][3] = max(rows[0][3], rows[1][2])
        cover = [{p + i * s + k for i in range(n) for k in range(w)} for p, n, w, s in rows]
        want = bool(cover[0] & cover[1])
        hits += want
        assert overlap(*rows) == want and overlap(*rows[::-1]) == want, rows
    assert 3000 < hits < 17000


def test_ends_of_the_range(overlap):
    big = 1 << 40
    assert not overlap((4096, 1 << 30, big - 1, big), (4096 + big - 1, 1 << 30, 1, big))       # side by side, 2^70 bytes
    assert overlap((4096, 1 << 30, big - 1, big), (4096 + 7 * big + 5, 1, 1, 0))
    assert not overlap((4096, 0, 16, 16), (4096, 1, 16, 16)) and not overlap((0, 1, 16, 16), (0, 1, 16, 16))


FAKE = 0x10000
REQ, PAGES = 4 * GOOD["n_req"], 4 * GOOD["n_pages"]


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses of nothing")
@pytest.mark.parametrize("call,kw", [
    (_plan, dict(positions=FAKE + 16)), (_plan, dict(positions=2 * FAKE - 4 * 4)), (_plan, dict(masks=3 * FAKE + 8)), (_plan, dict(masks=4 * FAKE + 4)),
    (_plan, dict(masks=FAKE - 4, words=2)),
    (_commit, dict(left=3 * FAKE + 4)), (_commit, dict(left=3 * FAKE - 4)), (_commit, dict(free=5 * FAKE + REQ * GOOD["max_pages"] - 4)),
    (_commit, dict(free=9 * FAKE - PAGES + 4)), (_commit, dict(free_left=7 * FAKE + 4)), (_commit, dict(free_left=8 * FAKE + PAGES - 4)),
    (_commit, dict(left=6 * FAKE + 4096, pool=6 * FAKE)), (_commit, dict(free_left=4 * FAKE + REQ)),
    (_encode, dict(codes=FAKE + 256)), (_encode, dict(codes=FAKE - 256)), (_encode, dict(scales=FAKE + 3 * 512 - 4)), (_encode, dict(scales=2 * FAKE + 764)),
    (_matmul, dict(out=FAKE + 2)), (_matmul, dict(out=FAKE - 28)), (_matmul, dict(out=3 * FAKE + 5 * 256 - 2)), (_matmul, dict(out=2 * FAKE + 22)),
    (_matmul, dict(out=4 * FAKE + 6)),
])
def test_a_part_in_the_place_of_others(lib, call, kw):  # noqa: F811
    assert call(**kw) == -1
    said = lib.cg_last_error()
    assert b"alias" in said or b"overlap" in said


@pytest.mark.gpu
def test_beside_one_another():
    """Lists in one array, and the matrices of a call as column ranges of the same rows, their ends touching."""
    ints = torch.zeros(4096, dtype=I32, device="cuda")
    at = 0

    def part(n):
        nonlocal at
        at += n
        return ints[at - n:at]

    lens, cu, parents, positions, masks = part(2), part(3), part(5), part(5), part(5).view(5, 1)
    lens.copy_(torch.tensor([21, 18])), cu.copy_(torch.tensor([0, 3, 5])), parents.copy_(torch.tensor([-1, 0, 0, -1, 0]))
    cg.tree_plan(3, parents, lens, cu, positions, masks)
    assert positions.tolist() == [18, 19, 19, 16, 17] and masks[:, 0].tolist() == [1, 3, 5, 1, 3]
    pages = cg.Pages(8, 16, 2, 128, 2, 4)
    table, leaves, count, stack, left, free_left = part(8), part(2), part(1), part(8), part(2), part(1)
    table.copy_(torch.tensor([3, 5, -1, -1, 1, 0, -1, -1])), leaves.copy_(torch.tensor([2, -1]))
    pool = torch.randn(2, 8, 2, 16, 128, device="cuda").to(BF16)
    cg.tree_commit(pages, 3, parents, leaves, lens, cu, table, pool, left, stack, count, free_left)
    assert left.tolist() == [20, 16] and free_left.tolist() == [1] and stack[0].item() == 0

    R, K = 300, 256
    wide = torch.zeros(R, 1024 + 256, dtype=torch.uint8, device="cuda")          # x in bytes 0 .. 511, codes behind, an output behind those
    x, codes, out = wide[:, :512].view(BF16), wide[:, 512:768].view(E4M3), wide[:, 768:].view(BF16)
    x.copy_(torch.randn(R, K, device="cuda"))
    scales, w, ws = torch.empty(R, 2, device="cuda"), torch.empty(256, K, dtype=E4M3, device="cuda"), torch.empty(2, 2, device="cuda")
    cg.block8_encode(torch.randn(256, K, device="cuda").to(BF16), w, ws, rows=128)
    cg.block8_encode(x, codes, scales)
    cg.block8_matmul(codes, scales, w, ws, out)
    apart, c2, s2 = torch.empty(R, 256, dtype=BF16, device="cuda"), torch.empty(R, K, dtype=E4M3, device="cuda"), torch.empty(R, 2, device="cuda")
    cg.block8_encode(x.contiguous(), c2, s2)
    cg.block8_matmul(c2, s2, w, ws, apart)
    assert torch.equal(c2.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s2, scales) and torch.equal(out, apart)
    with pytest.raises(cg.CodecGaugeError, match="overlap"):
        cg.block8_matmul(codes, scales, w, ws, wide[:, 766:1278].view(BF16))
    with pytest.raises(cg.CodecGaugeError, match="overlap"):
        cg.block8_encode(x, wide[:, 496:752].view(E4M3), scales)
    assert cg.get_status() == 0
