"""How the kernels over the 8-bit cache share out their work (csrc/kv8_line.cuh), compiled for the
host: every tile of every unit is walked over exactly once and nothing out of range is read, with
requests of more rows than tokens, without rows or tokens, and any grid (no GPU)."""
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LINES = {"few rows": 0, "attention, many rows": 1, "weigh, bf16": 2, "weigh, fp32": 3}


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    out = str(tmp_path_factory.mktemp("line") / "line")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2608_24063_gb300", "csrc"), os.path.join(HERE, "kv8_line_host.cpp"), "-o", out],
                   check=True)
    return out


def _check(program, kind, batches):
    """batches: (Hkv, G, causal, grid, [(tokens, rows)])"""
    text = "".join("%d %d %d %d 16 %d %d %s\n" % (kind, Hkv, G, causal, grid, len(req), " ".join("%d %d" % x for x in req))
                   for Hkv, G, causal, grid, req in batches)
    got = subprocess.run([program], input=text, capture_output=True, text=True, timeout=120, check=True).stdout.split("\n")
    for line, batch in zip(got, batches):
        assert line == "ok", (line, batch)
    assert len(got) == len(batches) + 1


def _random(seed):
    rnd = random.Random(seed)
    req = []
    for _ in range(rnd.choice([1, 2, 5, 40])):
        length = rnd.choice([0, 1, rnd.randrange(1, 60), rnd.randrange(300, 1300)])
        m = rnd.choice([0, 1, rnd.randrange(0, 9), rnd.randrange(0, length + 1), length + rnd.randrange(1, 700)])
        req.append((length, m))
    return rnd.randrange(1, 9), rnd.choice([1, 2, 7, 8, 65, 128]), rnd.randrange(2), rnd.choice([1, 2, 7, 76, 152]), req


@pytest.mark.parametrize("name", LINES)
def test_every_tile_once(program, name):
    _check(program, LINES[name], [_random(seed) for seed in range(150)])


@pytest.mark.parametrize("name", LINES)
def test_more_rows_than_tokens(program, name):
    _check(program, LINES[name], [(8, 8, 1, 152, [(20, 64)] * 24), (8, 8, 1, 152, [(200, 64)] * 23 + [(20, 64)]),
                                  (8, 8, 1, 152, [(20, 64)] + [(200, 64)] * 40), (4, 128, 1, 152, [(500, 600), (100, 500)] * 20)])
