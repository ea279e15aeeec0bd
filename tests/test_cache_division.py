"""The division of the cache attention's work over CTAs (cache_division.h, the
code that the kernels compile) on the host, up to the largest calls that are
accepted."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ITEM_COST = 3


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("division") / "cache_division_model")
    subprocess.run(
        ["g++", "-O1", "-std=c++17", "-Wall", "-Werror",
         "-I", os.path.join(ROOT, "paper_2607_20214_gb300", "csrc"),
         os.path.join(ROOT, "tests", "cache_division_model.cpp"), "-o", exe],
        check=True)

    def run(lines):
        text = "".join("%d %d %d %d %d\n" % x for x in lines)
        r = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stdout
        assert r.stdout == "%d ok\n" % len(lines)
    return run


def calls():
    """(B, H T, columns a group, tiles of the table) that the host accepts:
    (tiles + 7) B H T <= 2^31, H <= 65535, T <= 64."""
    rng = random.Random(1)
    yield 4096, 16384, 1, 1        # 2^26 items
    yield 4096, 1024 * 64, 4, 1    # 2^26 items in groups of four columns
    yield 4096, 65535, 1, 1
    yield 1, 65535, 1, 32761
    yield 1, 1, 1, (1 << 24) - 1   # the longest table
    yield 127, 1, 1, (1 << 24) - 1
    for _ in range(300):
        B = round(4096 ** rng.random())
        HT = round(65535 ** rng.random()) * rng.choice([1, 1, 2, 4, 64])
        most = (1 << 31) // (B * HT) - 7
        if most < 1:
            continue
        tiles = min(most, (1 << 24) - 1)
        yield B, HT, rng.choice([1, 2, 4, 8, 16]), max(
            1, round(tiles ** rng.choice([0.0, 0.5, 0.9, 1.0])))


@pytest.mark.parametrize("full", [304, 456])
def test_every_accepted_call_is_divided_as_wider_numbers_divide_it(model,
                                                                   full):
    rng = random.Random(2)
    lines = []
    for B, HT, cols, tiles in calls():
        HC = max(1, HT // cols)
        ctas = min(B * HC * min(tiles, 64), full)
        # all sequences full; some without queries, the others of any length
        lines.append((B * (tiles + ITEM_COST), B, HC, ctas, 0))
        live = rng.randint(0, B)
        lines.append((sum(rng.randint(1, tiles) + ITEM_COST
                          for _ in range(live)), live, HC, ctas, 0))
        if B <= 32 and B * HC <= full:
            lines.append((live, live, HC, B * HC, 1))
    model(lines)
