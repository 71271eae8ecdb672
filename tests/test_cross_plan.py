"""The choices of cross_plan.h, compiled for the host: bounds that hold for any hints, and both sides of the rules."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2507_11830_amd", "csrc")


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "cross_plan")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-function", "-Wno-unknown-pragmas", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I", CSRC, os.path.join(HERE, "cross_plan_host.cpp"), "-o", exe])

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(" ".join(str(int(x)) for x in l) for l in lines), capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in l.split()) for l in out.splitlines()]

    return ask


def hints(heads, batch, total_q, max_q, max_kv, can_cut=True):
    hq, hkv, d = heads
    group, cols = hq // hkv, 1
    while group & (group - 1) == 0 and cols < group and cols < 32:
        cols *= 2
    return total_q * hq, batch, batch * (hq // cols), cols, total_q, max_q, max_kv, d, can_cut


def test_any_hints(shape):
    rng = random.Random(1)
    big = lambda: int(2 ** rng.uniform(0, 31)) - 1
    lines = []
    for _ in range(4000):
        heads = rng.choice([(8, 1, 128), (32, 8, 128), (12, 3, 64), (1, 1, 64), (65536, 1, 128), (7, 7, 64)])
        lines.append(hints(heads, max(1, big()), max(1, big()), max(1, big()), big() if rng.random() < 0.7 else rng.randint(0, 300), rng.random() < 0.8))
    for line, (halves, ranked, pieces, blocks, waves, rounds, _, solo, tiles, splits, chunk) in zip(lines, shape(lines)):
        rows, batch, streams, cols, total_q, max_q, max_kv, d, can_cut = line
        assert 1 <= pieces <= 16 and (can_cut or pieces == 1)
        if pieces > 1:
            assert halves and pieces * rows <= 1 << 17  # what a workspace is sized for
            assert 2 * pieces <= -(-max_kv // 64)  # two key tiles each, one for either wave group
            assert pieces * max(rows // 128, streams) <= 256  # one round
        if batch == 1:
            assert not ranked
        if tiles:  # one round, the chunk covered, the keys too
            assert max_q * cols > 32 and tiles * (32 // cols) >= max_q and streams * tiles * splits <= (256 if d == 128 else 512)
            assert splits * chunk >= max_kv > (splits - 1) * chunk and chunk <= 1024 and (can_cut or splits == 1)
        if solo:
            assert d == 128 and pieces == 1 and not halves and max_kv > 256
        if blocks > 0:  # all keys fit LDS, twice on a CU with four waves; the grid holds all columns
            assert 32 * blocks >= max_kv and blocks * 128 * d * (2 if waves == 4 else 1) <= 160 * 1024 and waves in (4, 8) and 1 <= rounds <= 64
            assert max_kv <= (320 if d == 128 else 256) and -(-max_q * cols // (32 * waves * rounds)) <= 65535 and streams < 2**31


@pytest.mark.parametrize("heads,batch,total_q,max_q,max_kv,want", [
    ((8, 1, 128), 8, 8 * 4096, 4096, 4096, (0, 0, 1)),  # one length: whole tiles by order
    ((8, 1, 128), 1, 40, 40, 9000, (1, 0, None)),  # few queries on many keys: pieces
    ((8, 1, 128), 1, 40, 40, 500, (1, 0, 1)),  # little to cut
    ((32, 4, 128), 1, 1137, 1137, 4580, (0, 0, 1)),  # halves would be a second round for a tenth of them
    ((16, 2, 128), 2, 412, 206, 2284, (1, 0, 1)),
    ((16, 2, 64), 8, 4500, 1089, 1891, (0, 1, 1)),  # uneven, more than a round: longest first
], ids=str)
def test_both_sides(shape, heads, batch, total_q, max_q, max_kv, want):
    (halves, ranked, pieces, blocks, _, _, _, solo, *_), = shape([hints(heads, batch, total_q, max_q, max_kv)])
    assert blocks == 0 and not solo
    assert (halves, ranked) == want[:2]
    assert pieces == want[2] if want[2] else pieces >= 4
    assert shape([hints(heads, batch, total_q, max_q, max_kv, False)])[0][2] == 1


@pytest.mark.parametrize("heads,total_q,max_kv,want", [
    ((8, 1, 128), 57, 10, (1, 4, 1)), ((32, 8, 128), 43303, 18, (1, 4, 3)), ((8, 1, 128), 2**24, 18, (1, 4, 17)), ((8, 1, 128), 78, 128, (4, 4, 1)), ((8, 1, 128), 78, 129, (0,)),
    ((16, 2, 128), 13992, 229, (8, 8, 4)), ((16, 2, 64), 13992, 256, (8, 4, 4)), ((16, 2, 64), 13992, 257, (0,)), ((16, 2, 128), 13992, 320, (10, 8, 4)), ((16, 2, 128), 13992, 321, (0,)), ((16, 2, 64), 100, 0, (0,)),
], ids=str)
def test_keys_that_stay_in_lds(shape, heads, total_q, max_kv, want):
    assert shape([hints(heads, 1, total_q, total_q, max_kv)])[0][3:3 + len(want)] == want


@pytest.mark.parametrize("heads,batch,max_kv,want", [
    ((8, 1, 128), 50, 64, 1), ((8, 1, 128), 50, 66, 0), ((8, 1, 128), 257, 128, 1), ((8, 1, 128), 257, 129, 0), ((16, 2, 64), 256, 100, 0), ((16, 2, 64), 257, 100, 1)], ids=str)
def test_few_tokens_on_few_keys(shape, heads, batch, max_kv, want):
    assert shape([hints(heads, batch, batch, 1, max_kv)])[0][6] == want


@pytest.mark.parametrize("heads,batch,total_q,max_q,max_kv,want", [
    ((32, 4, 128), 12, 12 * 1212, 1212, 272, (1, 0)), ((32, 4, 128), 7, 7 * 313, 313, 529, (1, 0)), ((16, 2, 128), 6, 6 * 700, 1300, 700, (1, 1)),
    ((32, 4, 128), 12, 12 * 1212, 1212, 256, (0, 0)), ((8, 1, 128), 6, 6 * 714, 714, 2014, (0, 0)), ((8, 1, 128), 8, 8 * 4096, 4096, 4096, (0, 0)),
    ((16, 2, 64), 12, 12 * 1212, 1212, 500, (0, 0))], ids=str)
def test_two_workgroups_a_cu(shape, heads, batch, total_q, max_q, max_kv, want):
    s = shape([hints(heads, batch, total_q, max_q, max_kv)])[0]
    assert (s[7], s[1]) == want


@pytest.mark.parametrize("heads,batch,max_q,max_kv,want", [
    ((32, 8, 128), 2, 16, 278, (2, 1)), ((8, 1, 128), 1, 4, 278, (0,)), ((8, 1, 128), 1, 5, 512, (2, 1)), ((8, 1, 128), 1, 5, 513, (2, 3)), ((8, 1, 128), 32, 32, 400, (8, 1)),
    ((8, 1, 128), 33, 32, 400, (0,)), ((16, 2, 64), 32, 32, 400, (8, 1)), ((16, 2, 64), 33, 32, 400, (0,)), ((8, 1, 128), 8, 32, 2048, (8, 4)), ((8, 1, 128), 8, 32, 2049, (0,)), ((8, 1, 128), 9, 32, 600, (0,)),
    ((16, 2, 64), 6, 32, 1365, (8, 4)), ((16, 2, 64), 7, 32, 600, (0,)),
    ((8, 1, 128), 1, 8, 60000, (2, 118)), ((8, 1, 128), 1, 8, 70000, (0,))], ids=str)
def test_column_tiles(shape, heads, batch, max_q, max_kv, want):
    assert shape([hints(heads, batch, batch * max_q, max_q, max_kv)])[0][8:8 + len(want)] == want
