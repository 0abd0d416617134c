"""The schedule of the full-attention calls as the host makes it (no GPU needed): how units of work are
shared out over CTAs, and which decode steps are split."""
import os
import subprocess

import pytest

from paper_2609_15030_gb300 import build
from tests.attn_cases import MANY_SPLIT

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def schedule(tmp_path_factory):
    lib = build.build()
    exe = tmp_path_factory.mktemp("schedule") / "schedule"
    subprocess.run([build._nvcc(), *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.INCLUDE,
                    "-I", build.CSRC, os.path.join(HERE, "attn_schedule", "schedule.cu"), "-o", str(exe), lib,
                    "-Xlinker", "-rpath," + os.path.dirname(lib)], check=True, timeout=300)

    def run(*args):
        r = subprocess.run([str(exe), *map(str, args)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout
        return [int(x) for x in r.stdout.split()]
    return run


def test_every_unit_is_one_ctas(schedule):
    """Below and above 2^22 units (one prompt of 131,072 tokens of 32 heads has 8.4 million), up to 2^31."""
    assert schedule("shares")[0] > 50_000


def decode(schedule, batch, kv_heads, max_kv, d=128, prefix=0, sms=152):
    unsplit, joined, _, size, _ = schedule("decode", batch, 4 * kv_heads, kv_heads, d, max_kv, prefix, sms)
    assert joined == (not unsplit) and (size > 0) == bool(joined)
    return bool(unsplit)


@pytest.mark.parametrize("batch,kv_heads", [(38, 8), (37, 8), (76, 4), (64, 4), (304, 1), (1, 4), (384, 8)])
def test_decode_steps_of_long_bounds_are_split(schedule, batch, kv_heads):
    """The bound says nothing of the lengths: one request at it beside short ones must not be one CTA's."""
    for max_kv in (4 * 128 + 1, 1000, 2304, 4096, 12_800, 131_072):
        assert not decode(schedule, batch, kv_heads, max_kv), max_kv


def test_decode_steps_of_short_bounds_are_not(schedule):
    for batch, kv_heads in ((38, 8), (64, 4), (1, 2), (384, 8)):
        for max_kv in (0, 1, 128, 300, 384):
            assert decode(schedule, batch, kv_heads, max_kv), (batch, kv_heads, max_kv)


@pytest.mark.parametrize("unsplit", [0, 1])
@pytest.mark.parametrize("batch,max_kv,prefix", [(1, 1 << 20, 0), (1, 200_000_000, 0), (384, 300, 0),
                                                 (33, 200_000_000, 100), (64, 10, 1 << 30)])
def test_waits_last_as_long_as_the_work_may(schedule, batch, max_kv, prefix, unsplit):
    """1 s, and beside it more than the longest run of tiles takes (1.5 us each for two tiles of rows)."""
    *_, limit = schedule("decode", batch, 4, 1, 64, max_kv, prefix, 152, unsplit)
    longest = max(max_kv, prefix) // 128
    assert limit >= 1_000_000_000 + 10 * 1_500 * (longest if unsplit else longest // 304)
    assert limit < 3_000_000_000 or longest > 50_000


def test_the_gpu_tests_reach_both_joins_and_both_counts(schedule):
    """What tests/test_gpu_attn_bounds.py runs, on 152 SMs: more than 64 split items with one and with two tiles of
    rows (the join that takes all columns in one block), and more than 2^22 units."""
    for heads, kv_heads, pos0, n in MANY_SPLIT:
        lengths = [x for pair in zip(pos0, n) for x in pair]
        for d in (64, 128):
            unsplit, joined, groups, _, n_split = schedule("prefill", heads, kv_heads, d, 152, *lengths)
            assert not unsplit and joined and n_split > 64
            assert groups == (2 if max(n) * heads // kv_heads > 128 else 1)
    assert schedule("prefill", 32, 8, 64, 152, 0, 131_072)[3] > 1 << 22
    _, _, ctas, _, _ = schedule("decode", 384, 8, 8, 64, 180_224, 0, 152)
    assert ctas == 304 and 384 * 8 * (180_224 // 128 + 1) > 1 << 22
