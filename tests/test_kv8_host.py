"""Host-only checks of rotary positions and the 8-bit cache: the plan of the angles against its formulas, every argument
error before any CUDA call (no GPU needed)."""
import math

import pytest

import paper_2609_15030_gb300 as hs
from tests.kv8_helpers import VALUES, to_e4m3

FAKE = 1 << 20        # a 16-byte aligned non-null address that is never dereferenced
SHAPE = dict(batch=2, n_heads=8, n_kv_heads=2, head_dim=128, page_size=16, num_blocks=64, max_pages=8)
INV, MIS, UNS = hs.HS_ERR_INVALID_ARG, hs.HS_ERR_MISALIGNED, hs.HS_ERR_UNSUPPORTED
CONTEXT, LOW, HIGH = 8192, 1.0, 32.0


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_15030_gb300 import build
    build.build()


def shape(**kw):
    return hs.make_attn_shape(**{**SHAPE, **kw})


def plan(dims=128, layout=hs.HS_ROPE_HALF, **kw):
    a = dict(base=10000.0, scaling=hs.HS_ROPE_PLAIN)
    a.update(kw)
    return hs.hs_rope_plan(dims, layout, **a)


def formula(dims, base, scaling, f):
    theta = [base ** (-2.0 * i / dims) for i in range(dims // 2)]
    if scaling == hs.HS_ROPE_LINEAR:
        return [x / f for x in theta]
    if scaling == hs.HS_ROPE_BASE:
        return [(base * f ** (dims / (dims - 2))) ** (-2.0 * i / dims) for i in range(dims // 2)]
    if scaling == hs.HS_ROPE_TURNS:
        share = [(CONTEXT * x / (2 * math.pi) - LOW) / (HIGH - LOW) for x in theta]
    elif scaling == hs.HS_ROPE_INDEX:
        def index(t):
            return dims * math.log(CONTEXT / (2 * math.pi * t)) / (2 * math.log(base))
        a, b = max(math.floor(index(HIGH)), 0), min(math.ceil(index(LOW)), dims - 1)
        share = [1 - (i - a) / max(b - a, 0.001) for i in range(dims // 2)]
    else:
        return theta
    return [x * min(1, max(0, s)) + x / f * (1 - min(1, max(0, s))) for x, s in zip(theta, share)]


@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
@pytest.mark.parametrize("dims", [16, 48, 64, 128])
@pytest.mark.parametrize("scaling", range(5))
def test_angles(dims, base, scaling):
    for f in (1.0, 2.0, 32.0):
        r = plan(dims, base=base, scaling=scaling, factor=f, context=CONTEXT, low=LOW, high=HIGH, amplitude=1.25)
        want = formula(dims, base, scaling, f)
        for i, x in enumerate(want):
            # pow and its arguments' roundings, twice where the base is scaled
            assert abs(r.theta[i] - x) <= x * 2.0 ** -48, i
        assert list(r.theta[dims // 2:]) == [0.0] * (hs.HS_ROPE_MAX_PAIRS - dims // 2)
        assert (r.dims, r.layout, r.amplitude) == (dims, hs.HS_ROPE_HALF, 1.25)


def test_a_factor_of_one_and_fast_and_slow_pairs():
    a = plan(128, base=10000.0)
    for scaling in (hs.HS_ROPE_TURNS, hs.HS_ROPE_INDEX):
        r = plan(128, base=10000.0, scaling=scaling, factor=8.0, context=CONTEXT, low=LOW, high=HIGH)
        assert r.theta[0] == a.theta[0] and r.theta[63] == a.theta[63] / 8.0
        # falling, and never below the divided or above the kept angle
        for i in range(64):
            assert a.theta[i] / 8.0 <= r.theta[i] <= a.theta[i]
            assert i == 0 or r.theta[i] < r.theta[i - 1]


@pytest.mark.parametrize("kw,code", [
    (dict(dims=0), INV), (dict(dims=-16), INV), (dict(dims=24), UNS), (dict(dims=144), UNS), (dict(layout=2), INV),
    (dict(layout=-1), INV), (dict(base=1.0), INV), (dict(base=0.5), INV), (dict(base=math.nan), INV),
    (dict(base=math.inf), INV), (dict(scaling=5), INV), (dict(scaling=-1), INV), (dict(amplitude=0.0), INV),
    (dict(amplitude=math.nan), INV), (dict(scaling=1, factor=0.5), INV), (dict(scaling=2, factor=math.inf), INV),
    (dict(scaling=2, base=1e300, factor=1e300), INV), (dict(scaling=1, factor=math.nan), INV),
    (dict(scaling=3, factor=2.0, context=0), INV), (dict(scaling=3, factor=2.0, context=8, low=0.0), INV),
    (dict(scaling=4, factor=2.0, context=8, low=2.0, high=2.0), INV),
    (dict(scaling=4, factor=2.0, context=8, low=1.0, high=math.inf), INV)], ids=str)
def test_plan_arguments(kw, code):
    with pytest.raises(hs.HsError) as e:
        plan(**kw)
    assert e.value.status == code


def apply(sh=None, **kw):
    a = dict(shape=sh or shape(), rope=plan(), q=FAKE, k=FAKE, in_stride=0, pos=FAKE, n_rows=4, q_out=FAKE,
             q_out_stride=0, k_out=FAKE, k_out_stride=0, stream=0)
    a.update(kw)
    hs.hs_rope_apply(**a)


def append(sh=None, **kw):
    a = dict(shape=sh or shape(), k=FAKE, v=FAKE, kv_stride=0, slots=FAKE, n_rows=4, cache=FAKE, stream=0)
    a.update(kw)
    hs.hs_kv8_append(**a)


def append_rope(sh=None, **kw):
    a = dict(shape=sh or shape(), rope=plan(), q=FAKE, k=FAKE, v=FAKE, in_stride=0, pos=FAKE, slots=FAKE, n_rows=4,
             q_out=FAKE, q_out_stride=0, cache=FAKE, stream=0)
    a.update(kw)
    hs.hs_kv8_append_rope(**a)


def decode(sh=None, **kw):
    a = dict(shape=sh or shape(), q=FAKE, cache=FAKE, block_table=FAKE, kv_len=FAKE, max_kv_len=100, o=FAKE, lse=None,
             workspace=FAKE, workspace_bytes=1 << 40, stream=0)
    a.update(kw)
    hs.hs_kv8_decode(**a)


def read(sh=None, **kw):
    a = dict(shape=sh or shape(), cache=FAKE, block_table=FAKE, kv_len=FAKE, max_kv_len=100, out=FAKE, out_blocks=64,
             out_table=FAKE, stream=0)
    a.update(kw)
    hs.hs_kv8_read(**a)


def refused(call, kw, code):
    with pytest.raises(hs.HsError) as e:
        call(**kw)
    assert e.value.status == code


def bent(**kw):
    r = plan()
    for name, x in kw.items():
        if name == "theta":
            r.theta[3] = x
        else:
            setattr(r, name, x)
    return r


ROPES = [(dict(rope=bent(dims=0)), INV), (dict(rope=bent(dims=144)), INV), (dict(rope=bent(dims=40)), UNS),
         (dict(rope=bent(layout=2)), INV), (dict(rope=bent(amplitude=-1.0)), INV),
         (dict(rope=bent(theta=math.nan)), INV), (dict(rope=bent(theta=math.inf)), INV)]


@pytest.mark.parametrize("kw,code", ROPES, ids=lambda x: "")
@pytest.mark.parametrize("call", [apply, append_rope])
def test_ropes_are_checked(call, kw, code):
    refused(call, kw, code)


def test_a_plan_wider_than_the_head_is_refused():
    for call in (apply, append_rope):
        refused(call, dict(sh=shape(head_dim=64)), INV)
        refused(call, dict(sh=shape(head_dim=64), rope=plan(64), n_rows=-1), INV)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INV), (dict(k=None), INV), (dict(q_out=None), INV), (dict(k_out=None), INV),
    (dict(q=None, q_out=None, k=None, k_out=None), INV), (dict(pos=None), INV), (dict(n_rows=-1), INV),
    (dict(in_stride=1016), INV), (dict(in_stride=-8), INV), (dict(in_stride=1028), MIS), (dict(q_out_stride=1016), INV),
    (dict(k_out_stride=248), INV), (dict(k_out_stride=260), MIS), (dict(q=FAKE + 8), MIS), (dict(k=FAKE + 2), MIS),
    (dict(q_out=FAKE + 8), MIS), (dict(k_out=FAKE + 8), MIS), (dict(pos=FAKE + 4), MIS),
    (dict(sh=shape(n_heads=7)), INV), (dict(sh=shape(n_kv_heads=0)), INV), (dict(sh=shape(dtype=2)), INV),
    (dict(sh=shape(head_dim=96)), UNS), (dict(sh=shape(n_heads=258)), UNS),
    (dict(sh=shape(n_heads=2048, n_kv_heads=2048)), UNS)], ids=str)
def test_apply_arguments(kw, code):
    refused(apply, kw, code)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INV), (dict(v=None), INV), (dict(slots=None), INV), (dict(cache=None), INV), (dict(n_rows=-1), INV),
    (dict(k=FAKE + 8), MIS), (dict(v=FAKE + 2), MIS), (dict(cache=FAKE + 4), MIS), (dict(slots=FAKE + 4), MIS),
    (dict(sh=shape(head_dim=32)), UNS), (dict(sh=shape(page_size=48)), UNS), (dict(sh=shape(dtype=-1)), INV),
    (dict(sh=shape(n_kv_heads=1025, n_heads=1025)), UNS), (dict(sh=shape(num_blocks=1 << 31)), UNS),
    (dict(n_rows=1 << 31), UNS)], ids=str)
@pytest.mark.parametrize("call", [append, append_rope])
def test_append_arguments(call, kw, code):
    refused(call, kw, code)


@pytest.mark.parametrize("kw,code", [(dict(kv_stride=-8), INV), (dict(kv_stride=248), INV), (dict(kv_stride=260), MIS)],
                         ids=str)
def test_append_strides(kw, code):
    refused(append, kw, code)


@pytest.mark.parametrize("kw,code", [
    (dict(in_stride=1016), INV), (dict(in_stride=1028), MIS), (dict(q_out_stride=1016), INV), (dict(q=None), INV),
    (dict(q_out=None), INV), (dict(pos=None), INV), (dict(pos=FAKE + 4), MIS), (dict(q=FAKE + 8), MIS),
    (dict(q_out=FAKE + 8), MIS), (dict(sh=shape(n_heads=7)), INV), (dict(sh=shape(n_heads=258)), UNS)], ids=str)
def test_append_rope_arguments(kw, code):
    refused(append_rope, kw, code)


SHAPES = [
    (dict(n_kv_heads=0), INV), (dict(n_heads=0), INV), (dict(n_heads=7), INV), (dict(batch=-1), INV),
    (dict(dtype=2), INV), (dict(num_blocks=-1), INV), (dict(max_pages=-1), INV), (dict(scale=0.0), INV),
    (dict(scale=math.inf), INV), (dict(q_stride=1016), INV), (dict(o_stride=-8), INV), (dict(unsplit=2), INV),
    (dict(head_dim=96), UNS), (dict(page_size=8), UNS), (dict(page_size=512), UNS), (dict(n_heads=258), UNS),
    (dict(batch=385), UNS), (dict(num_blocks=1 << 31), UNS), (dict(q_stride=1028), MIS)]


@pytest.mark.parametrize("kw,code", SHAPES, ids=str)
def test_decode_shapes(kw, code):
    refused(decode, dict(sh=shape(**kw)), code)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INV), (dict(cache=None), INV), (dict(block_table=None), INV), (dict(o=None), INV),
    (dict(kv_len=None), INV), (dict(q=FAKE + 8), MIS), (dict(cache=FAKE + 8), MIS), (dict(o=FAKE + 2), MIS),
    (dict(lse=FAKE + 2), MIS), (dict(block_table=FAKE + 1), MIS), (dict(kv_len=FAKE + 2), MIS),
    (dict(workspace=FAKE + 8), MIS), (dict(workspace_bytes=-1), INV), (dict(max_kv_len=-1), INV),
    (dict(max_kv_len=129), INV), (dict(sh=shape(max_pages=1 << 40), max_kv_len=1 << 31), UNS),
    (dict(sh=shape(num_blocks=0)), INV)], ids=str)
def test_decode_arguments(kw, code):
    refused(decode, kw, code)


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), INV), (dict(block_table=None), INV), (dict(out=None), INV), (dict(kv_len=None), INV),
    (dict(out_table=None), INV), (dict(cache=FAKE + 8), MIS), (dict(out=FAKE + 8), MIS), (dict(kv_len=FAKE + 2), MIS),
    (dict(block_table=FAKE + 2), MIS), (dict(out_table=FAKE + 2), MIS), (dict(max_kv_len=-1), INV),
    (dict(max_kv_len=129), INV), (dict(out_blocks=-1), INV), (dict(out_blocks=0), INV),
    (dict(sh=shape(num_blocks=0)), INV), (dict(sh=shape(batch=-1)), INV), (dict(sh=shape(batch=385)), UNS),
    (dict(sh=shape(head_dim=96)), UNS), (dict(sh=shape(max_pages=1 << 40), max_kv_len=1 << 31), UNS),
    (dict(sh=shape(max_pages=1 << 40, batch=64), max_kv_len=1 << 30), UNS)], ids=str)
def test_read_arguments(kw, code):
    refused(read, kw, code)


def test_caches_beyond_31_bits_of_rows():
    """65 rows of 128 bytes to a block: the decode step counts them in 31 bits, the other calls do not."""
    big = (1 << 31) // 65 + 1
    refused(decode, dict(sh=shape(num_blocks=big)), UNS)
    refused(decode, dict(sh=shape(num_blocks=big - 1), q=None), INV)
    refused(append, dict(sh=shape(num_blocks=big), k=None), INV)


def test_empty_calls_touch_nothing():
    apply(n_rows=0, pos=None)
    apply(n_rows=0, q=None, q_out=None, k=None, k_out=None)
    append(n_rows=0, k=None, cache=None)
    append_rope(n_rows=0, q=None, q_out=None, pos=None)
    decode(shape(batch=0), kv_len=None)
    read(shape(batch=0), kv_len=None)
    read(max_kv_len=0, cache=None)
    assert hs.hs_kv8_decode_workspace_bytes(shape(batch=0), 0) == 0


@pytest.mark.parametrize("kv_heads,page,d,want", [(4, 16, 128, 16384 + 128), (8, 32, 128, 65536 + 128),
                                                  (2, 16, 64, 4096 + 128), (1, 256, 64, 32768 + 128),
                                                  (32, 256, 128, 2 * 32 * (32768 + 64))])
def test_block_bytes(kv_heads, page, d, want):
    n = hs.hs_kv8_block_bytes(shape(n_heads=kv_heads, n_kv_heads=kv_heads, page_size=page, head_dim=d))
    assert n == want and n % 128 == 0
    refused(lambda **kw: hs.hs_kv8_block_bytes(shape(**kw)), dict(page_size=17), UNS)


def test_the_tests_own_rounding():
    """Every value is its own byte, and what lies between two goes to the nearer, ties to the even one."""
    for b in list(range(127)) + list(range(128, 255)):
        assert to_e4m3(VALUES[b:b + 1]).item() == b
    for b in range(126):
        a, c = VALUES[b].item(), VALUES[b + 1].item()
        mid = (a + c) / 2
        for x, want in ((mid, b + b % 2), (mid + (c - a) / 64, b + 1), (mid - (c - a) / 64, b)):
            assert to_e4m3(VALUES.new_tensor([x])).item() == want, (b, x)


@pytest.mark.parametrize("amplitude", [2.0 ** -21, 2.0 ** 21, 1e-300, 1e300, math.inf])
@pytest.mark.parametrize("call", [apply, append_rope])
def test_amplitudes_out_of_range(call, amplitude):
    with pytest.raises(hs.HsError) as e:
        plan(amplitude=amplitude)
    assert e.value.status == INV
    with pytest.raises(hs.HsError) as e:
        call(rope=bent(amplitude=amplitude))
    assert e.value.status == INV
    assert plan(amplitude=2.0 ** -20).amplitude == 2.0 ** -20 and plan(amplitude=2.0 ** 20).amplitude == 2.0 ** 20
