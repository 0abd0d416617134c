"""Host-only checks of the full-attention calls: every argument error is reported before any CUDA
call, and what is empty returns without one (no GPU needed)."""
import math
import time

import pytest

import paper_2609_15030_gb300 as hs

FAKE = 1 << 20        # a 16-byte aligned non-null address that is never dereferenced
SHAPE = dict(batch=2, n_heads=8, n_kv_heads=2, head_dim=128, page_size=16, num_blocks=64, max_pages=8)
INV, MIS, UNS = hs.HS_ERR_INVALID_ARG, hs.HS_ERR_MISALIGNED, hs.HS_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_15030_gb300 import build
    build.build()


def shape(**kw):
    return hs.make_attn_shape(**{**SHAPE, **kw})


def append(sh=None, **kw):
    a = dict(shape=sh or shape(), k=FAKE, v=FAKE, kv_stride=0, slots=FAKE, n_rows=4, cache=FAKE,
             stream=0)
    a.update(kw)
    hs.hs_kv_append(**a)


def prefill(sh=None, **kw):
    a = dict(shape=sh or shape(), q=FAKE, cache=FAKE, block_table=FAKE, o=FAKE, lse=None, pos0=[0, 5],
             n_tokens=[3, 4], cu_rows=[0, 3, 7], workspace=FAKE, workspace_bytes=1 << 40, stream=0)
    a.update(kw)
    hs.hs_attn_prefill(**a)


def decode(sh=None, **kw):
    a = dict(shape=sh or shape(), q=FAKE, cache=FAKE, block_table=FAKE, kv_len=FAKE, max_kv_len=100,
             o=FAKE, lse=None, workspace=FAKE, workspace_bytes=1 << 40, stream=0)
    a.update(kw)
    hs.hs_attn_decode(**a)


def shared(sh=None, **kw):
    a = dict(shape=sh or shape(), q=FAKE, cache=FAKE, prefix_table=FAKE, prefix_len=50,
             block_table=FAKE, kv_len=FAKE, max_kv_len=100, o=FAKE, lse=None, workspace=FAKE,
             workspace_bytes=1 << 40, stream=0)
    a.update(kw)
    hs.hs_attn_decode_shared(**a)


SHAPES = [
    (dict(n_kv_heads=0), INV), (dict(n_heads=0), INV), (dict(n_heads=7), INV), (dict(batch=-1), INV),
    (dict(dtype=2), INV), (dict(num_blocks=-1), INV), (dict(max_pages=-1), INV),
    (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=math.inf), INV),
    (dict(scale=math.nan), INV), (dict(q_stride=1016), INV), (dict(o_stride=-8), INV),
    (dict(unsplit=2), INV), (dict(page_size=0), INV),
    (dict(head_dim=96), UNS), (dict(page_size=8), UNS), (dict(page_size=24), UNS),
    (dict(page_size=512), UNS), (dict(n_heads=258), UNS), (dict(batch=385), UNS),
    (dict(num_blocks=1 << 31), UNS), (dict(q_stride=1028), MIS), (dict(o_stride=1025), MIS),
]


@pytest.mark.parametrize("kw,code", SHAPES, ids=str)
@pytest.mark.parametrize("call", [prefill, decode, shared])
def test_shapes_are_checked(call, kw, code):
    none = dict(pos0=[], n_tokens=[], cu_rows=[]) if call is prefill and kw.get("batch") == -1 else {}
    with pytest.raises(hs.HsError) as e:
        call(shape(**kw), **none)
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INV), (dict(v=None), INV), (dict(slots=None), INV), (dict(cache=None), INV),
    (dict(n_rows=-1), INV), (dict(kv_stride=-8), INV), (dict(kv_stride=128), INV),
    (dict(kv_stride=260), MIS), (dict(k=FAKE + 8), MIS), (dict(v=FAKE + 2), MIS),
    (dict(cache=FAKE + 4), MIS), (dict(slots=FAKE + 4), MIS),
    (dict(sh=shape(head_dim=32)), UNS), (dict(sh=shape(page_size=48)), UNS),
    (dict(sh=shape(dtype=-1)), INV)], ids=str)
def test_append_arguments(kw, code):
    with pytest.raises(hs.HsError) as e:
        append(**kw)
    assert e.value.status == code


POINTERS = [(dict(q=None), INV), (dict(cache=None), INV), (dict(block_table=None), INV),
            (dict(o=None), INV), (dict(q=FAKE + 8), MIS), (dict(cache=FAKE + 8), MIS),
            (dict(o=FAKE + 2), MIS), (dict(lse=FAKE + 2), MIS), (dict(block_table=FAKE + 1), MIS),
            (dict(workspace=FAKE + 8), MIS), (dict(workspace_bytes=-1), INV)]


@pytest.mark.parametrize("kw,code", POINTERS, ids=str)
@pytest.mark.parametrize("call", [prefill, decode, shared])
def test_pointers_are_checked(call, kw, code):
    with pytest.raises(hs.HsError) as e:
        call(**kw)
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(pos0=[0, -1]), INV), (dict(n_tokens=[3, -1]), INV), (dict(n_tokens=[4, 4]), INV),
    (dict(cu_rows=[0, 3, 2]), INV), (dict(cu_rows=[-1, 3, 7]), INV),
    (dict(pos0=[0, 125]), INV),                                     # beyond the table's pages
    (dict(cu_rows=[0, 3, 1 << 30], n_tokens=[3, 4]), hs.HS_OK),
    (dict(cu_rows=[0, 1 << 29, (1 << 29) + 4]), UNS),
    (dict(sh=shape(max_pages=1 << 31), pos0=[0, (1 << 31) - 4]), UNS),
    (dict(sh=shape(max_pages=1 << 40), pos0=[0, 1 << 41]), INV)], ids=str)
def test_prefill_lengths_are_checked(kw, code):
    if code == hs.HS_OK:        # large gaps are fine: refused for another reason
        kw, code = dict(kw, q=None), INV
    with pytest.raises(hs.HsError) as e:
        prefill(**kw)
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(max_kv_len=-1), INV), (dict(max_kv_len=129), INV), (dict(kv_len=None), INV),
    (dict(sh=shape(max_pages=1 << 40), max_kv_len=1 << 31), UNS)], ids=str)
@pytest.mark.parametrize("call", [decode, shared])
def test_decode_lengths_are_checked(call, kw, code):
    with pytest.raises(hs.HsError) as e:
        call(**kw)
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [(dict(prefix_len=-1), INV), (dict(prefix_table=None), INV),
                                     (dict(prefix_len=1 << 31), UNS)], ids=str)
def test_prefixes_are_checked(kw, code):
    with pytest.raises(hs.HsError) as e:
        shared(**kw)
    assert e.value.status == code


@pytest.mark.parametrize("call,kw", [(decode, dict(kv_len=FAKE + 2)), (shared, dict(kv_len=FAKE + 1)),
                                     (shared, dict(prefix_table=FAKE + 2))], ids=str)
def test_device_arrays_of_lengths_and_blocks_are_aligned(call, kw):
    with pytest.raises(hs.HsError) as e:
        call(**kw)
    assert e.value.status == MIS


def test_a_prefill_of_too_many_tiles_is_refused_at_once():
    """384 requests of 8 M row tiles each: the count stops where 31 bits are exceeded."""
    batch, n = 384, (1 << 31) // 128 - (1 << 14)
    sh = shape(batch=batch, n_heads=128, n_kv_heads=1, max_pages=1 << 30)
    start = time.monotonic()
    try:
        hs.hs_attn_prefill_workspace_bytes(sh, [0] * batch, [n] * batch)
        status = hs.HS_OK
    except hs.HsError as e:
        status = e.status
    assert status in (UNS, hs.HS_ERR_CUDA)        # HS_ERR_CUDA: without a device
    assert time.monotonic() - start < 1


def test_nothing_to_do_needs_no_gpu():
    append(n_rows=0)
    append(n_rows=0, k=None, v=None, slots=None, cache=None)
    prefill(n_tokens=[0, 0], cu_rows=[0, 0, 0], q=None, o=None, cache=None, block_table=None)
    prefill(shape(batch=0), pos0=[], n_tokens=[], cu_rows=[0])
    decode(shape(batch=0), q=None, kv_len=None)
    shared(shape(batch=0), q=None, prefix_table=None)
    assert hs.hs_attn_prefill_workspace_bytes(shape(), [0, 9], [0, 0]) == 0
    assert hs.hs_attn_decode_workspace_bytes(shape(batch=0), 100) == 0


@pytest.mark.parametrize("call,args", [
    (hs.hs_attn_prefill_workspace_bytes, ([0, 0], [1, 1])), (hs.hs_attn_decode_workspace_bytes, (50,)),
    (hs.hs_attn_decode_shared_workspace_bytes, (20, 50))], ids=["prefill", "decode", "shared"])
def test_workspace_sizes_check_their_arguments(call, args):
    for kw, code in SHAPES:
        if kw.get("batch") == -1 and isinstance(args[0], list):
            continue        # the binding has no lists of -1 lengths
        with pytest.raises(hs.HsError) as e:
            call(shape(**kw), *args)
        assert e.value.status == code, kw


def test_the_binding_lays_the_shape_out_as_the_header_does():
    """Sizes and offsets of the C struct: int32 x 6, int64 x 4, float, int32."""
    f = {n: getattr(hs.hs_attn_shape, n).offset for n, _ in hs.hs_attn_shape._fields_}
    assert f == dict(batch=0, n_heads=4, n_kv_heads=8, head_dim=12, page_size=16, dtype=20,
                     num_blocks=24, max_pages=32, q_stride=40, o_stride=48, scale=56, unsplit=60)
