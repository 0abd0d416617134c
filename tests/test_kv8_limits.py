"""Host-only limits of the 8-bit cache's calls and of rotary positions (no GPU needed)."""
import pytest

import paper_2609_15030_gb300 as hs

from tests.test_kv8_host import FAKE, INV, MIS, append_rope, apply, bent, built, refused  # noqa: F401  (built: the library)


@pytest.mark.parametrize("theta", [2.0 ** 64, -2.0 ** 64, 1e300])
@pytest.mark.parametrize("call", [apply, append_rope])
def test_angles_of_2_to_the_64_and_more_are_refused(call, theta):
    refused(call, dict(rope=bent(theta=theta)), INV)


@pytest.mark.parametrize("theta", [2.0 ** 63, -2.0 ** 63, 5e-324, -1e-300])
@pytest.mark.parametrize("call", [apply, append_rope])
def test_smaller_angles_are_taken(call, theta):
    call(rope=bent(theta=theta), n_rows=0)


@pytest.mark.parametrize("page,heads,ok", [(16, 1, False), (16, 2, True), (32, 1, True), (256, 3, True)])
def test_slices_of_scales_are_multiples_of_16_bytes(page, heads, ok):
    """One KV head's scales of a page of 16 tokens are 8 bytes: a slice of them is refused, not cut."""
    shape = hs.make_attn_shape(0, 6, 6, 128, page, 4, 1)
    size = hs.hs_kv8_block_bytes(shape)
    at = 6 * 2 * page * 128 + 2 * page // 2
    for call in (hs.hs_restore_kv_page_slices, hs.hs_save_kv_page_slices):
        def slices(n_pages):
            call(FAKE, FAKE, 1, FAKE, n_pages, size, 1, at, heads * page // 2, 4, None, 0)
        if ok:
            slices(0)
        else:
            refused(lambda **kw: slices(**kw), dict(n_pages=1), MIS)
