"""Host-only limits of the 8-bit cache's calls and of rotary positions (no GPU needed)."""
import pytest

from tests.test_kv8_host import INV, append_rope, apply, bent, built, refused  # noqa: F401  (built: the library)


@pytest.mark.parametrize("theta", [2.0 ** 64, -2.0 ** 64, 1e300])
@pytest.mark.parametrize("call", [apply, append_rope])
def test_angles_of_2_to_the_64_and_more_are_refused(call, theta):
    refused(call, dict(rope=bent(theta=theta)), INV)


@pytest.mark.parametrize("theta", [2.0 ** 63, -2.0 ** 63, 5e-324, -1e-300])
@pytest.mark.parametrize("call", [apply, append_rope])
def test_smaller_angles_are_taken(call, theta):
    call(rope=bent(theta=theta), n_rows=0)
