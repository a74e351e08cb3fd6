"""The largest pools: n_pages * H * page < 2^32 rows, for pages of any size (no GPU needed; no rows, so nothing is launched)."""
import pytest

from test_paged_refusals import UNSUPPORTED, append, attention, gather, step


@pytest.mark.parametrize("page", [8, 16, 24, 40, 128, 136, 1000])
@pytest.mark.parametrize("H,k", [(1, 1), (3, 2), (32, 8)])
@pytest.mark.parametrize("f", [attention, step, append, gather])
def test_largest_pool(f, H, k, page):
    most = (2 ** 32 - 1) // (H * page)
    sizes = {"B": 0, "H": H, "k": k, "page": page, "max_blocks": 16}
    assert f(n_pages=most, **sizes) == 0
    assert f(n_pages=most + 1, **sizes) == UNSUPPORTED
