"""Limits of the 8-bit cache's calls, on the host (no GPU needed)."""
import pytest

import paper_2604_09603_amd as pkg
from tests.test_q8_checks import UNSUPPORTED, _attn, _commit, _lib, _store  # noqa: F401 (_lib: a fixture)


def test_most_kv_heads_of_the_attention():
    """32 rows of new values are addressed with 32-bit offsets: 31 rows of 2^19 heads and the last
    chunk of one more stay below 2^32, of 2^19 + 1 heads and on they are not tried."""
    most = 1 << 19
    assert 31 * most * 256 + 256 < 1 << 32
    kw = dict(num_pages=1, page_size=32, max_rows=0, ws_bytes=1 << 60)
    assert _attn(hkv=most, hq=most, **kw) == pkg.OK
    assert _attn(hkv=most + 1, hq=most + 1, **kw) == UNSUPPORTED
    assert _attn(hkv=1 << 20, hq=1 << 20, **kw) == UNSUPPORTED


@pytest.mark.parametrize("call,kw", [(_store, dict(num_rows=0)), (_commit, dict(k_new=None))])
def test_most_kv_heads_of_the_writers(call, kw):
    assert call(hkv=(1 << 20) + 1, **kw) == UNSUPPORTED
    assert call(hkv=1 << 20, **kw) != UNSUPPORTED
