"""Calls with a window whose cache has rows so long that no scratch can be asked for: refused before anything is launched."""
import pytest

from paper_2609_11582_b200 import binding as B
from paper_2609_11582_b200 import build as build_mod
from tests.test_paged_cpu import P16, S4, cache
from tests.test_sight_cpu import tree, window

LONG = dict(n_layers=64, batch=512, n_kv_heads=8, n_q_heads=64, max_pages=32768, n_pages=4096)


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("sight", [(5, 1), (4096, 64), (100000, 0)])
def test_rows_beyond_what_scratch_is_known_for(L, n, sight):
    """okq_paged_workspace_bytes has no size for these rows (2^31 pieces of work and more, were they full), so that no scratch is large enough:
    not even where the window itself is short."""
    c = cache(**LONG)
    assert L.okq_paged_workspace_bytes(c, 64, n) == 0 and L.okq_debug_paged_plan(c, 64, n) == 0
    w, s = sight
    for ws_bytes in (0, 16, 1 << 40):
        assert window(L, c, count=64, n=n, window=w, sinks=s, ws_bytes=ws_bytes) == B.ERR_UNSUPPORTED
        assert tree(L, c, count=64, n=n, ws_bytes=ws_bytes) == B.ERR_UNSUPPORTED
    assert L.okq_debug_paged_plan_window(c, 64, n, w, s) == 0
    # a layer at a time there is one
    need = L.okq_paged_workspace_bytes(c, 1, n)
    assert need > 0 and L.okq_debug_paged_plan_window(c, 1, n, w, s) != 0
    assert window(L, c, count=1, n=n, window=w, sinks=s, ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_refusals_of_the_testing_aid(L):
    c = cache()
    go = lambda window=0, sinks=0, seen=0, limit=1000, c=c: L.okq_debug_paged_timeout_sight(c, 0, 1, P16, S4, 1, window, sinks, seen, P16, 1 << 30, P16, S4,  # noqa: E731
                                                                                            limit, None)
    assert go() == go(window=-1) == go(window=5, sinks=-1) == go(window=5, seen=P16) == go(window=5, limit=0) == go(window=5, c=None) == B.ERR_INVALID_ARG
    assert go(seen=P16 + 4) == B.ERR_ALIGNMENT
