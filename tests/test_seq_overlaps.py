"""Stores of the operators over packed token rows that would meet are refused at creation (no GPU needed)."""
import itertools

import numpy as np
import pytest

from test_seq_ops import ATT, ROT, L, _at, _create  # noqa: F401  (L: fixture)

ES = 2
PAGES, KV, PAGE, D = 8, 2, 16, 64        # of ROT and ATT


def _refused(L, base, changes):
    rc, h = _create(L, **dict(base, **changes))
    assert rc == L.EINVAL and h.value is None, changes
    return L.load().miriam_last_error()


def _accepted(L, base, changes):
    rc, h = _create(L, **dict(base, **changes))
    assert rc == 0, (changes, L.load().miriam_last_error())
    L.load().miriam_op_destroy(h)


# ----------------------------------------------------- places of the two caches
@pytest.mark.parametrize("changes", [
    dict(v_cache=_at(3) + 8 * ES),                                   # v a few values behind k
    dict(v_cache=_at(3) + 2048 * ES),                                # a page behind it: its pages are k's next ones
    dict(v_cache=_at(3) - 2048 * ES),
    dict(v_cache=_at(3) + 1024 * ES, cache_page=4096),               # values of head 0 where the keys of head 1 lie
    dict(cache_head=8), dict(cache_page=64),                         # heads, pages that overlap
    dict(cache_head=64, cache_token=64),
    dict(cache_page=1024, cache_head=2048),                          # pages within the heads' steps, but longer than theirs
    dict(v_cache=_at(3) + 64 * ES, cache_token=96, cache_head=1600, cache_page=3200),   # interleaved, tokens too near
    dict(v_cache=_at(3) + (4096 * 3 + 2000) * ES, cache_page=4096),  # reaching into the pages it should lie between
    dict(v_cache=_at(3) - 4096 * 7 * ES, cache_page=4096),           # its last page is k's first
])
def test_caches_whose_places_overlap_are_refused(L, changes):  # noqa: F811
    assert b"overlap" in _refused(L, ROT, changes)


@pytest.mark.parametrize("changes", [
    dict(v_cache=_at(3) + PAGES * 2048 * ES),                        # one behind the other
    dict(v_cache=_at(3) - PAGES * 2048 * ES),
    dict(v_cache=_at(3) + 2048 * ES, cache_page=4096),               # keys and values of a page in turn
    dict(v_cache=_at(3) + 1024 * ES, cache_page=4096, cache_head=2048),                  # of a head
    dict(v_cache=_at(3) + 64 * ES, cache_token=128, cache_head=2048, cache_page=4096),   # of a token
    dict(v_cache=_at(3) + 128 * ES, cache_token=256, cache_head=64, cache_page=4096),    # of a token's heads
    dict(v_cache=_at(3) + (4096 * 3 + 2048) * ES, cache_page=4096),  # keys and values in turn, some pages later
    dict(v_cache=_at(3) - 4096 * 8 * ES, cache_page=4096),
    dict(cache_token=128, cache_head=64),                            # a token's heads together
    dict(cache_page=64, cache_token=512, cache_head=512 * 16),       # pages innermost
    dict(kv_heads=1, cache_head=1), dict(pages=1, cache_page=1),     # steps that nothing takes
])
def test_caches_of_their_own_places_are_accepted(L, changes):  # noqa: F811
    _accepted(L, ROT, changes)


def test_what_is_accepted_has_places_of_its_own(L):  # noqa: F811
    """Small strides and distances, place by place: what is accepted has places of its own, dense caches of such places
    are accepted, and beside a cache that is accepted any other that shares none."""
    pages, kv, page, d = 3, 2, 2, 2
    base = dict(ROT, pages=pages, kv_heads=kv, page=page, head_dim=d, rot=2, heads=2)
    grid = np.array(list(itertools.product(range(pages), range(kv), range(page))))

    def accepted(**changes):
        rc, h = _create(L, **dict(base, **changes))
        if rc == 0:
            L.load().miriam_op_destroy(h)
        return rc == 0

    pairs = interleaved = 0
    for sp, sh, st in itertools.product((2, 3, 4, 6, 8, 12, 16, 24), repeat=3):
        at = ((grid @ np.array([sp, sh, st]))[:, None] + np.arange(d)).ravel()
        strides = dict(cache_page=sp, cache_head=sh, cache_token=st)
        alone, own = accepted(**strides), len(set(at)) == len(at)       # (the other cache is far away)
        assert own or not alone, strides
        assert alone or not own or max(at) + 1 > len(at), strides
        for apart in list(range(-40, 41)) if alone else ():
            ok = accepted(**strides, v_cache=_at(3) + apart * ES)
            assert ok == (not set(at) & set(at + apart)), (strides, apart)
            pairs += ok
            interleaved += ok and abs(apart) <= max(at)
    assert pairs > 100 and interleaved > 100


# --------------------------------------------- outputs over what a pass reads
OUT = 10 * 4 * 64 * ES                   # bytes of y in ROT and ATT
CACHE = PAGES * 2048 * ES                # and of a cache


@pytest.mark.parametrize("array,size", [("q_start", 12), ("kv_len", 8), ("page_table", 2 * 4 * 4)])
@pytest.mark.parametrize("base,out,reach", [(ROT, "y", OUT), (ROT, "k_cache", CACHE), (ROT, "v_cache", CACHE), (ATT, "y", OUT)])
def test_outputs_over_the_batchs_arrays_are_refused(L, base, out, reach, array, size):  # noqa: F811
    at = base[out]
    for start in (at, at + reach - 4, at - size + 4):
        _refused(L, base, {array: start})
    for start in (at + reach, at - size):                            # right behind it, and right before
        _accepted(L, base, {array: start})


@pytest.mark.parametrize("out,reach", [("y", OUT), ("k_cache", CACHE), ("v_cache", CACHE)])
def test_outputs_over_the_frequencies_are_refused(L, out, reach):  # noqa: F811
    at, size = ROT[out], 32 * 8
    for start in (at, at + reach - 8, at - size + 8):
        _refused(L, ROT, dict(freq=start))
    for start in (at + reach, at - size):
        _accepted(L, ROT, dict(freq=start))
    _accepted(L, ROT, dict(freq=at, rot=0))                          # nothing is turned, nothing is read


def test_strided_outputs_and_tables(L):  # noqa: F811
    _refused(L, ATT, dict(page_table=_at(2) + 9 * 512 * ES, ldy=512))       # in the last row of a strided y
    _refused(L, ATT, dict(page_table=_at(2) - 400, ldt=100))                # the table's second row
    _refused(L, ATT, dict(ldt=1 << 60))
    _accepted(L, ATT, dict(kv_len=_at(3), q_start=_at(3), page_table=_at(3)))   # only read: may share memory
    _accepted(L, dict(ROT, kv_heads=0, k_cache=None, v_cache=None), dict(page_table=_at(2)))   # no cache: no table
