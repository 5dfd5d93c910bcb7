"""The calls for drafted tokens refuse addresses off their entries' own size (CPU: they return before any GPU work)."""
import pytest

FAKE = 1 << 20  # an address that no call below gets to use


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


def _filled(a, names, **kw):
    for n in names:
        setattr(a, n, FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


VERIFY = dict(probs=4, draft_probs=2, ids=8, cu_q=4, drafts=4, accept=4, sample=4, accepted=4, rejected=4, next=8)


@pytest.mark.parametrize("name", list(VERIFY))
def test_verification_refuses_addresses_off_their_entries(sp, name):
    for off in range(1, VERIFY[name]):
        for rows in (3, 0):
            a = _filled(sp.SpVerifyArgs(), VERIFY, stride=100, draft_stride=100, rows=rows, vocab=100, requests=1, dtype=1, draft_dtype=0)
            setattr(a, name, FAKE + off)
            assert sp._lib.sp_verify_drafts(a, None) == 3, (off, rows)
            a.requests = 0
            assert sp._lib.sp_verify_drafts(a, None) == 0


RETRACT = ("cached", "drop", "table", "free_pages", "free_count", "next_count", "lens", "status")


@pytest.mark.parametrize("name", RETRACT)
@pytest.mark.parametrize("requests", [2, 0])
def test_taking_tokens_back_refuses_addresses_off_their_entries(sp, name, requests):
    for off in (1, 2, 3):
        a = _filled(sp.SpKvRetractArgs(), RETRACT, pages=4, requests=requests, width=2, page_size=16)
        setattr(a, name, FAKE + off)
        assert sp._lib.sp_kv_retract(a, None) == 3, off
