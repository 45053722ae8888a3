"""Refusals of the calls over pages and of the sampler: decided on the host, no kernel is launched, no GPU needed."""
import ctypes

import numpy as np
import pytest

from oracle import earn_oracle as O
from paper_2507_00715_amd import binding as B

FAKE = 256     # never dereferenced: validation fails first


def _desc(dtype=B.EARN_BF16, hq=4, hkv=2, d=64):
    return B.AttnDesc(dtype, hq, hkv, d, None, 0.0, 10000.0)


def refused(rc, code, needle=""):
    assert rc == code and needle in B.last_error(), (rc, B.last_error())


def test_store_refusals():
    def call(desc=None, k=FAKE, cu=FAKE, batch=2, total=8, pages=FAKE, table=FAKE, max_pages=4, n_pages=9, page=16):
        return B.lib().earn_cache_store(ctypes.byref(desc or _desc()), k, FAKE, cu, None, batch, total, pages, FAKE, table, max_pages,
                                        n_pages, page, None)

    refused(call(desc=_desc(d=32)), B.EARN_ERR_UNSUPPORTED, "head_dim")
    refused(call(desc=_desc(dtype=3)), B.EARN_ERR_UNSUPPORTED, "dtype")
    for kw in (dict(batch=0), dict(total=-1), dict(k=None), dict(cu=None), dict(pages=None), dict(table=None), dict(max_pages=0),
               dict(n_pages=0), dict(page=0), dict(page=-16), dict(pages=264), dict(k=264)):
        refused(call(**kw), B.EARN_ERR_INVALID_ARG, "earn_cache_store")
    assert call(total=0, k=None) == B.EARN_OK


def test_decode_refusals():
    def call(desc=None, q=FAKE, S=2, pages=FAKE, table=FAKE, length=FAKE, page=16, bound=100, w_in=None, w_out=None, w_rows=0, out=FAKE,
             ws=FAKE, ws_bytes=1 << 40):
        return B.lib().earn_decode_attn_paged(ctypes.byref(desc or _desc()), q, FAKE, FAKE, FAKE, pages, FAKE, table, length, S, 4, 9,
                                              page, bound, w_in, w_out, w_rows, out, ws, ws_bytes, None)

    refused(call(desc=_desc(hq=5)), B.EARN_ERR_INVALID_ARG, "multiple")
    refused(call(desc=_desc(hq=129, hkv=1)), B.EARN_ERR_UNSUPPORTED, "query heads")
    refused(call(S=70000), B.EARN_ERR_UNSUPPORTED, "streams")
    for kw in (dict(q=None), dict(S=0), dict(pages=None), dict(table=None), dict(length=None), dict(page=0), dict(bound=-1),
               dict(bound=(1 << 26) + 1), dict(w_in=FAKE), dict(w_out=FAKE), dict(out=None), dict(q=264), dict(out=258)):
        refused(call(**kw), B.EARN_ERR_INVALID_ARG, "earn_decode_attn_paged")
    need = B.earn_decode_paged_workspace_bytes(_desc(), 2, 100000, False)
    more = B.earn_decode_paged_workspace_bytes(_desc(), 2, 100000, True)
    assert more > need + 2 * 4 * 100000 * 4 > 0
    refused(call(bound=100000, ws_bytes=need - 1), B.EARN_ERR_WORKSPACE_TOO_SMALL)
    refused(call(bound=100000, ws=None), B.EARN_ERR_WORKSPACE_TOO_SMALL)
    refused(call(bound=100000, ws=272), B.EARN_ERR_INVALID_ARG, "aligned")
    refused(call(bound=100000, w_out=FAKE, w_rows=10, ws_bytes=more - 1), B.EARN_ERR_WORKSPACE_TOO_SMALL)
    assert B.earn_decode_paged_workspace_bytes(_desc(d=96), 2, 100, False) == 0
    assert B.earn_decode_paged_workspace_bytes(_desc(hq=32, hkv=32), 64, 50, False) == 0


def test_evict_refusals():
    def call(desc=None, pages=FAKE, length=FAKE, S=2, bound=100, w=FAKE, w_rows=100, budget=64, first=4, last=8, fresh=FAKE, new_pages=4,
             kept=FAKE, len_out=FAKE, w_out=None, w_rows_out=0):
        return B.lib().earn_cache_evict(ctypes.byref(desc or _desc()), pages, FAKE, FAKE, length, S, 10, 40, 16, bound, w, w_rows, budget,
                                        first, last, fresh, new_pages, kept, len_out, w_out, w_rows_out, None, 0, None)

    refused(call(desc=_desc(d=256)), B.EARN_ERR_UNSUPPORTED, "head_dim")
    for kw in (dict(pages=None), dict(length=None), dict(S=0), dict(bound=-1), dict(w=None), dict(w_rows=99), dict(budget=0), dict(budget=(1 << 26) + 1, new_pages=1 << 30), dict(first=-1),
               dict(last=-1), dict(first=60), dict(fresh=None), dict(new_pages=3), dict(kept=None), dict(len_out=None), dict(w_out=FAKE),
               dict(w_out=512, w_rows_out=63)):
        refused(call(**kw), B.EARN_ERR_INVALID_ARG, "earn_cache_evict")


def test_sample_refusals():
    def call(logits=FAKE, dtype=B.EARN_F32, stride=100, rows=2, vocab=100, u=FAKE, token=FAKE):
        return B.lib().earn_sample(logits, dtype, stride, rows, vocab, None, None, None, None, u, token, None, None, FAKE, 1 << 40, None)

    refused(call(dtype=2), B.EARN_ERR_UNSUPPORTED, "dtype")
    refused(call(vocab=524289, stride=524289), B.EARN_ERR_UNSUPPORTED, "vocab")
    refused(call(rows=(1 << 21) + 1), B.EARN_ERR_UNSUPPORTED, "rows")
    for kw in (dict(logits=None), dict(logits=258), dict(stride=99), dict(rows=-1), dict(vocab=0), dict(u=None), dict(token=None)):
        refused(call(**kw), B.EARN_ERR_INVALID_ARG, "earn_sample")
    assert call(rows=0, logits=None) == B.EARN_OK


# ---- the oracles against statements of their own ----
def test_paged_oracle_equals_the_contiguous_one():
    rng = np.random.default_rng(0)
    S, hq, hkv, d, page, n = 3, 4, 2, 64, 5, [13, 0, 20]
    table = rng.permutation(12).reshape(3, 4).astype(np.int32)
    table = np.hstack([table, np.array([[12], [13], [14]], dtype=np.int32)])
    kp, vp = rng.standard_normal((15, hkv, page, d)), rng.standard_normal((15, hkv, page, d))
    q, kn, vn = (rng.standard_normal((S, h, d)) for h in (hq, hkv, hkv))
    rows = [[(table[u, r // page], r % page) for r in range(n[u])] for u in range(S)]
    shared = lambda p: np.array([p[a, :, b] for u in range(S) for a, b in rows[u]])
    cu = np.concatenate([[0], np.cumsum(n)])
    gk, gv = np.zeros((S, 1, hkv, d)), np.zeros((S, 1, hkv, d))
    pos = [30, 4, 21]
    want = O.decode_attn(q, kn, vn, pos, shared(kp), shared(vp), cu, list(range(S)), gk, gv, [0] * S)
    got = O.paged_decode(q, kn, vn, pos, kp, vp, table, n)
    np.testing.assert_allclose(got["out"], want["out"], rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(got["key"], gk[:, 0], rtol=1e-13, atol=1e-14)
    np.testing.assert_allclose([p.sum(1) for p in got["probs"]], 1.0, rtol=1e-12)


def test_evict_oracle_by_hand():
    w = np.array([[[5, 1, 3, 3, 9, 0, 3, np.nan]]], dtype=np.float32)
    assert O.cache_evict(w, [8], 4, 0, 1) == [[[0, 2, 4, 7]]]
    assert O.cache_evict(w, [8], 5, 1, 0) == [[[0, 2, 3, 4, 6]]]
    assert O.cache_evict(w, [7], 7, 1, 0) == [[[0, 1, 2, 3, 4, 5, 6]]]
    assert O.cache_evict(w, [8], 8, 0, 0)[0][0] == list(range(8)) and O.cache_evict(w, [-1], 4, 0, 0) == [[[]]]


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.24, 0), (0.26, 2), (0.49, 2), (0.51, 3), (0.99, 3)])
def test_sample_oracle_by_hand(u, token):
    l = np.log(np.array([1.0, 0.5, 1.0, 2.0, 0.25]))
    got = O.sample_token(l, u, top_k=4, top_p=0.8)       # 2 + 1 + 1 of 4.5 reach 3.6
    assert (got["token"], got["n_kept"]) == (token, 3) and abs(got["logprob"] - np.log([0.25, 0, 0.25, 0.5][token])) < 1e-12
    assert O.sample_token(l, u, min_p=0.4)["n_kept"] == 3 and O.sample_token(l, u, temperature=0.0)["token"] == 3
