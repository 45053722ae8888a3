"""Sizes and arguments of the calls over pages, decided on the host: no kernel is launched, no GPU needed."""
import pytest

from paper_2507_00715_amd import binding as B

HEADS = [(B.EARN_BF16, 12, 2, 128), (B.EARN_BF16, 8, 1, 64), (B.EARN_BF16, 34, 2, 64), (B.EARN_BF16, 32, 32, 128), (B.EARN_F32, 4, 4, 64),
         (B.EARN_F32, 12, 1, 128)]


def desc_of(dtype, hq, hkv, d):
    return B.AttnDesc(dtype, hq, hkv, d, None, 0.0, 10000.0)


def rows_around(steps):
    return sorted({max(0, s + o) for s in steps for o in (-65, -64, -63, -33, -32, -31, -2, -1, 0, 1, 2, 31, 32, 33, 63, 64, 65)})


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("chunk", [0, 64, 100, 2048])
def test_a_decode_workspace_serves_every_smaller_call(heads, weights, chunk):
    """A program sizes the workspace once, for its largest batch and cache; no smaller batch or bound may ask for more."""
    desc = desc_of(*heads)
    streams = [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 33, 63, 64, 65, 66, 100, 127, 128, 129, 200, 255, 256, 257, 300, 511, 512, 513, 4000]
    rows = rows_around([0, 100, 640, 1024, 1088, 2048, 2176, 3264, 4096, 8192, 16384, 32768, 65536, 131072, 278528, 557056, 65535 * 64,
                        65535 * 1088])
    rows = [r for r in rows if r <= 1 << 26]
    B.earn_set_tuning("paged_chunk", chunk)
    try:
        most = [0] * len(rows)                       # of fewer streams, at this bound or a smaller one
        for n in streams:
            so_far = 0
            for i, r in enumerate(rows):
                need = B.earn_decode_paged_workspace_bytes(desc, n, r, weights)
                so_far = max(so_far, most[i])
                assert need >= so_far, f"{n} streams, bound {r}: {need} bytes, {so_far} for something smaller"
                assert need <= B.earn_decode_paged_workspace_bytes(desc, n, r, True)
                most[i] = so_far = need
    finally:
        B.earn_set_tuning("paged_chunk", 0)


def test_the_decode_workspace_at_sizes_where_a_smaller_call_asked_for_more():
    desc = desc_of(B.EARN_BF16, 12, 2, 128)
    need = [B.earn_decode_paged_workspace_bytes(desc, 1, r, False) for r in (32767, 32895, 40000)]
    assert need == sorted(need) and need[0] > 0
    desc = desc_of(B.EARN_BF16, 8, 1, 64)
    for weights in (False, True):
        assert B.earn_decode_paged_workspace_bytes(desc, 64, 1024, weights) <= B.earn_decode_paged_workspace_bytes(desc, 65, 1024, weights)


WRONG_KINDS = """
import torch
from paper_2507_00715_amd import binding as B
assert_is_off = True
assert not assert_is_off                      # python -O: this line does nothing
bf, i = torch.bfloat16, lambda *s: torch.zeros(*s, dtype=torch.int32)
z = lambda *s: torch.zeros(*s, dtype=bf)
desc = B.make_desc(bf, 4, 2, 64)
pools = dict(k_pages=z(4, 2, 16, 64), v_pages=z(4, 2, 16, 64))
store = dict(k=z(5, 2, 64), v=z(5, 2, 64), cu_seqlens=i(2), start=i(1), page_table=i(1, 2), **pools)
decode = dict(q=z(1, 4, 64), k_new=z(1, 2, 64), v_new=z(1, 2, 64), q_pos=i(1), page_table=i(1, 2), cache_len=i(1), max_cache_len=31,
              out=z(1, 4, 64), weights_in=torch.zeros(1, 2, 32), weights_out=torch.zeros(1, 2, 32), **pools)
evict = dict(page_table=i(1, 2), cache_len=i(1), max_cache_len=31, weights=torch.zeros(1, 2, 32), budget=9, n_first=0, n_last=0,
             new_table=i(1, 1), kept_out=i(1, 2, 9), len_out=i(1), weights_out=torch.zeros(1, 2, 9), **pools)
sample = dict(logits=torch.zeros(2, 9), uniform=torch.zeros(2), token_out=i(2), top_k=i(2), top_p=torch.zeros(2))
wrong = 0
def refused(call, good, **bad):
    global wrong
    try:
        call(**dict(good, **bad))
        text = "accepted"
    except AssertionError:
        return
    except Exception as e:
        text = repr(e)
    wrong += 1
    print(call, list(bad), text)
for name in ("cu_seqlens", "start", "page_table"):
    refused(lambda **kw: B.earn_cache_store(desc, **kw), store, **{name: store[name].long()})
for name, x in (("k", z(5, 4, 64)), ("v", z(4, 2, 64)), ("k", store["k"].float()), ("cu_seqlens", i(3)), ("start", i(2)), ("v_pages", z(4, 2, 8, 64)),
                ("k_pages", z(4, 1, 16, 64)), ("k_pages", pools["k_pages"].float())):
    refused(lambda **kw: B.earn_cache_store(desc, **kw), store, **{name: x})
for call in (B.earn_decode_attn_paged, B.bind_decode_attn_paged):
    for name in ("q_pos", "page_table", "cache_len"):
        refused(lambda **kw: call(desc, **kw), decode, **{name: decode[name].long()})
    for name, x in (("q", z(1, 2, 64)), ("out", z(2, 4, 64)), ("k_new", z(1, 4, 64)), ("q", decode["q"].float()), ("cache_len", i(2)),
                    ("weights_out", decode["weights_out"].double()), ("weights_in", torch.zeros(1, 2, 31))):
        refused(lambda **kw: call(desc, **kw), decode, **{name: x})
for name in ("page_table", "cache_len", "new_table", "kept_out", "len_out"):
    refused(lambda **kw: B.earn_cache_evict(desc, **kw), evict, **{name: evict[name].long()})
for name, x in (("new_table", i(2, 1)), ("new_table", i(1)), ("kept_out", i(1, 2, 8)), ("len_out", i(2)), ("weights", torch.zeros(1, 64)),
                ("weights_out", torch.zeros(2, 2, 9)), ("weights", evict["weights"].double())):
    refused(lambda **kw: B.earn_cache_evict(desc, **kw), evict, **{name: x})
for name, x in (("token_out", i(2).long()), ("top_k", i(2).long()), ("uniform", torch.zeros(2).double()), ("uniform", torch.zeros(1)), ("top_p", torch.zeros(3))):
    refused(B.earn_sample, sample, **{name: x})
raise SystemExit(1 if wrong else 0)
"""


@pytest.mark.parametrize("flags", [[], ["-O"]], ids=["plain", "optimised"])
def test_wrong_types_and_shapes_are_refused_without_asserts_too(flags):
    """A table of 64-bit numbers would be read as 32-bit ones: the checks stay where Python drops its assert statements."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    source = WRONG_KINDS if flags else WRONG_KINDS.replace("assert not assert_is_off", "pass")
    r = subprocess.run([sys.executable, *flags, "-c", source], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]


FAKE = 1 << 20     # never dereferenced: the calls are refused


def test_sums_that_overlap_their_source_are_refused():
    """A call that reads sums while another of its threads writes them has no defined result, whatever part of them overlaps."""
    import ctypes
    desc = desc_of(B.EARN_BF16, 4, 2, 64)
    S, rows, budget = 2, 100, 64
    for other in (FAKE + 4, FAKE - 4, FAKE + S * 2 * rows * 4 - 4, FAKE - S * 2 * rows * 4 + 4):
        rc = B.lib().earn_decode_attn_paged(ctypes.byref(desc), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, S, 7, 9, 16, rows, FAKE, other,
                                            rows, FAKE, FAKE, 1 << 40, None)
        assert rc == B.EARN_ERR_INVALID_ARG and "overlap" in B.last_error(), (rc, B.last_error())
    # what only touches, or is the same, passes on to the next check (here: of the workspace)
    for other in (FAKE, FAKE + S * 2 * rows * 4, FAKE - S * 2 * rows * 4):
        rc = B.lib().earn_decode_attn_paged(ctypes.byref(desc), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, S, 7, 9, 16, rows, FAKE, other,
                                            rows, FAKE, None, 0, None)
        assert rc == B.EARN_ERR_WORKSPACE_TOO_SMALL, (rc, B.last_error())
    for other in (FAKE, FAKE + 4, FAKE + S * 2 * rows * 4 - 4, FAKE - S * 2 * budget * 4 + 4):
        rc = B.lib().earn_cache_evict(ctypes.byref(desc), FAKE, FAKE, FAKE, FAKE, S, 10, 40, 16, rows, FAKE, rows, budget, 4, 8, FAKE, 4, FAKE, FAKE,
                                      other, budget, None, 0, None)
        assert rc == B.EARN_ERR_INVALID_ARG and "overlap" in B.last_error(), (rc, B.last_error())
