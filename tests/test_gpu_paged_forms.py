"""The forms of decode over pages that other tests do not reach, and calls at once: against the oracle of test_gpu_paged, whose bounds hold."""
import threading

import pytest
import torch

from test_gpu_paged import BF, DEV, F32, Case, _B, i32

pytestmark = pytest.mark.gpu


def bound_call(B, case, desc, ws, bound):
    """The case's step with weights, bound to buffers of its own: (call, out, weights)."""
    dev = [x.to(DEV) for x in (case.q, case.kn, case.vn, case.kp, case.vp, case.w_in)]
    out = torch.full((case.S, case.hq, case.d), float("nan"), dtype=case.dtype, device=DEV)
    w_out = torch.full_like(dev[5], 7.0)
    call = B.bind_decode_attn_paged(desc, dev[0], dev[1], dev[2], i32(case.pos), dev[3], dev[4], i32(case.table), i32(case.lens), bound,
                                    out, dev[5], w_out, ws)
    return call, out, w_out


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_setting_that_changes_during_a_call_does_not_outgrow_its_workspace(dtype):
    """Another thread sets the rows of a split back and forth: a call is refused, or gives what it gives alone; behind its workspace
    nothing is written."""
    B = _B()
    case = Case(dtype, 8, 2, 64, 16, [3000, 170])
    desc = B.make_desc(dtype, 8, 2, 64)
    B.earn_set_tuning("paged_chunk", 2048)
    try:
        need = B.earn_decode_paged_workspace_bytes(desc, 2, 3000, True)
        whole = torch.full((need + (8 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
        call, out, w_out = bound_call(B, case, desc, whole[:need], 3000)
        call()
        torch.cuda.synchronize()
        want = out.clone(), w_out.clone()
        done = threading.Event()

        def flip():
            while not done.is_set():
                B.earn_set_tuning("paged_chunk", 64)
                B.earn_set_tuning("paged_chunk", 2048)

        other = threading.Thread(target=flip)
        other.start()
        served = 0
        try:
            for _ in range(2000):
                try:
                    call()
                    served += 1
                except B.EarnError as e:
                    assert e.code == B.EARN_ERR_WORKSPACE_TOO_SMALL
        finally:
            done.set()
            other.join()
        torch.cuda.synchronize()
        assert served > 0 and torch.equal(out, want[0]) and torch.equal(w_out, want[1])
        assert (whole[need:] == 0x5A).all()
    finally:
        B.earn_set_tuning("paged_chunk", 0)


@pytest.mark.parametrize("n", [90, 1500], ids=["whole", "split"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_follow_a_softmax_that_is_nan(dtype, n):
    """Where all scores are -inf, or one is +inf or NaN, every weight of that softmax is NaN, that of a row of score -inf too; rows
    without a page weigh 0 all the same, and another kv head's sums are untouched by it."""
    B = _B()
    page, inf = 16, float("inf")
    case = Case(dtype, 2, 2, 64, page, [n] * 4)
    case.table[:, 2] = -1                                   # rows 32 .. 47 are not there
    desc = B.make_desc(dtype, 2, 2, 64, rope_base=0.0)
    case.q[:, 0] = case.q[:, 0].abs() + 0.5
    lowest = torch.finfo(dtype).min
    at = lambda u, r: (int(case.table[u, r // page]), 0, r % page)
    for r in [r for r in range(n) if r // page != 2]:
        case.kp[at(0, r)] = lowest                          # products of 64 of them overflow
        if r < 20:
            case.kp[at(1, r)] = lowest
            case.kp[at(2, r)] = lowest
            case.kp[at(3, r)] = lowest
    case.kn[0, 0] = lowest
    case.kp[at(1, n - 5)] = inf
    case.kp[at(2, 60)] = float("nan")
    out, w_out = case.run(B, True, desc=desc)
    there = torch.ones(n + 1, dtype=torch.bool)
    there[32:48] = False
    for u in range(3):
        assert torch.isnan(out[u, 0].float()).all(), u
        assert torch.equal(torch.isnan(w_out[u, 0, :n + 1].cpu()), there), u
        assert torch.equal(w_out[u, 0, 32:48].cpu(), case.w_in[u, 0, 32:48]), u
    assert torch.isfinite(out[3].float()).all() and torch.isfinite(w_out[3]).all()
    assert torch.equal(w_out[3, 0, :20].cpu(), case.w_in[3, 0, :20])       # -inf among finite scores: nothing
    assert torch.isfinite(out[:, 1].float()).all() and torch.isfinite(w_out[:, 1]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("budget", [40, 100])
def test_a_row_without_a_page_is_a_row_of_zeros_after_eviction(dtype, budget):
    """Eviction's precondition is that every row has a page.  Where one has none, it comes out as documented: zeros that the next step
    attends to (cut down to the budget, and moved whole), and the validation mode refuses the call."""
    B = _B()
    page, n = 16, 90
    case = Case(dtype, 4, 2, 64, page, [n])
    case.table[0, 2] = -1                                   # rows 32 .. 47
    desc = B.make_desc(dtype, 4, 2, 64)
    kp, vp = case.kp.to(DEV), case.vp.to(DEV)
    per = -(-(budget + 1) // page)
    m, base = min(n, budget), kp.shape[0]
    grow = lambda x: torch.cat([x, torch.full((per, 2, page, 64), float("nan"), dtype=dtype, device=DEV)])
    kp, vp = grow(kp), grow(vp)
    fresh = i32([list(range(base, base + per))])
    kept, length = torch.empty(1, 2, budget, dtype=torch.int32, device=DEV), i32([0])
    w = case.w_in.to(DEV)
    w[:, :, 30:50] += 1.0                                   # the rows that are not there are among the largest
    old = B.earn_set_validation(True)
    try:
        with pytest.raises(B.EarnError) as e:
            B.earn_cache_evict(desc, kp, vp, i32(case.table), i32([n]), n, w, budget, 2, 3, fresh, kept, length)
        assert e.value.code == B.EARN_ERR_INVALID_ARG and "page_table[0][2] = -1" in str(e.value)
    finally:
        B.earn_set_validation(old)
    B.earn_cache_evict(desc, kp, vp, i32(case.table), i32([n]), n, w, budget, 2, 3, fresh, kept, length)
    torch.cuda.synchronize()
    assert length.tolist() == [m] and set(range(32, 48)) <= set(kept[0, 0].tolist()) & set(kept[0, 1].tolist())
    after = Case(dtype, 4, 2, 64, page, [m])
    after.q, after.kn, after.vn = case.q, case.kn, case.vn
    after.n_pages = per
    after.table = torch.arange(per, dtype=torch.int32).numpy()[None]
    after.kp, after.vp = kp[base:].cpu(), vp[base:].cpu()
    for c in range(2):
        for i, r in enumerate(kept[0, c].tolist()[:m]):
            got = after.kp[i // page, c, i % page]
            assert torch.equal(got, torch.zeros(64, dtype=dtype) if 32 <= r < 48 else case.kp[int(case.table[0, r // page]), c, r % page])
    out, w_out = after.run(B, True)
    after.kp, after.vp = after.kp.nan_to_num(0.0), after.vp.nan_to_num(0.0)      # behind the last row
    after.g_kp, after.g_vp = after.g_kp.nan_to_num(0.0), after.g_vp.nan_to_num(0.0)
    after.check(out, w_out)


def whole_bound(case):
    return max(max(case.lens), 0)


def streamed_bound(case):
    """A bound by value for which the rows would exceed 256 MB, so that the bf16 kernels that keep nothing in the caches run; the rows
    themselves are few."""
    per_row = 2 * case.S * case.hkv * case.d * (2 if case.dtype == BF else 4)
    return (256 << 20) // per_row + 1


FORMS = [
    # dtype, hq, hkv, d, page, rows of the streams: groups up to 8 and more heads, both head sizes, split ...
    (BF, 14, 2, 64, 16, [1500, 2999]),
    (BF, 8, 1, 64, 8, [3000, -1, 640]),
    (BF, 9, 1, 64, 24, [2000, 1088]),
    (BF, 16, 1, 128, 16, [2000, 1089, 0]),
    (BF, 9, 1, 128, 7, [1300]),
    (BF, 20, 1, 64, 32, [1700]),                  # two workgroups for the heads of a group
    (F32, 1, 1, 64, 16, [1300, 257]),
    (F32, 2, 1, 64, 5, [1300]),
    (F32, 3, 1, 64, 16, [1290]),
    (F32, 4, 1, 128, 16, [1300, 31]),
    (F32, 2, 1, 128, 16, [1333]),
    (F32, 1, 1, 128, 64, [1301]),
    (F32, 7, 1, 64, 16, [1300]),
    (F32, 8, 1, 128, 3, [1300, 2]),
    # ... and whole, by eight waves
    (BF, 9, 1, 64, 16, [129, 400, 600]),
    (BF, 16, 1, 128, 16, [300, 512]),
    (BF, 8, 1, 64, 8, [639, 100]),
]


@pytest.mark.parametrize("weights", [False, True], ids=["plain", "weights"])
@pytest.mark.parametrize("bound_of", [whole_bound, streamed_bound])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", FORMS)
def test_every_form_of_the_decode_kernels(dtype, hq, hkv, d, page, lens, bound_of, weights):
    B = _B()
    case = Case(dtype, hq, hkv, d, page, lens)
    out, w_out = case.run(B, weights, bound=bound_of(case))
    case.check(out, w_out)


@pytest.mark.parametrize("chunk", [1, 64, 192, 2048, 100000])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", [
    (BF, 8, 2, 64, 1, [2500, 63, 64]), (BF, 16, 1, 128, 3, [2049, 0, 128]), (F32, 4, 2, 64, 1, [2100, 64]), (F32, 8, 1, 128, 16, [2048, 65])])
def test_splits_of_any_number_of_rows(dtype, hq, hkv, d, page, lens, chunk):
    """The fewest rows of a split, so that many are joined, and the most, whose pages of one row fill the list of page numbers."""
    B = _B()
    case = Case(dtype, hq, hkv, d, page, lens)
    B.earn_set_tuning("paged_chunk", chunk)
    try:
        for weights in (False, True):
            out, w_out = case.run(B, weights)
            case.check(out, w_out)
    finally:
        B.earn_set_tuning("paged_chunk", 0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_workspace_for_the_largest_call_serves_smaller_ones(dtype):
    """Sized once, with what is behind it left alone; the bound and the number of streams vary from call to call."""
    B = _B()
    desc = B.make_desc(dtype, 8, 1, 64)
    need = B.earn_decode_paged_workspace_bytes(desc, 6, 40000, True)
    whole = torch.full((need + 4096,), 255, dtype=torch.uint8, device=DEV)
    for lens, bound in (([700] * 6, 700), ([1500, 20], 1500), ([3000], 32767), ([3000, 1, 2], 40000), ([900], 900), ([100] * 5, 639)):
        case = Case(dtype, 8, 1, 64, 16, lens)
        call, out, w_out = bound_call(B, case, desc, whole[:need], bound)
        call()
        torch.cuda.synchronize()
        want, w_want = case.run(B, True, bound=bound)
        case.check(want, w_want)
        assert torch.equal(out, want) and torch.equal(w_out, w_want)
    assert (whole[need:] == 255).all()
