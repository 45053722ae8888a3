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
