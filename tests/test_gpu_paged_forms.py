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
