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
