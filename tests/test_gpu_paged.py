"""Caches in pages against the fp64 oracle: storing a prefill's rows, decode over pages with running weight sums, eviction by
those sums.

Bounds of the decode tests, from the arithmetic of the kernels.  A base-2 score is a sum of d products of fp32 numbers in fp32
(the rotated query is a rotation by angles that are off by less than 2^-20, then scaled): it is off by at most
(d + 32) 2^-24 t log2 e, t the largest sum of the magnitudes of a row's terms.  A weight is a quotient of two exponentials of
such scores: off by a factor 2^(2 err) at most, and by a few fp32 roundings (2^-20 covers exp2, sums over lanes, splits and
heads).  Outputs are sums of weights times values, rounded once to their type: half a step, finfo.eps / 2.
"""
import numpy as np
import pytest
import torch

from oracle import earn_oracle as O
from paper_2507_00715_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _B():
    from paper_2507_00715_amd import binding
    binding.lib()
    return binding


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def tables(rows, page, rng, spare=2, width=None):
    """Page tables for streams of `rows` rows each, pages in random order; -1 behind a stream's last page."""
    need = [-(-max(r, 0) // page) for r in rows]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    width = max(max(need), 1) if width is None else width
    table = np.full((len(rows), width), -1, dtype=np.int32)
    at = 0
    for u, m in enumerate(need):
        table[u, :m] = order[at:at + m]
        at += m
    return table, n_pages, order[at:]


class Case:
    """Inputs of a decode step; lens: rows of every stream, -1 an idle one."""

    def __init__(self, dtype, hq, hkv, d, page, lens, seed=0, room=None, k_scale=1.0):
        self.dtype, self.hq, self.hkv, self.d, self.page, self.lens = dtype, hq, hkv, d, page, list(lens)
        g = torch.Generator().manual_seed(seed + sum(lens) + page)
        rng = np.random.default_rng(seed + page)
        self.S = len(lens)
        self.rnd = lambda *s: torch.randn(*s, generator=g).to(dtype)
        self.table, self.n_pages, self.spare = tables([n + 1 if n >= 0 else 0 for n in lens] if room is None else room, page, rng)
        self.kp, self.vp = self.rnd(self.n_pages, hkv, page, d) * k_scale, self.rnd(self.n_pages, hkv, page, d)
        self.q, self.kn, self.vn = self.rnd(self.S, hq, d), self.rnd(self.S, hkv, d), self.rnd(self.S, hkv, d)
        self.pos = [max(n, 0) + 3 + 11 * u for u, n in enumerate(lens)]
        self.rows = max(max(lens), 0) + 5
        self.w_in = torch.rand(self.S, hkv, self.rows, generator=g)

    def run(self, B, weights, desc=None, w_in=True, bound=None, in_place=False):
        dev = lambda x: x.to(DEV)
        desc = desc or B.make_desc(self.dtype, self.hq, self.hkv, self.d)
        self.g_kp, self.g_vp = dev(self.kp), dev(self.vp)
        out = torch.full((self.S, self.hq, self.d), float("nan"), dtype=self.dtype, device=DEV)
        w_out = w_dev = None
        if weights:
            w_dev = dev(self.w_in) if w_in else None
            w_out = w_dev if in_place else torch.full((self.S, self.hkv, self.rows), 7.0, device=DEV)
        bound = max(max(self.lens), 0) if bound is None else bound
        need = B.earn_decode_paged_workspace_bytes(desc, self.S, bound, weights)
        ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device=DEV)        # NaN wherever it is read unwritten
        B.earn_decode_attn_paged(desc, dev(self.q), dev(self.kn), dev(self.vn), i32(self.pos), self.g_kp, self.g_vp,
                                 i32(self.table), i32(self.lens), bound, out, w_dev, w_out, ws)
        torch.cuda.synchronize()
        return out, w_out

    def check(self, out, w_out, w_in=True, in_place=False, **oracle):
        """Against the oracle, which attends the new key as the pages hold it."""
        S, hkv, d, page = self.S, self.hkv, self.d, self.page
        kp, vp = W.to_f64(self.kp), W.to_f64(self.vp)
        free = O.paged_decode(W.to_f64(self.q), W.to_f64(self.kn), W.to_f64(self.vn), self.pos, kp, vp, self.table, self.lens,
                              **oracle)
        half_step = torch.finfo(self.dtype).eps / 2
        stored = free["key"].copy()
        k_want, v_want = self.kp.clone(), self.vp.clone()
        for u, n in enumerate(self.lens):
            if n < 0:
                continue
            at = int(self.table[u, n // page]) if n // page < self.table.shape[1] else -1
            if not 0 <= at < self.n_pages:
                if self.dtype == BF:       # not stored: as the kernel rounds it, up to a tie
                    stored[u] = W.to_f64(torch.from_numpy(free["key"][u]).float().to(BF))
                continue
            got = self.g_kp[at, :, n % page].cpu()
            k_want[at, :, n % page], v_want[at, :, n % page] = got, self.vn[u]
            big = np.abs(free["key"][u]).max()
            assert (np.abs(W.to_f64(got) - free["key"][u]) <= np.abs(free["key"][u]) * half_step * 1.001 + big * 2.0 ** -18).all(), u
            stored[u] = W.to_f64(got)
        same = lambda a, b: torch.equal(a.cpu().view(torch.int16 if self.dtype == BF else torch.int32),
                                        b.view(torch.int16 if self.dtype == BF else torch.int32))
        assert same(self.g_kp, k_want) and same(self.g_vp, v_want), "pages hold something else than the appended rows"
        ref = O.paged_decode(W.to_f64(self.q), W.to_f64(self.kn), W.to_f64(self.vn), self.pos, kp, vp, self.table, self.lens,
                             stored_key=stored, **oracle)
        got = W.to_f64(out)
        group = self.hq // hkv
        heads = oracle.get("q_to_kv") or [a // group for a in range(self.hq)]
        for u, n in enumerate(self.lens):
            if n < 0:
                assert (got[u] == 0).all(), "an idle stream's outputs"
                if w_out is not None:
                    assert torch.equal(w_out[u].cpu(), self.w_in[u] if in_place else torch.full_like(self.w_in[u], 7.0))
                continue
            err = (d + 32) * 2.0 ** -24 * ref["terms"][u] * np.log2(np.e)
            factor = np.exp2(2 * err) - 1 + 2.0 ** -20
            for a in range(self.hq):
                v, there = O.paged_rows(vp, self.table[u], heads[a], n)
                v = np.vstack([v, W.to_f64(self.vn)[u, heads[a]]])
                bar = (ref["probs"][u][a][:, None] * np.abs(v)).sum(0) * factor[a]
                bar = bar + (np.abs(ref["out"][u, a]) + bar) * half_step + 1e-30
                worst = np.abs(got[u, a] - ref["out"][u, a]) / bar
                assert worst.max() <= 1, f"stream {u}, head {a}: {worst.max():.3g} of the bound"
            if w_out is None:
                continue
            w = w_out[u].cpu().double().numpy()
            old = self.w_in[u].double().numpy() if w_in else np.zeros(self.w_in[u].shape)
            m = min(n + 1, self.rows)
            for c in range(hkv):
                mine = [a for a in range(self.hq) if heads[a] == c]
                add = np.array([ref["probs"][u][a] for a in mine])
                want = add.sum(0)
                had = min(n, self.rows)
                want[:had] += old[c, :had]
                bar = (add * factor[mine][:, None]).sum(0) + want * 2.0 ** -22 + 1e-30
                assert (np.abs(w[c, :m] - want[:m]) <= bar[:m]).all(), f"stream {u}, kv head {c}: weights"
                rest = self.w_in[u, c, m:].numpy() if in_place else np.full(self.rows - m, 7.0, dtype=np.float32)
                assert (w_out[u, c, m:].cpu().numpy() == rest).all(), "rows behind the last one"


DECODE = [
    # dtype, hq, hkv, d, page, rows of the streams
    (F32, 4, 4, 64, 16, [0, 1, 15, 16, 17, 97]),
    (F32, 8, 2, 128, 5, [0, 63, 64, 65, 320]),
    (F32, 7, 1, 64, 1, [33, 2]),
    (F32, 12, 1, 128, 8, [1, 130, -1]),
    (F32, 40, 2, 64, 32, [200]),
    (BF, 4, 4, 64, 16, [0, 1, 2, 15, 16, 17, 31, 32, 33, 127]),
    (BF, 14, 2, 64, 16, [500, -1, 3, 0]),
    (BF, 32, 8, 128, 64, [0, 63, 64, 65, 1000]),
    (BF, 12, 2, 128, 7, [6, 7, 8, 259, 1]),
    (BF, 3, 3, 128, 1, [40, 0]),
    (BF, 16, 1, 128, 256, [255, 256, 257]),
    (BF, 9, 1, 64, 3, [77, -1]),
    (BF, 34, 2, 64, 8, [90, 0]),
    (BF, 130, 10, 64, 16, [50]),
    (BF, 8, 8, 128, 128, [3000, 9]),
    (F32, 2, 2, 64, 64, [2500, 130]),
    (BF, 12, 2, 128, 33, [9001]),
    (F32, 6, 2, 128, 48, [5003, 0, 4096]),
]


@pytest.mark.parametrize("weights", [False, True], ids=["plain", "weights"])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", DECODE)
def test_decode_over_pages(dtype, hq, hkv, d, page, lens, weights):
    B = _B()
    case = Case(dtype, hq, hkv, d, page, lens)
    out, w_out = case.run(B, weights)
    case.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_stream_of_a_long_cache_is_split_and_joined(dtype):
    """The bound passed by value may be far above the lengths; the result does not depend on it but for rounding."""
    B = _B()
    case = Case(dtype, 12, 2, 128, 16, [1311])
    for bound in (1311, 1312, 20000, 300000):
        out, w_out = case.run(B, True, bound=bound)
        case.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_in_place_from_zero_and_cut_to_their_rows(dtype):
    B = _B()
    case = Case(dtype, 8, 2, 64, 16, [300, 5, -1, 70])
    out, w_out = case.run(B, True, in_place=True)
    case.check(out, w_out, in_place=True)
    out, w_out = case.run(B, True, w_in=False)
    case.check(out, w_out, w_in=False)
    case.rows = 64                       # fewer sums than rows
    case.w_in = case.w_in[:, :, :64].contiguous()
    out, w_out = case.run(B, True)
    case.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_map_scale_and_no_rotation(dtype):
    B = _B()
    q_to_kv = [1, 0, 0, 1, 1, 0]
    case = Case(dtype, 6, 2, 64, 16, [130, 40])
    desc = B.make_desc(dtype, 6, 2, 64, softmax_scale=0.37, rope_base=0.0, q_to_kv=q_to_kv)
    out, w_out = case.run(B, True, desc=desc)
    case.check(out, w_out, scale=0.37, rope_base=0.0, q_to_kv=q_to_kv)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_without_a_page_weigh_nothing(dtype):
    """Entries outside the pool, in the middle and at the place of the new row; a table that is full."""
    B = _B()
    case = Case(dtype, 4, 2, 128, 16, [100, 70, 64, 33])
    case.table[0, [1, 3]] = [-1, case.n_pages]       # two pages in the middle
    case.table[1, :4] = -5                           # all but the last, partly filled one
    case.table[2, 4] = 1 << 30                       # the new row has no place
    case.table[3, :] = -1                            # nothing but the new token
    out, w_out = case.run(B, True)
    case.check(out, w_out)
    full = Case(dtype, 4, 2, 128, 16, [48, 20], room=[48, 48])
    out, w_out = full.run(B, True)                   # stream 0 fills its table: attended, not stored
    full.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 24])
def test_holes_of_eight_rows_within_a_block(dtype, d, page):
    """Pages missing inside the 32 rows that are read together, at each place of them."""
    B = _B()
    case = Case(dtype, 4, 2, d, page, [96, 100, 32, 192])
    case.table[0, [0, 2]] = -1
    case.table[1, [1, 3]] = [case.n_pages, -7]
    case.table[2, 1] = -1
    case.table[3, 1:7] = -1
    out, w_out = case.run(B, True)
    case.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_streams_share_pages(dtype):
    B = _B()
    case = Case(dtype, 8, 2, 64, 16, [100, 90, 64])
    case.table[1, :4] = case.table[0, :4]
    case.table[2, :4] = case.table[0, :4]
    out, w_out = case.run(B, True)
    case.check(out, w_out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_lies_behind_a_stream_is_not_read(dtype):
    """NaN and infinities in the rest of the last page, in other pages and in unused weights leave no trace."""
    B = _B()
    case = Case(dtype, 8, 2, 128, 32, [100, 31, 0])
    plain, w_plain = case.run(B, True)
    used = np.zeros((case.n_pages, 32), dtype=bool)
    for u, n in enumerate(case.lens):
        for r in range(n):
            used[case.table[u, r // 32], r % 32] = True
    for pages, x in ((case.kp, float("nan")), (case.vp, float("inf"))):
        pages.transpose(1, 2)[~torch.from_numpy(used)] = x
    out, w_out = case.run(B, True)
    assert torch.equal(out, plain) and torch.equal(w_out, w_plain)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 64])
def test_infinite_and_nan_rows_give_what_fp32_gives(dtype, page):
    """A key that is infinite in one element gives a score of either infinity: -inf weighs nothing, +inf or NaN makes the
    row of the softmax NaN; an infinite value comes through in its own element."""
    B = _B()
    case = Case(dtype, 4, 2, 64, page, [150, 150, 150])
    desc = B.make_desc(dtype, 4, 2, 64, rope_base=0.0)
    kp, vp = case.kp, case.vp
    at = lambda u, r: (int(case.table[u, r // page]), slice(None), r % page)
    kp[at(0, 40)][:, 7] = float("inf")
    vp[at(1, 77)][:, 5] = float("-inf")
    kp[at(2, 3)][:, 1] = float("nan")
    out, w_out = case.run(B, True, desc=desc)
    q = case.q.float()
    for a in range(4):
        if q[0, a, 7] > 0:
            assert torch.isnan(out[0, a]).all()
        else:
            assert torch.isfinite(out[0, a].float()).all()
    want = torch.zeros(64, dtype=torch.bool)
    want[5] = True
    assert (torch.isinf(out[1].float().cpu()) == want).all() and (out[1, :, 5].float() < 0).all()
    assert torch.isnan(out[2].float()).all() and torch.isfinite(w_out[1]).all()


@pytest.mark.parametrize("weights", [False, True])
def test_large_scores_and_masks_of_the_lowest_value(weights):
    """Scores of some hundred (one key dominates); keys of the type's lowest value, whose scores overflow to -inf."""
    B = _B()
    case = Case(BF, 4, 2, 64, 16, [200, 90], k_scale=30.0)
    out, w_out = case.run(B, weights)
    case.check(out, w_out)
    case = Case(F32, 4, 2, 64, 16, [90])
    desc = B.make_desc(F32, 4, 2, 64, rope_base=0.0)
    case.q.abs_()
    rows = [int(case.table[0, r // 16]) * 16 + r % 16 for r in range(5, 40)]
    case.kp.transpose(1, 2).reshape(-1, 2, 64)[rows] = torch.finfo(F32).min
    kp = case.kp.transpose(1, 2).reshape(-1, 2, 64)
    kp[rows] = torch.finfo(F32).min
    case.kp = kp.view(case.n_pages, 16, 2, 64).transpose(1, 2).contiguous()
    out, w_out = case.run(B, True, desc=desc)
    assert torch.isfinite(out).all() and (w_out[0, :, 5:40].cpu() == case.w_in[0, :, 5:40]).all()


def test_pool_beyond_32_bit_offsets():
    """Pools of 4.3 GB each: the rows lie behind the first 2^32 bytes and 2^31 elements."""
    B = _B()
    n_pages, hkv, page, d = 8200, 16, 128, 128
    kp = torch.zeros(n_pages, hkv, page, d, dtype=BF, device=DEV)
    vp = torch.zeros_like(kp)
    small = Case(BF, 16, 16, 128, 128, [300, 40])
    table = n_pages - 1 - np.where(small.table >= 0, small.table, n_pages)
    small.table = np.where(small.table >= 0, table, -1).astype(np.int32)
    order = [n_pages - 1 - i for i in range(small.n_pages)]
    kp[order], vp[order] = small.kp.to(DEV), small.vp.to(DEV)
    out = torch.empty(2, 16, 128, dtype=BF, device=DEV)
    desc = B.make_desc(BF, 16, 16, 128)
    B.earn_decode_attn_paged(desc, small.q.to(DEV), small.kn.to(DEV), small.vn.to(DEV), i32(small.pos), kp, vp, i32(small.table),
                             i32(small.lens), 300, out)
    torch.cuda.synchronize()
    small.table = np.where(small.table >= 0, n_pages - 1 - small.table, -1).astype(np.int32)
    small.g_kp, small.g_vp = kp[order], vp[order]
    small.check(out, None)
    fresh = i32([[n_pages - 100 - 4 * u - i for i in range(2)] for u in range(2)])
    kept, length = torch.empty(2, 16, 200, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    table = i32(np.where(small.table >= 0, n_pages - 1 - small.table, -1))
    B.earn_cache_evict(desc, kp, vp, table, i32(small.lens), 300, torch.rand(2, 16, 320, device=DEV), 200, 4, 9, fresh, kept, length)
    assert length.tolist() == [200, 40]
    for c in (0, 15):
        rows = kept[0, c].long()
        old = kp[table[0, rows // 128].long(), c, rows % 128]
        new = torch.cat([kp[fresh[0, 0], c], kp[fresh[0, 1], c]])[:200]
        assert torch.equal(old, new)


STORE = [
    (F32, 4, 64, 16, [96, 128], None),
    (BF, 2, 128, 32, [1, 0, 31, 32, 33, 100], [0, 5, 7, 31, 32, 60]),
    (BF, 3, 64, 7, [20, 1, 0], [3, 0, 0]),
    (F32, 1, 128, 1, [9, 4], [0, 2]),
]


@pytest.mark.parametrize("dtype,hkv,d,page,lens,start", STORE)
def test_store(dtype, hkv, d, page, lens, start):
    B = _B()
    rng = np.random.default_rng(page)
    g = torch.Generator().manual_seed(page)
    first = start or [0] * len(lens)
    table, n_pages, _ = tables([n + s for n, s in zip(lens, first)], page, rng)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total = int(cu[-1])
    k, v = (torch.randn(total + 4, hkv, d, generator=g).to(dtype) for _ in range(2))   # four rows behind the last sequence
    kp, vp = (torch.randn(n_pages, hkv, page, d, generator=g).to(dtype) for _ in range(2))
    want_k, want_v = kp.float().numpy(), vp.float().numpy()
    table[0, -1] = -1 if len(lens) == 2 else table[0, -1]           # a page that is missing: those rows are dropped
    O.paged_store(k.float().numpy(), v.float().numpy(), cu, start, want_k, want_v, table)
    gk, gv = kp.to(DEV), vp.to(DEV)
    desc = B.make_desc(dtype, hkv, hkv, d)
    B.earn_cache_store(desc, k.to(DEV), v.to(DEV), i32(cu), None if start is None else i32(start), gk, gv, i32(table))
    torch.cuda.synchronize()
    assert np.array_equal(gk.float().cpu().numpy(), want_k) and np.array_equal(gv.float().cpu().numpy(), want_v)


EVICT = [
    # dtype, hkv, d, page, rows, budget, first, last
    (BF, 2, 128, 16, [100, 64, 65, 63, 0, -1, 1], 64, 4, 8),
    (F32, 4, 64, 8, [50, 51, 200], 50, 0, 0),
    (BF, 1, 64, 32, [1000, 3000], 33, 1, 32),          # nothing but the protected rows
    (BF, 3, 128, 5, [77, 12], 12, 12, 0),
    (F32, 2, 128, 64, [2049, 1024, 5000], 1000, 10, 100),
    (BF, 8, 64, 128, [40000, 33000], 4096, 32, 256),
    (BF, 2, 64, 1, [9, 2], 1, 0, 0),
    (F32, 2, 64, 16, [30, 7], 100, 3, 3),               # within the budget: moved whole
]


def weight_kinds(rng, shape):
    yield "spread", np.exp(4 * rng.standard_normal(shape)).astype(np.float32)
    yield "ties", np.round(rng.random(shape) * 4).astype(np.float32) / 4
    yield "equal", np.full(shape, 0.25, dtype=np.float32)
    odd = rng.standard_normal(shape).astype(np.float32)
    pick = rng.integers(0, 8, shape)
    for i, x in enumerate([np.nan, np.inf, -np.inf, 0.0, -0.0]):
        odd[pick == i] = x
    yield "odd", odd


@pytest.mark.parametrize("dtype,hkv,d,page,lens,budget,first,last", EVICT)
def test_evict(dtype, hkv, d, page, lens, budget, first, last):
    B = _B()
    rng = np.random.default_rng(budget)
    g = torch.Generator().manual_seed(budget)
    S, bound = len(lens), max(lens)
    table, n_pages, spare = tables(lens, page, rng, spare=S * -(-budget // page) + 1)
    fresh = spare[:-1].reshape(S, -1)
    kp, vp = (torch.randn(n_pages, hkv, page, d, generator=g).to(dtype) for _ in range(2))
    desc = B.make_desc(dtype, hkv, hkv, d)
    rows = bound + 3
    for kind, w in weight_kinds(rng, (S, hkv, rows)):
        kept_ref = O.cache_evict(w, lens, budget, first, last)
        gk, gv = kp.to(DEV), vp.to(DEV)
        kept = torch.full((S, hkv, budget), -9, dtype=torch.int32, device=DEV)
        w_out = torch.full((S, hkv, budget + 2), 7.0, device=DEV)
        length = i32(lens)
        B.earn_cache_evict(desc, gk, gv, i32(table), length, bound, torch.from_numpy(w).to(DEV), budget, first, last, i32(fresh),
                           kept, length, w_out)          # lengths in place
        torch.cuda.synchronize()
        assert length.tolist() == [min(n, budget) for n in lens]
        want_k, want_v = kp.clone(), vp.clone()
        want = np.full((S, hkv, budget), -1)
        want_w = np.full((S, hkv, budget + 2), 7.0, dtype=np.float32)
        for u in range(S):
            for c in range(hkv):
                r = np.array(kept_ref[u][c], dtype=np.int64)
                m = len(r)
                want[u, c, :m], want_w[u, c, :m] = r, w[u, c, r]
                i = np.arange(m)
                want_k[fresh[u, i // page], c, i % page] = kp[table[u, r // page], c, r % page]
                want_v[fresh[u, i // page], c, i % page] = vp[table[u, r // page], c, r % page]
        assert np.array_equal(kept.cpu().numpy(), want), kind
        assert np.array_equal(w_out.cpu().numpy(), want_w, equal_nan=True), kind
        assert torch.equal(gk.cpu(), want_k) and torch.equal(gv.cpu(), want_v), kind
        w_none = torch.full_like(kept, -9)
        B.earn_cache_evict(desc, gk, gv, i32(table), i32(lens), bound, torch.from_numpy(w).to(DEV), budget, first, last, i32(fresh),
                           w_none, length)               # without weights_out
        assert torch.equal(w_none, kept)


def test_evict_of_rows_without_a_page():
    """Rows that have no page are kept or not by their weights like others, as zeros; a new page outside the pool takes nothing."""
    B = _B()
    kp = torch.randn(8, 2, 16, 64, device=DEV)
    vp = torch.randn_like(kp)
    before = kp.clone()
    w = torch.rand(1, 2, 64, device=DEV)
    kept, length = torch.empty(1, 2, 32, dtype=torch.int32, device=DEV), i32([0])
    B.earn_cache_evict(B.make_desc(F32, 2, 2, 64), kp, vp, i32([[0, 99, -1, 3]]), i32([64]), 64, w, 32, 0, 0, i32([[5, -4]]), kept, length)
    torch.cuda.synchronize()
    for c in range(2):
        rows = kept[0, c].tolist()
        assert rows == sorted(torch.topk(w[0, c], 32).indices.tolist())
        for i, r in enumerate(rows[:16]):
            want = before[[0, 0, 0, 3][r // 16], c, r % 16] if r // 16 in (0, 3) else torch.zeros(64, device=DEV)
            assert torch.equal(kp[5, c, i], want)
    for page in (0, 1, 2, 3, 4, 6, 7):
        assert torch.equal(kp[page], before[page])
