"""The operators over pages as a serving program uses them: a whole loop against the oracle, captured graphs, two streams of
work at once, the checks of device-side preconditions."""
import numpy as np
import pytest
import torch

from oracle import earn_oracle as O
from paper_2507_00715_amd import workloads as W
from parity import check_attn
from test_gpu_paged import BF, DEV, F32, Case, _B, i32, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 8, 2, 64), (F32, 4, 4, 64), (BF, 12, 2, 128)])
def test_generate_evict_and_go_on(dtype, hq, hkv, d):
    """Prompts go to pages (in two pieces), tokens are generated with running weight sums, caches that outgrow the budget are
    cut down to it, generation goes on; every token is drawn from logits that the attention's outputs give.  The oracle keeps
    plain lists of rows per stream and head and never sees a page; it is told the tokens' keys and values alone."""
    B = _B()
    page, budget, first, last, steps, vocab = 16, 40, 2, 6, 14, 500
    lens = [37, 30, 12]
    S = len(lens)
    g = torch.Generator().manual_seed(d + hq)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype)
    desc = B.make_desc(dtype, hq, hkv, d)
    per = -(-(max(lens) + steps) // page)
    n_pages = 2 * S * per
    free = list(np.random.default_rng(0).permutation(n_pages))
    take = lambda: i32([[int(free.pop()) for _ in range(per)] for _ in range(S)])
    kp, vp = torch.zeros(n_pages, hkv, page, d, dtype=dtype, device=DEV), torch.zeros(n_pages, hkv, page, d, dtype=dtype, device=DEV)
    table = take()
    k, v = rnd(sum(lens), hkv, d), rnd(sum(lens), hkv, d)      # as a prefill leaves them: keys rotated
    cu = np.concatenate([[0], np.cumsum(lens)])
    cut = [n // 3 for n in lens]
    pick = lambda a, b: torch.cat([torch.arange(int(cu[u]) + a[u], int(cu[u]) + b[u]) for u in range(S)])
    for a, b in (([0] * S, cut), (cut, lens)):
        rows = pick(a, b)
        B.earn_cache_store(desc, k[rows].to(DEV), v[rows].to(DEV), i32(np.concatenate([[0], np.cumsum(np.array(b) - a)])), i32(a), kp, vp,
                           table)
    keys = [[[W.to_f64(k[r, c]) for r in range(cu[u], cu[u + 1])] for c in range(hkv)] for u in range(S)]
    values = [[[W.to_f64(v[r, c]) for r in range(cu[u], cu[u + 1])] for c in range(hkv)] for u in range(S)]
    sums = torch.zeros(S, hkv, per * page, device=DEV)
    cache_len, pos = i32(lens), i32(lens)
    head = torch.randn(hq * d, vocab, generator=g) / np.sqrt(hq * d) * 8
    ws = torch.empty(max(B.earn_decode_paged_workspace_bytes(desc, S, per * page - 1, True), 1), dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(1)
    evicted = 0
    for step in range(steps):
        q, kn, vn = rnd(S, hq, d), rnd(S, hkv, d), rnd(S, hkv, d)
        out = torch.empty(S, hq, d, dtype=dtype, device=DEV)
        B.earn_decode_attn_paged(desc, q.to(DEV), kn.to(DEV), vn.to(DEV), pos, kp, vp, table, cache_len, per * page - 1, out, sums, sums, ws)
        at = [lens[u] + step for u in range(S)]
        qr, kr = O.rope(W.to_f64(q), at), O.rope(W.to_f64(kn), at)
        want = np.zeros((S, hq, d))
        for u in range(S):
            for c in range(hkv):
                keys[u][c].append(W.to_f64(torch.from_numpy(kr[u, c]).to(dtype)))
                values[u][c].append(W.to_f64(vn[u, c]))
                for a in range(c * (hq // hkv), (c + 1) * (hq // hkv)):
                    s = np.array(keys[u][c]) @ qr[u, a] / np.sqrt(d)
                    e = np.exp(s - s.max())
                    want[u, a] = (e / e.sum()) @ np.array(values[u][c])
        check_attn(out, want, dtype, f"step {step}")
        # a token of every stream
        logits = (out.float().cpu().reshape(S, -1) @ head).to(DEV)
        u_now = rng.random(S).astype(np.float32)
        token, logprob = torch.empty(S, dtype=torch.int32, device=DEV), torch.empty(S, device=DEV)
        B.earn_sample(logits, torch.from_numpy(u_now).to(DEV), token, top_p=torch.full((S,), 0.9, device=DEV), logprob_out=logprob)
        for u in range(S):
            ref = O.sample_token(logits[u].cpu().numpy(), float(u_now[u]), top_p=float(np.float32(0.9)))
            assert ref["margin"] > vocab * 2.0 ** -43 and int(token[u]) == ref["token"]
        cache_len += 1
        pos += 1
        if int(cache_len.max()) > budget + 4:
            evicted += 1
            fresh = take()
            kept = torch.empty(S, hkv, budget, dtype=torch.int32, device=DEV)
            new_sums = torch.zeros_like(sums)
            w = sums.cpu().numpy()
            ref = O.cache_evict(w, cache_len.tolist(), budget, first, last)
            B.earn_cache_evict(desc, kp, vp, table, cache_len, int(cache_len.max()), sums, budget, first, last, fresh, kept, cache_len, new_sums)
            for u in range(S):
                for c in range(hkv):
                    r = ref[u][c]
                    assert kept[u, c, :len(r)].tolist() == r
                    keys[u][c], values[u][c] = [keys[u][c][i] for i in r], [values[u][c][i] for i in r]
                    np.testing.assert_array_equal(new_sums[u, c, :len(r)].cpu().numpy(), w[u, c, r])
            free.extend(table.flatten().tolist())
            table, sums = fresh, new_sums
    assert evicted >= 2 and max(len(x) for u in range(S) for x in keys[u]) <= budget + 5


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step_replays_as_the_eager_one(dtype):
    """Decode with weights, eviction and sampling recorded into a graph, lengths and tables read at every replay: the program changes
    them between the replays, along with eager work and synchronisations."""
    B = _B()
    from paper_2507_00715_amd.pipeline import capture_graph
    hq, hkv, d, page, bound, budget, vocab, S = 8, 2, 64, 16, 159, 48, 700, 3
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).to(DEV)
    rng = np.random.default_rng(5)
    table_np, n_pages, spare = tables([160] * S, page, rng, spare=S * 3 + 1)
    table, fresh = i32(table_np), i32(spare[:-1].reshape(S, 3))
    kp, vp, q, kn, vn = rnd(n_pages, hkv, page, d), rnd(n_pages, hkv, page, d), rnd(S, hq, d), rnd(S, hkv, d), rnd(S, hkv, d)
    desc = B.make_desc(dtype, hq, hkv, d)
    cache_len, pos, u = i32([0] * S), i32([0] * S), torch.zeros(S, device=DEV)
    out, w_in = torch.empty(S, hq, d, dtype=dtype, device=DEV), torch.rand(S, hkv, 160, generator=g).to(DEV)
    w_out, w_new = torch.zeros(S, hkv, 160, device=DEV), torch.zeros(S, hkv, budget, device=DEV)
    kept, length = torch.zeros(S, hkv, budget, dtype=torch.int32, device=DEV), i32([0] * S)
    logits = torch.randn(S, vocab, generator=g).to(DEV) * 3
    token, logprob = i32([0] * S), torch.zeros(S, device=DEV)
    top_p = torch.full((S,), 0.8, device=DEV)
    ws = torch.empty(max(B.earn_decode_paged_workspace_bytes(desc, S, bound, True), 1), dtype=torch.uint8, device=DEV)
    outputs = (out, w_out, w_new, kept, length, token, logprob, kp, vp)

    def calls():
        B.earn_decode_attn_paged(desc, q, kn, vn, pos, kp, vp, table, cache_len, bound, out, w_in, w_out, ws)
        B.earn_cache_evict(desc, kp, vp, table, cache_len, bound, w_out, budget, 2, 8, fresh, kept, length, w_new)
        B.earn_sample(logits, u, token, top_p=top_p, logprob_out=logprob)

    start = kp.clone(), vp.clone()

    def set_to(lens, uniform):
        kp.copy_(start[0]), vp.copy_(start[1])
        cache_len.copy_(i32(lens)), pos.copy_(i32([max(n, 0) + 5 for n in lens])), u.copy_(torch.tensor(uniform))
        for t in (out, w_out, w_new, kept, length, token, logprob):
            t.fill_(7)

    set_to([3, 4, 5], [0.1, 0.2, 0.3])
    calls()
    torch.cuda.synchronize()
    graph = capture_graph([calls])
    for lens, uniform in (([100, 0, 159], [0.3, 0.9, 0.01]), ([47, 48, 49], [0.5, 0.6, 0.7]), ([-1, 159, 20], [0.99, 0.0, 0.4]), ([100, 0, 159], [0.2, 0.8, 0.5])):
        set_to(lens, uniform)
        calls()
        torch.cuda.synchronize()
        eager = [t.clone() for t in outputs]
        set_to(lens, uniform)
        torch.randn(1 << 20, device=DEV).sum().item()          # the program's own work
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs, eager):
            assert torch.equal(a, b)


def test_two_streams_of_work_at_once():
    """Two decode calls and two draws on streams of their own, each with its own workspace, overlapping: each gives what it gives
    alone, to the bit."""
    B = _B()
    cases = [Case(BF, 8, 2, 128, 16, [3000, 20, 700], seed=1), Case(F32, 4, 4, 64, 32, [2000, 1500], seed=2)]
    alone = [c.run(B, True) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    logits = [torch.randn(40, 30000, generator=torch.Generator().manual_seed(i)).to(DEV) * 2 for i in range(2)]
    u = torch.rand(40, generator=torch.Generator().manual_seed(9)).to(DEV)
    tokens = [[torch.empty(40, dtype=torch.int32, device=DEV) for _ in range(3)] for _ in cases]
    for i in range(2):
        B.earn_sample(logits[i], u, tokens[i][2], top_p=torch.full((40,), 0.9, device=DEV))
    prepared = []
    for c in cases:
        desc = B.make_desc(c.dtype, c.hq, c.hkv, c.d)
        dev = [x.to(DEV) for x in (c.q, c.kn, c.vn, c.kp, c.vp, c.w_in)]
        ws = torch.empty(B.earn_decode_paged_workspace_bytes(desc, c.S, max(c.lens), True), dtype=torch.uint8, device=DEV)
        out, w_out = torch.empty(c.S, c.hq, c.d, dtype=c.dtype, device=DEV), torch.full_like(dev[5], 7.0)
        prepared.append((B.bind_decode_attn_paged(desc, dev[0], dev[1], dev[2], i32(c.pos), dev[3], dev[4], i32(c.table), i32(c.lens),
                                                  max(c.lens), out, dev[5], w_out, ws), out, w_out))
    top_p = torch.full((40,), 0.9, device=DEV)
    torch.cuda.synchronize()
    for turn in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                prepared[i][0]()
                B.earn_sample(logits[i], u, tokens[i][turn % 2], top_p=top_p)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(prepared[i][1], alone[i][0]) and torch.equal(prepared[i][2], alone[i][1])
        assert torch.equal(tokens[i][0], tokens[i][2]) and torch.equal(tokens[i][1], tokens[i][2])


def test_repeated_calls_give_the_same_bits():
    B = _B()
    case = Case(BF, 12, 2, 128, 16, [5000, 33])
    first = case.run(B, True)
    for _ in range(3):
        again = case.run(B, True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_device_side_preconditions_in_the_validation_mode():
    B = _B()
    z = lambda *s: torch.zeros(*s, dtype=BF, device=DEV)
    desc = B.make_desc(BF, 4, 2, 64)
    kp, vp = z(9, 2, 16, 64), z(9, 2, 16, 64)
    out = torch.full((2, 4, 64), 7.0, dtype=BF, device=DEV)
    old = B.earn_set_validation(True)

    def refused(fn, needle):
        with pytest.raises(B.EarnError) as e:
            fn()
        assert e.value.code == B.EARN_ERR_INVALID_ARG and needle in str(e.value), str(e.value)
        torch.cuda.synchronize()
        assert (out == 7.0).all() and (kp == 0).all() and (vp == 0).all()

    try:
        def decode(table=((0, 1, 2), (3, 4, 5)), lens=(20, 40), pos=(1, 2), bound=47):
            B.earn_decode_attn_paged(desc, z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), i32(pos), kp, vp, i32(table), i32(lens), bound, out)
        refused(lambda: decode(lens=(20, 48)), "more than the bound")
        refused(lambda: decode(lens=(20, 48), bound=60), "hold")
        refused(lambda: decode(table=((0, 9, 2), (3, 4, 5))), "outside")
        refused(lambda: decode(table=((0, -1, 2), (3, 4, 5))), "outside")
        refused(lambda: decode(table=((0, 1, 2), (3, 4, 1))), "written")
        refused(lambda: decode(pos=(-1, 2)), "q_pos")

        def store(cu=(0, 20, 50), start=(0, 0), table=((0, 1, 2), (3, 4, 5))):
            B.earn_cache_store(desc, z(50, 2, 64), z(50, 2, 64), i32(cu), i32(start), kp, vp, i32(table))
        refused(lambda: store(cu=(0, 30, 20)), "decreases")
        refused(lambda: store(start=(-1, 0)), "negative")
        refused(lambda: store(start=(0, 20)), "hold")
        refused(lambda: store(table=((0, 77, 2), (3, 4, 5))), "outside")
        refused(lambda: store(table=((0, 3, 2), (3, 4, 5))), "written")

        def evict(table=((0, 1, 2), (3, 4, 2)), lens=(40, 40), fresh=((5, 6), (7, 8)), bound=48):
            B.earn_cache_evict(desc, kp, vp, i32(table), i32(lens), bound, torch.zeros(2, 2, 48, device=DEV), 20, 1, 1, i32(fresh),
                               torch.zeros(2, 2, 20, dtype=torch.int32, device=DEV), i32([0, 0]))
        refused(lambda: evict(lens=(40, 49)), "more than the bound")
        refused(lambda: evict(table=((0, 1, 2), (3, 4, 9))), "outside")
        refused(lambda: evict(fresh=((5, 6), (7, 9))), "outside")
        refused(lambda: evict(fresh=((5, 6), (7, 5))), "written")
        refused(lambda: evict(fresh=((5, 6), (7, 4))), "written")
        # what holds passes: idle streams, entries behind the rows, shared source pages
        decode(table=((0, 1, -7), (3, 4, 5)))
        decode(table=((99, 99, 99), (3, 4, 5)), lens=(-1, 40), pos=(-3, 2))
        store()
        evict()
        torch.cuda.synchronize()
    finally:
        B.earn_set_validation(old)


def test_tensors_of_another_kind_are_refused():
    B = _B()
    desc = B.make_desc(BF, 4, 2, 64)
    z = lambda *s: torch.zeros(*s, dtype=BF, device=DEV)
    good = dict(q=z(1, 4, 64), k_new=z(1, 2, 64), v_new=z(1, 2, 64), q_pos=i32([0]), k_pages=z(4, 2, 16, 64), v_pages=z(4, 2, 16, 64),
                page_table=i32([[0, 1]]), cache_len=i32([3]), max_cache_len=31, out=z(1, 4, 64))
    B.earn_decode_attn_paged(desc, **good)
    for name, bad in (("q", z(1, 64, 4).transpose(1, 2)), ("q", z(1, 4, 64).cpu()), ("q", z(1, 4, 64).float()), ("cache_len", i32([3]).long()),
                      ("k_pages", z(4, 16, 2, 64)), ("page_table", i32([[0, 1], [2, 3]])), ("out", z(1, 2, 64))):
        with pytest.raises(AssertionError):
            B.earn_decode_attn_paged(desc, **dict(good, **{name: bad}))
    x, u, t = torch.zeros(2, 9, device=DEV), torch.zeros(2, device=DEV), i32([0, 0])
    for args in ((x.t(), u, t), (x.cpu(), u, t), (x, u.double(), t), (x, u, t.long()), (x, u[:1], t)):
        with pytest.raises(AssertionError):
            B.earn_sample(*args)
    with pytest.raises(B.EarnError):
        B.earn_sample(x.half(), u, t)
