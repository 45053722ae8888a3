"""earn_sample against the definition in fp64 (oracle.sample_token): tokens, counts and log-probabilities.

The library holds weights as multiples of 2^-44 of the best one's, each off by half of that and by 2^-46 of itself: a sum over n
tokens is off by 3/2 n 2^-45, and so is u or p times another one; with what 64-bit sums lose on either side that is less than n 2^-43.  The oracle tells how near to a border a row came; rows that come nearer than that are none of these (asserted).
Log-probabilities are fp32: half a step, and n 2^-43 from the sums (which are at least 1).
"""
import numpy as np
import pytest
import torch

from oracle import earn_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _B():
    from paper_2507_00715_amd import binding
    binding.lib()
    return binding


def draw(B, logits, u, pad=0, **params):
    """logits [rows, vocab] on the CPU, u and each of params a list; returns (token, logprob, n_kept)."""
    rows, vocab = logits.shape
    wide = torch.full((rows, vocab + pad), float("inf"), dtype=logits.dtype)     # what lies between the rows would win
    wide[:, :vocab] = logits
    f = lambda x: torch.tensor(x, dtype=torch.float32, device=DEV)
    dev = {k: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV) if k == "top_k" else f(v) for k, v in params.items()}
    token, count = (torch.full((rows,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    logprob = torch.full((rows,), 9.0, device=DEV)
    need = B.earn_sample_workspace_bytes(rows, vocab)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device=DEV)
    B.earn_sample(wide.to(DEV)[:, :vocab], f(u), token, logprob_out=logprob, n_kept_out=count, workspace=ws, **dev)
    torch.cuda.synchronize()
    return token.tolist(), logprob.tolist(), count.tolist()


def check(B, logits, u, pad=0, **params):
    rows, vocab = logits.shape
    token, logprob, count = draw(B, logits, u, pad, **params)
    values = logits.double().numpy()
    f32 = lambda x: float(np.float32(x))
    for r in range(rows):
        args = {k: (v[r] if k == "top_k" else f32(v[r])) for k, v in params.items() if v is not None}
        ref = O.sample_token(values[r], f32(u[r]), **args)
        assert ref["margin"] > vocab * 2.0 ** -43, f"row {r} sits on a border"
        assert (token[r], count[r]) == (ref["token"], ref["n_kept"]), (r, args, u[r], token[r], count[r], ref)
        if ref["token"] < 0:
            assert logprob[r] == -np.inf
        else:
            assert abs(logprob[r] - ref["logprob"]) <= abs(ref["logprob"]) * 2.0 ** -24 + vocab * 2.0 ** -43, r
    return token


def logits_of(kind, rows, vocab, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * 2.5
    if kind == "flat":
        x *= 1e-3
    elif kind == "peaked":
        x = x * 6
    elif kind == "ties":
        x = torch.round(x)
    elif kind == "masked":
        x[torch.rand(rows, vocab, generator=g) < 0.7] = float("-inf")
        x[torch.rand(rows, vocab, generator=g) < 0.1] = torch.finfo(dtype).min
        x[torch.rand(rows, vocab, generator=g) < 0.05] = float("nan")
        x[:, vocab // 2] = 1.0
    return x.to(dtype)


PARAMS = [
    {},
    dict(temperature=[0.7]), dict(temperature=[5.0]), dict(temperature=[0.02]),
    dict(top_k=[1]), dict(top_k=[2]), dict(top_k=[40]), dict(top_k=[10 ** 6]),
    dict(top_p=[0.9]), dict(top_p=[0.3]), dict(top_p=[0.9999]), dict(top_p=[1e-6]),
    dict(min_p=[0.05]), dict(min_p=[1.0]), dict(min_p=[3.0]),
    dict(temperature=[0.8], top_k=[50], top_p=[0.95]), dict(temperature=[1.7], top_k=[7], top_p=[0.5], min_p=[0.1]),
    dict(temperature=[0.05], top_k=[30]), dict(temperature=[0.0]), dict(top_p=[0.0]),
]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["normal", "flat", "peaked", "ties", "masked"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1000, 8191, 32000])
def test_against_the_definition(vocab, kind, dtype):
    B = _B()
    rows = 4
    logits = logits_of(kind, rows, vocab, vocab + len(kind), dtype)
    u = [0.0, 0.137, 0.5003, 0.99991]
    for params in PARAMS:
        check(B, logits, u, pad=vocab % 5, **{k: v * rows for k, v in params.items()})


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("vocab", [131071, 262144, 524288])
def test_large_vocabularies(vocab, dtype):
    B = _B()
    logits = logits_of("normal", 3, vocab, 5, dtype)
    for params in (dict(), dict(top_k=[64] * 3, top_p=[0.9] * 3), dict(top_p=[0.95] * 3), dict(min_p=[0.02] * 3)):
        check(B, logits, [0.11, 0.517, 0.93], **params)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_equal_logits_take_the_lowest_indices(dtype):
    """All logits equal, in more tokens than any list holds: the first k are kept, the border falls between them."""
    B = _B()
    vocab = 40000
    logits = torch.full((4, vocab), 1.5).to(dtype)
    token = check(B, logits, [0.25003, 0.50003, 0.75003, 0.99997], top_k=[30001] * 4)
    assert token == [int(x * 30001) for x in (0.25003, 0.50003, 0.75003, 0.99997)]
    check(B, logits, [0.1, 0.2, 0.3, 0.9], top_p=[0.61234] * 4)
    token, _, count = draw(B, logits, [0.0, 0.5, 0.25, 0.75], top_p=[0.5] * 4)       # borders that are met exactly
    assert count == [20000] * 4 and token == [0, 10000, 5000, 15000]
    # two levels: the lower one is cut
    logits[:, ::2] = 0.5
    check(B, logits, [0.1, 0.5001, 0.7, 0.99], top_k=[20007, 30003, 25000, 20001])
    check(B, logits, [0.1, 0.5001, 0.7, 0.99], top_p=[0.8003, 0.9001, 0.7503, 0.7001])


def test_rows_left_empty_and_infinite_logits():
    B = _B()
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(7, 50)
    x[0] = -inf
    x[1] = nan
    x[2, 3] = x[2, 44] = inf
    x[3] = -inf
    x[3, 17] = -3e38
    x[4] = torch.finfo(F32).min
    x[5, :] = nan
    x[5, 9] = inf
    x[6, 1:] = -inf
    u = [0.5, 0.5, 0.4999, 0.9, 0.5001, 0.3, 0.99]
    for params in (dict(), dict(top_k=[5] * 7), dict(top_p=[0.7] * 7), dict(top_k=[3] * 7, top_p=[0.4] * 7, min_p=[0.5] * 7)):
        token, logprob, count = draw(B, x, u, **params)
        assert token[:2] == [-1, -1] and count[:2] == [0, 0] and logprob[:2] == [-inf, -inf]
        assert token[2] == 3 and count[2] in (1, 2)
        assert token[3] == 17 and count[3] == 1 and logprob[3] == 0.0
        assert token[5] == 9 and count[5] == 1 and token[6] == 0 and count[6] == 1
    token, logprob, count = draw(B, x, u)
    assert count[2] == 2 and abs(logprob[2] + np.log(2)) < 1e-6 and count[4] == 50 and token[4] == 25
    token, _, _ = draw(B, x, [0.75] * 7)
    assert token[2] == 44


def test_uniform_numbers_outside_their_range_and_odd_parameters():
    B = _B()
    x = torch.zeros(8, 10)
    token, _, _ = draw(B, x, [-1.0, 1.0, 7.0, float("nan"), float("inf"), 0.0, 1.0 - 2.0 ** -24, 0.95])
    assert token == [0, 9, 9, 0, 9, 0, 9, 9]
    nan = float("nan")
    token, _, count = draw(B, x, [0.5] * 8, temperature=[nan, -1.0, 0.0, 1.0, 1.0, float("inf"), 1e-45, 1e38],
                           top_p=[1.0, 1.0, 1.0, nan, -2.0, 1.0, 1.0, 2.0], min_p=[0, 0, 0, 0, 0, nan, 0, -1.0], top_k=[0, 0, 0, 0, 0, -4, 0, 99])
    assert token == [0, 0, 0, 0, 0, 5, 5, 5] and count == [1, 1, 1, 1, 1, 10, 10, 10]


def test_temperatures_and_logits_of_the_smallest_numbers():
    """Differences of logits over temperatures that both lie at the lower end of fp32, and temperatures at the upper end."""
    B = _B()
    x = torch.arange(9, dtype=torch.float32).repeat(6, 1) * 1e-44
    t = [1e-44, 3e-44, 1e-45, 1e-38, 1e38, 3e-37]
    for params in (dict(), dict(top_p=[0.8] * 6), dict(top_k=[4] * 6), dict(min_p=[0.1] * 6)):
        check(B, x, [0.0371, 0.4001, 0.9001, 0.3001, 0.6003, 0.9502], temperature=t, **params)
    wide = torch.tensor([[3e38, -3e38, 1e38, -1e38, 0.0, 2e38]] * 4)          # differences beyond fp32
    for params in (dict(), dict(top_p=[0.9] * 4), dict(top_k=[5] * 4, top_p=[0.95] * 4), dict(min_p=[0.02] * 4)):
        check(B, wide, [0.05, 0.6, 0.9, 0.97], temperature=[1e38, 3e38, float("inf"), 7e37], **params)
    far = torch.tensor([[0.0, -1e-37, -2e-37, -1e-36, -5e-36, -1e38]] * 4)
    check(B, far, [0.1, 0.7, 0.95, 0.9999], temperature=[1e-37, 2e-37, 1e-38, 1e-45], top_p=[0.99] * 4)


def test_frequencies_follow_the_weights():
    """The draw with u = (i + 1/2) / n takes token t round(n p_t) times, up to one each way for its two borders."""
    B = _B()
    n, vocab = 20000, 37
    row = torch.randn(vocab, generator=torch.Generator().manual_seed(1)) * 2
    token, _, _ = draw(B, row.expand(n, vocab).contiguous(), [(i + 0.5) / n for i in range(n)], temperature=[0.9] * n)
    share = torch.softmax(row.double() / np.float64(np.float32(0.9)), 0).numpy() * n
    assert (np.abs(np.bincount(token, minlength=vocab) - share) <= 1.01).all()
    assert token == sorted(token)


def test_many_rows_of_few_tokens_and_settings_of_their_own():
    B = _B()
    rng = np.random.default_rng(3)
    rows, vocab = 700, 300
    logits = logits_of("normal", rows, vocab, 9, F32)
    u = (rng.integers(1, 4000, rows) / 4001).tolist()
    check(B, logits, u, pad=1, temperature=rng.choice([0.0, 0.3, 0.9, 1.4], rows).tolist(), top_k=rng.integers(-1, 60, rows).tolist(),
          top_p=rng.choice([0.35, 0.91, 1.0, 0.0], rows).tolist(), min_p=rng.choice([0.0, 0.03, 0.4], rows).tolist())
