"""arb_logits against its formulas: processed logits bit for bit (every operation is one IEEE rounding in fp32, which numpy does alike),
tokens exactly, log-probabilities against 64 bits.

Tolerance of a log-probability x[t] - m - log(l): the sum of up to 2^18 exponentials in a tree with 16 serial terms at the leaves
(16 + 14 roundings of 2^-24), exponentials of relative error (2 + 1.2 |x - m|) 2^-23 that weigh e^(x - m) (on average below 4 * 2^-23
where x - m has the weight), the logarithm's 2^-21 absolute: below 2^-18; the two differences round to 2^-24 of |x| + |m| each."""
import numpy as np
import pytest
import torch

from tests import helpers as H

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2512_05033_b200 import binding
    return binding


def reference(x, **o):
    """float32 [S, V] -> (processed float32, tokens, logprobs float64), operation by operation."""
    x = x.astype(np.float32).copy()
    S, V = x.shape
    f = np.float32
    with np.errstate(all="ignore"):
        for s in range(S):
            if o.get("history") is not None:
                n = o["history"].shape[1] if o.get("history_lens") is None else min(max(int(o["history_lens"][s]), 0), o["history"].shape[1])
                t = o["history"][s, :n]
                count = np.bincount(t[(t >= 0) & (t < V)], minlength=V)
                rep = f(1) if o.get("repetition") is None else o["repetition"][s]
                pre = f(0) if o.get("presence") is None else o["presence"][s]
                fre = f(0) if o.get("frequency") is None else o["frequency"][s]
                y = np.where(x[s] > 0, x[s] / rep, x[s] * rep).astype(f)
                y = (y - pre).astype(f) - (fre * count.astype(f)).astype(f)
                x[s] = np.where(count > 0, y, x[s])
            if o.get("bias_offsets") is not None:
                total, bias = len(o["bias_tokens"]), np.zeros(V, f)
                begin, end = (min(max(int(v), 0), total) for v in o["bias_offsets"][s:s + 2])
                for i in range(begin, end):
                    if 0 <= o["bias_tokens"][i] < V:
                        bias[o["bias_tokens"][i]] = f(bias[o["bias_tokens"][i]] + o["bias_values"][i])
                x[s] = x[s] + bias
            greedy = False
            if o.get("temperature") is not None:
                greedy = not o["temperature"][s] > 0
                if not greedy:
                    x[s] = x[s] / o["temperature"][s]
            if o.get("mask") is not None:
                bits = np.unpackbits(o["mask"][s].view(np.uint8), bitorder="little")[:V]
                x[s] = np.where(bits != 0, x[s], -np.inf)
        tokens, logprobs = np.full(S, -1), np.full(S, -np.inf)
        for s in range(S):
            y = x[s] if o.get("noise") is None or (o.get("temperature") is not None and not o["temperature"][s] > 0) else (x[s] + o["noise"][s]).astype(f)
            y = np.where(np.isnan(y), -np.inf, y)
            if y.max() > -np.inf:
                tokens[s] = int(np.argmax(y))
            z = x[s].astype(np.float64)
            if np.isnan(z).any() or (z == np.inf).any():
                logprobs[s] = np.nan
            elif tokens[s] >= 0:
                m = z.max()
                logprobs[s] = z[tokens[s]] - m - np.log(np.exp(z - m).sum())
    return x, tokens, logprobs


def inputs(seed, S, V, dtype=torch.float32, history=0, biases=0, mask=False, temperature=False, noise=False, dup=False):
    r = np.random.RandomState(seed)
    x = torch.from_numpy(r.randn(S, V).astype(np.float32) * 3).to(dtype)
    o = {}
    if history:
        o["history"] = r.randint(-2, V + 2, (S, history)).astype(np.int32)
        o["history"][:, : history // 2] = r.randint(0, max(1, V // 10), (S, history // 2))
        o["history_lens"] = r.randint(0, history + 2, S).astype(np.int32)
        o["repetition"] = (1 + r.rand(S)).astype(np.float32)
        o["presence"] = r.rand(S).astype(np.float32)
        o["frequency"] = r.rand(S).astype(np.float32)
    if biases:
        counts = r.randint(0, biases + 1, S)
        o["bias_offsets"] = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
        n = int(o["bias_offsets"][-1])
        o["bias_tokens"] = r.randint(-1, min(V, 5) if dup else V + 1, n).astype(np.int32)
        o["bias_values"] = (r.randn(n) * 4).astype(np.float32)
    if mask:
        o["mask"] = r.randint(-2 ** 31, 2 ** 31, (S, -(-V // 32))).astype(np.int32)
    if temperature:
        o["temperature"] = (0.3 + r.rand(S)).astype(np.float32)
        o["temperature"][r.rand(S) < 0.2] = 0.0
    if noise:
        o["noise"] = (-np.log(-np.log(r.rand(S, V).clip(1e-7, 1 - 1e-7)))).astype(np.float32)
    return x, o


def check(x, o, stride=None, ctx=None):
    c = ctx or H.ctx()
    S, V = x.shape
    d = {k: torch.from_numpy(v).cuda() for k, v in o.items()}
    xs = x.cuda()
    if stride:
        xs = torch.full((S, stride), float("nan"), dtype=x.dtype, device="cuda")[:, :V].copy_(x)
    buf = torch.full((S * V + 64,), 55.0, device="cuda")
    out, tokens, logprobs = c.logits(xs, out=buf[32:-32].view(S, V), **d)
    assert c.poll_status() == 0
    want, wt, wl = reference(x.float().numpy(), **o)
    got = out.cpu().numpy()
    assert np.array_equal(got, want, equal_nan=True), f"{(got != want).sum()} of {got.size} logits differ"
    assert np.array_equal(tokens.cpu().numpy(), wt)
    assert bool((buf[:32] == 55).all()) and bool((buf[-32:] == 55).all())
    lp = logprobs.double().cpu().numpy()
    assert np.array_equal(np.isfinite(lp), np.isfinite(wl)) and np.array_equal(np.isnan(lp), np.isnan(wl))
    fine = np.isfinite(wl)
    big = np.abs(np.where(np.isfinite(want), want, 0)).max(-1)
    assert bool((np.abs(lp - wl)[fine] <= (2.0 ** -18 + 2.0 ** -22 * big)[fine]).all())
    return out, tokens, logprobs


SIZES = [(1, 1), (1, 7), (3, 8), (2, 33), (5, 4095), (4, 4096), (3, 4097), (2, 4103), (7, 12289), (1, 32000), (16, 50003), (3, 128001)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S,V", SIZES)
def test_everything_at_once(S, V, dtype):
    check(*inputs(S * V, S, V, dtype, history=37, biases=9, mask=True, temperature=True, noise=True))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("only", [{}, {"history": 300}, {"history": 1}, {"biases": 70, "dup": True}, {"mask": True}, {"temperature": True}, {"noise": True}])
def test_each_alone(only, dtype):
    check(*inputs(5, 6, 5003, dtype, **only))


@pytest.mark.parametrize("dtype,stride", [(torch.bfloat16, 5056), (torch.float32, 5003 + 1), (torch.bfloat16, 5003 + 3), (torch.float32, 5003 + 2)])
def test_padded_rows(dtype, stride):
    check(*inputs(6, 5, 5003, dtype, history=50, mask=True, noise=True), stride=stride)


def test_ties_go_to_the_lowest_token_across_slices():
    x = torch.zeros(3, 20000)
    x[0, [4095, 4096, 19999]] = 2.0
    x[1, 19999] = 1.0
    _, tokens, _ = check(x, {})
    assert tokens.tolist() == [4095, 19999, 0]
    _, tokens, _ = check(x.bfloat16(), {})
    assert tokens.tolist() == [4095, 19999, 0]


def test_masked_rows_infinities_and_nan():
    x, o = inputs(7, 8, 9000, mask=True)
    o["mask"][0] = 0                                           # nothing allowed
    o["mask"][1] = 0
    o["mask"][1, 200] = 1 << 5                                 # one token
    o["mask"][2, 10] &= ~np.int32(1 << 3)
    x[2, 323] = float("nan")                                   # NaN where nothing is allowed: does not show
    x[3] = -float("inf")                                       # every logit -inf
    x[4, 17], o["mask"][4, 0] = float("nan"), -1               # NaN among the allowed: never wins, logprob NaN
    x[5, 100:200] = -float("inf")
    x[6, 77], o["mask"][6, 2] = float("inf"), -1               # wins; logprob NaN
    x[7] = torch.finfo(torch.float32).min                      # the type's lowest value everywhere
    _, tokens, logprobs = check(x, o)
    assert tokens[0] == -1 and tokens[1] == 6405 and tokens[3] == -1 and tokens[6] == 77
    assert float(logprobs[1]) == 0.0 and float(logprobs[0]) == -np.inf
    _, tokens, _ = check(torch.full((2, 300), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16), {})
    assert tokens.tolist() == [0, 0]


def test_a_token_listed_twice_gets_its_sum_in_order():
    S, V = 2, 6000
    x = torch.zeros(S, V)
    values = np.array([1e8, 1.0, -1e8, 0.25] * 20 + [3.0], np.float32)
    o = {"bias_offsets": np.array([0, 81, 81], np.int32), "bias_tokens": np.full(81, 4100, np.int32), "bias_values": values}
    check(x, o)
    o["bias_offsets"] = np.array([-5, 300, 1000], np.int32)    # offsets beyond the list are clamped
    check(x, o)


def test_a_token_listed_many_times():
    """Hundreds of entries of one token beside every token of a small vocabulary, in the history too."""
    r = np.random.RandomState(4)
    V, n = 4200, 4200
    x = torch.from_numpy(r.randn(2, V).astype(np.float32))
    tokens = np.concatenate((r.permutation(V), np.full(700, 17), np.full(300, 4199))).astype(np.int32)
    o = {"bias_offsets": np.array([0, len(tokens), len(tokens)], np.int32), "bias_tokens": tokens,
         "bias_values": r.randn(len(tokens)).astype(np.float32), "history": np.full((2, 1000), 17, np.int32),
         "repetition": np.array([1.3, 1.1], np.float32), "frequency": np.array([0.01, 0.02], np.float32)}
    check(x, o)


@pytest.mark.parametrize("V,n", [(4 * 4096 + 5, 12000), (9 * 4096 - 1, 5000)])
def test_long_histories_of_many_rows(V, n):
    """More rows than CTAs at a time, so that a CTA has many pieces, and more special tokens than it holds for all of them."""
    r = np.random.RandomState(V)
    S = 640
    x = torch.from_numpy(r.randn(S, V).astype(np.float32)).bfloat16()
    o = {"history": np.stack([r.permutation(V)[:n] for _ in range(S)]).astype(np.int32), "presence": r.rand(S).astype(np.float32)}
    o["history_lens"] = np.where(np.arange(S) % 3 == 0, n // 8, n).astype(np.int32)
    o["bias_offsets"] = (np.arange(S + 1) * 2).astype(np.int32)
    o["bias_tokens"] = r.randint(0, V, 2 * S).astype(np.int32)
    o["bias_values"] = r.randn(2 * S).astype(np.float32)
    check(x, o)


def test_what_is_not_wanted_is_left_out():
    x, o = inputs(8, 3, 7001, history=20)
    c, b = H.ctx(), _binding()
    d = {k: torch.from_numpy(v).cuda() for k, v in o.items()}
    full = c.logits(x.cuda(), **d)
    none, tokens, logprobs = c.logits(x.cuda(), want_out=False, **d)
    assert none is None and torch.equal(tokens, full[1]) and torch.equal(logprobs, full[2])
    # in place, and through the pointer-level call without tokens
    y = x.cuda()
    c.logits(y, out=y, **d)
    assert torch.equal(y, full[0])
    y = x.cuda()
    p = b.LogitsParams(dtype=b.ARB_F32, rows=3, vocab=7001, logits=y.data_ptr(), out=y.data_ptr())
    import ctypes
    assert b.lib.arb_logits(c._h, ctypes.byref(p), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(y.cpu(), x)


def test_the_same_call_gives_the_same_bits_and_a_graph_replays():
    c = _binding().Context(0)
    x, o = inputs(9, 20, 50003, torch.bfloat16, history=400, biases=30, mask=True, temperature=True, noise=True)
    d = {k: torch.from_numpy(v).cuda() for k, v in o.items()}
    xs = x.cuda()
    first = [t.clone() for t in c.logits(xs, **d)]
    for _ in range(5):
        for a, b in zip(c.logits(xs, **d), first):
            assert torch.equal(a, b)
    bufs = [torch.empty_like(t) for t in first]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.logits(xs, **d, out=bufs[0], tokens=bufs[1], logprobs=bufs[2], stream=s)
        c.logits(xs, **d, out=bufs[0], tokens=bufs[1], logprobs=bufs[2], stream=s)
    for _ in range(3):
        for t in bufs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(bufs, first):
            assert torch.equal(a, b)
    assert c.poll_status() == 0
    c.close()


def test_gumbel_noise_draws_from_the_softmax():
    """2000 draws of one row of 8 tokens: frequencies within 5 standard deviations of softmax(x)."""
    n = 2000
    r = np.random.RandomState(3)
    row = np.array([0.0, 1.0, 2.0, -1.0, 0.5, -np.inf, 1.5, 0.2], np.float32)
    x = torch.from_numpy(np.tile(row, (n, 1)))
    noise = (-np.log(-np.log(r.rand(n, 8)))).astype(np.float32)
    _, tokens, _ = check(x, {"noise": noise})
    p = np.exp(row) / np.exp(row).sum()
    count = np.bincount(tokens.cpu().numpy(), minlength=8)
    assert count[5] == 0 and bool((np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S", [1, 64, 640])
@pytest.mark.parametrize("V", [1, 2045, 2046, 2047, 2048, 2049, 9 * 2048 - 2, 9 * 2048 - 1])
def test_vocabularies_that_end_with_a_piece(V, S, dtype):
    """A row may start inside a group of four tokens, so the pieces of a row that starts on one may reach past its end by a whole piece:
    nothing of the history or the biases lies there, least of all tokens outside the vocabulary."""
    if S == 640 and V > 4096:
        S = 600                                          # (a run of all a row's pieces, the last in a window of its own)
    x, o = inputs(V + S, S, V, dtype, history=40, biases=12, mask=True, temperature=True)
    o["history"][:, 1] = np.random.RandomState(V).choice([-2 ** 31, -1, V, V + 5, V + 3000, 2 ** 31 - 1], S)
    far = np.arange(len(o["bias_tokens"])) % 5 == 0
    o["bias_tokens"][far] = np.random.RandomState(S).choice([-2 ** 31, -V, V, V + 1, 2 * V + 4096, 2 ** 31 - 1], far.sum())
    check(x, o)


@pytest.mark.parametrize("V", [126974, 126975, 151550, 151551])
def test_large_vocabularies_that_end_with_a_piece(V):
    check(*inputs(V, 3, V, torch.bfloat16, history=500, biases=40, temperature=True))
    check(*inputs(V, 70, V, torch.bfloat16, history=50, biases=40))


def _events_ms(f):
    f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("repeats", ["one", "pairs", "many", "all"])
def test_long_lists_of_biases_with_repeats(repeats):
    """A list as long as the vocabulary: with one token in it twice, with every token twice, with one token 20000 times, of one
    token alone.  Sums are taken in the order of the list; a call takes about as long as one without repeats, not the square of it."""
    V, r = 60001, np.random.RandomState(3)
    if repeats == "one":
        tokens = np.concatenate((r.permutation(V), [V // 2]))
    elif repeats == "pairs":
        tokens = np.concatenate((r.permutation(V), r.permutation(V)))
    elif repeats == "many":
        tokens = r.permutation(np.concatenate((np.arange(V), np.full(20000, 1234))))
    else:
        tokens = np.full(V, 777)
    n = len(tokens)
    o = {"bias_offsets": np.array([0, 3, n + 3], np.int32), "bias_tokens": np.concatenate(([5, 6, 5], tokens)).astype(np.int32),
         "bias_values": r.randn(n + 3).astype(np.float32)}
    x = torch.from_numpy(r.randn(2, V).astype(np.float32))
    check(x, o)
    d = {k: torch.from_numpy(v).cuda() for k, v in o.items()}
    xs = x.cuda()
    assert _events_ms(lambda: H.ctx().logits(xs, **d)) < 25.0


def test_rows_that_leave_no_records_ask_for_no_workspace():
    """A context with a small workspace serves calls whose rows are each one CTA's, and calls that want the logits alone."""
    c = _binding().Context(0, workspace_bytes=64 << 10)
    x, o = inputs(11, 9000, 70, history=5)
    want, wt, _ = reference(x.numpy(), **o)
    d = {k: torch.from_numpy(v).cuda() for k, v in o.items()}
    out, tokens, _ = c.logits(x.cuda(), **d)
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(tokens.cpu().numpy(), wt)
    assert c.poll_status() == 0
    c.close()


def test_lengths_beyond_32_bits_are_refused_and_flags_raise_their_own_error():
    c, x = H.ctx(), torch.zeros(1, 70, device="cuda")
    long = lambda *shape: torch.zeros(1, dtype=torch.int32, device="cuda").expand(*shape)  # noqa: E731
    off = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="too long"):
        c.logits(x, bias_offsets=off, bias_tokens=long(2 ** 32 + 1), bias_values=torch.zeros(1, device="cuda"))
    for more in ({"history": long(1, 2 ** 32 + 5)}, {"mask": long(1, 2 ** 32 + 5)}):
        with pytest.raises(ValueError):
            c.logits(x, **more)

    class Neither:
        def __bool__(self):
            raise ValueError("neither true nor false")

    q, kv = torch.zeros(1, 4, 128, device="cuda"), torch.zeros(1, 2, 128, device="cuda")
    pool, table, lens = torch.zeros(1, 2, 16, 128, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for flag in ("interleaved", "update_lens"):
        with pytest.raises(ValueError, match="neither"):
            c.rope_append(q, kv, kv, torch.zeros(64, device="cuda"), table, lens, lens, pool, pool.clone(), **{flag: Neither()})
