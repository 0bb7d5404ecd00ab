"""arb_attn_rules against its definition in 64 bits.

Tolerance.  Let A = sum_j p_j |v_j| of an output element and z = softmax_scale * |q| * max_j |k_j| a bound of the row's scores.  A
score's fp32 error is at most (D + 4) 2^-24 z (its D products and sums, the factors after them) + cap * 2^-21 (the tanh's argument and
value) + 2^-22 S (its own rounding and the exponent's; S the largest score, bias included, of a key whose weight counts); the
weights carry twice that (numerator and denominator) and the tensor cores' weights are rounded to bf16, 2^-8.  The bias is exact
near the row and has no weight far from it.  The output is rounded once: finfo.eps / 2 of the value."""
import math

import numpy as np
import pytest
import torch

from tests import helpers as H

pytestmark = pytest.mark.gpu
P = 16
BF, F32 = torch.bfloat16, torch.float32


def _binding():
    from paper_2512_05033_b200 import binding
    return binding


class Inputs:
    def __init__(self, seed, dtype, hq, hkv, D, lens, new, std=2.0, cap=0.0, window=0, slopes=False, prefix=None, first=None, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.D, self.cap, self.window = dtype, hq, hkv, D, cap, window
        B, T = len(lens), sum(new)
        need = [-(-x // P) for x in lens]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g)
        self.table, at = torch.full((B, max(need) + 1), -1, dtype=torch.int32), 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c].int()
            at += c
        self.q = (torch.randn(T, hq, D, generator=g) * std).to(dtype)
        self.k = torch.randn(self.pages, hkv, P, D, generator=g).to(dtype)
        self.v = torch.randn(self.pages, hkv, P, D, generator=g).to(dtype)
        for b, x in enumerate(lens):     # what lies behind a sequence's last key must not matter
            if x % P:
                self.k[self.table[b, x // P], :, x % P:] = float("nan")
                self.v[self.table[b, x // P], :, x % P:] = float("inf")
        self.lens, self.new = torch.tensor(lens, dtype=torch.int32), torch.tensor(new, dtype=torch.int32)
        self.slopes = 2.0 ** (-8.0 * (torch.arange(hq) + 1) / hq) if slopes else None
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int32)
        self.first = None if first is None else torch.tensor(first, dtype=torch.int32)

    def sees(self, b, row0):
        n, L = int(self.new[b]), int(self.lens[b])
        pos, key = torch.arange(L - n, L)[:, None], torch.arange(L)
        m = key <= pos
        if self.prefix is not None:
            m = m | ((pos < int(self.prefix[b])) & (key < int(self.prefix[b])))
        if self.window:
            m = m & (key > pos - self.window)
        if self.first is not None:
            m = m & (key >= self.first[row0:row0 + n, None])
        return m, (pos - key).abs()

    def reference(self, scale=None):
        """(out, bar) in 64 bits."""
        D, G = self.D, self.hq // self.hkv
        scale = scale or D ** -0.5
        outs, bars, row0 = [], [], 0
        for b in range(len(self.lens)):
            n, L = int(self.new[b]), int(self.lens[b])
            if n == 0:
                continue
            m, dist = self.sees(b, row0)
            page = self.table[b, :-(-L // P)].long()
            page = torch.where((page >= 0) & (page < self.pages), page, 0)   # (entries no row needs may be anything)
            k, v = (x[page].transpose(0, 1).flatten(1, 2)[:, :L].double() for x in (self.k, self.v))
            o, bar = torch.zeros(n, self.hq, D, dtype=torch.float64), torch.zeros(n, self.hq, D, dtype=torch.float64)
            for h in range(self.hq):
                q, kk, vv = self.q[row0:row0 + n, h].double(), k[h // G], v[h // G]
                seen = m.any(0)
                kk, vv = torch.where(seen[:, None], kk, 0.0), torch.where(seen[:, None], vv, 0.0)
                s = q @ kk.T * scale
                if self.cap:
                    s = self.cap * torch.tanh(s / self.cap)
                if self.slopes is not None:
                    s = s - self.slopes[h].double() * dist
                s = torch.where(m, s, -math.inf)
                top = s.amax(-1, keepdim=True)
                p = torch.where(m, torch.exp(s - torch.where(torch.isinf(top), 0.0, top)), 0.0)
                p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
                o[:, h] = p @ vv
                z = scale * q.norm(dim=-1, keepdim=True) * kk.norm(dim=-1).max()
                counts = torch.where(p > 2.0 ** -30, s.abs(), 0.0).amax(-1, keepdim=True)
                d = (D + 4) * 2.0 ** -24 * z + self.cap * 2.0 ** -21 + 2.0 ** -22 * (1 + counts)
                rel = 2 * d + (2.0 ** -8 if self.dtype == BF else 2.0 ** -20)
                bar[:, h] = rel * (p @ vv.abs()) + torch.finfo(self.dtype).eps / 2 * o[:, h].abs() + 1e-30
            outs.append(o)
            bars.append(bar)
            row0 += n
        return torch.cat(outs), torch.cat(bars)

    def args(self):
        cu = lambda t: None if t is None else t.cuda()  # noqa: E731
        return (tuple(cu(t) for t in (self.q, self.k, self.v, self.table, self.lens, self.new)) + (int(self.new.max()),),
                dict(cap=self.cap, window=self.window, slopes=cu(self.slopes), prefix_lens=cu(self.prefix), first_keys=cu(self.first)))


def check(x, scale=0.0, bits=0, ctx=None):
    c = ctx or H.ctx()
    args, rules = x.args()
    buf = torch.full((x.q.shape[0] + 2,) + tuple(x.q.shape[1:]), 333.0, dtype=x.dtype, device="cuda")
    out = c.attn_rules(*args, **rules, out=buf[1:-1], softmax_scale=scale)
    assert c.poll_status() == bits
    assert bool((buf[0] == 333).all()) and bool((buf[-1] == 333).all())
    ref, bar = x.reference(scale)
    err = (out.double().cpu() - ref).abs()
    assert bool(torch.isfinite(out).all())
    assert bool((err <= bar).all()), f"off by {err.max():.3e}, {(err / bar).max():.2f} of the bar"
    return out


RULES = {
    "none": {},
    "cap": {"cap": 8.0},
    "cap_tight": {"cap": 0.7},
    "window": {"window": 100},
    "window_one": {"window": 1},
    "slopes": {"slopes": True},
    "all": {"cap": 5.0, "window": 333, "slopes": True},
}


@pytest.mark.parametrize("rules", list(RULES))
@pytest.mark.parametrize("dtype,hq,hkv,D", [(BF, 12, 2, 128), (BF, 32, 8, 64), (F32, 8, 2, 64), (F32, 3, 3, 128), (BF, 8, 1, 128)])
def test_tokens(dtype, hq, hkv, D, rules):
    """q_len 1 over lengths from one key on, idle slots between."""
    lens, new = [1, 16, 17, 500, 1, 2049, 100, 333, 334], [1, 1, 1, 1, 0, 1, 1, 1, 1]
    check(Inputs(1, dtype, hq, hkv, D, lens, new, **RULES[rules]))


@pytest.mark.parametrize("rules", list(RULES))
@pytest.mark.parametrize("dtype,hq,hkv,D", [(BF, 28, 4, 128), (BF, 4, 4, 64), (F32, 8, 2, 64), (F32, 5, 1, 128), (BF, 16, 2, 64), (BF, 6, 2, 128)])
def test_chunks(dtype, hq, hkv, D, rules):
    """Steps and tokens in one batch: steps that start at the cache's first key, end inside a page, pass a tile of rows."""
    lens, new = [2, 300, 129, 700, 64, 1500], [2, 17, 129, 1, 0, 140]
    check(Inputs(2, dtype, hq, hkv, D, lens, new, **RULES[rules]))


def _documents(lens, new, length, shift):
    return [max(0, p - (p + shift) % length) for L, n in zip(lens, new) for p in range(L - n, L)]


@pytest.mark.parametrize("dtype,hq,hkv,D", [(BF, 8, 2, 128), (BF, 8, 8, 64), (F32, 4, 2, 64)])
@pytest.mark.parametrize("document,prefix", [(37, None), (500, None), (None, 100), (150, 60), (1, 30)])
def test_documents_and_prefixes(dtype, hq, hkv, D, document, prefix):
    lens, new = [300, 1000, 40, 290, 700], [300, 200, 40, 1, 450]
    first = _documents(lens, new, document, 11) if document else None
    prefix = [0, 900, prefix, 290, prefix * 5] if prefix else None
    check(Inputs(3, dtype, hq, hkv, D, lens, new, prefix=prefix, first=first, cap=6.0 if document == 150 else 0.0))
    check(Inputs(4, dtype, hq, hkv, D, lens, new, prefix=prefix, first=first, window=90, slopes=True))


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128)])
def test_rows_that_see_nothing_and_documents_in_any_order(dtype, D):
    """First keys past the row (no key is left), negative ones, and ones that go down from row to row."""
    lens, new = [400, 200, 50], [130, 1, 50]
    r = np.random.RandomState(0)
    first = r.randint(-50, 420, sum(new)).tolist()
    first[130] = 200                                     # the single token sees nothing
    x = Inputs(5, dtype, 8, 2, D, lens, new, first=first)
    out = check(x)
    assert not bool(out[130].any())
    first[130] = 199                                     # ... and itself alone
    check(Inputs(5, dtype, 8, 2, D, lens, new, first=first, cap=3.0, slopes=True))
    check(Inputs(6, dtype, 8, 2, D, lens, new, first=[10 ** 9] * sum(new)))
    check(Inputs(6, dtype, 8, 2, D, lens, new, first=[10 ** 9] * sum(new), prefix=[2000, -3, 0]))


@pytest.mark.parametrize("dtype,D,new", [(BF, 128, 1), (BF, 128, 40), (BF, 64, 40), (F32, 64, 1), (F32, 128, 40)])
def test_what_is_hidden_does_not_reach_the_result(dtype, D, new):
    """NaN and infinities in keys and values that no row sees, inside the pages that are read; bad table entries before the window."""
    x = Inputs(7, dtype, 8, 2, D, [1000, 777], [new, new], window=200, slopes=True)
    for b, L in enumerate((1000, 777)):
        dead = max(0, L - new - 200 + 1)                # keys 0 .. dead - 1
        for j in range(dead):
            x.k[x.table[b, j // P], :, j % P] = float("nan")
            x.v[x.table[b, j // P], :, j % P] = float("inf") if j % 2 else float("nan")
        x.table[b, :dead // P] = 1 << 29                # never looked up
    check(x)


@pytest.mark.parametrize("dtype,D,new", [(BF, 128, 1), (BF, 128, 20), (BF, 64, 20), (F32, 64, 1), (F32, 128, 20)])
def test_large_scores(dtype, D, new):
    """Scores far beyond the cap, both signs; the same without a cap."""
    check(Inputs(8, dtype, 8, 2, D, [300, 200], [new, new], std=40.0, cap=20.0))
    check(Inputs(8, dtype, 8, 2, D, [300, 200], [new, new], std=40.0))


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_a_long_cache(dtype, D):
    lens, new = [40000, 900, 21000], [1, 1, 70]
    check(Inputs(9, dtype, 4, 1, D, lens, new, cap=10.0))
    check(Inputs(9, dtype, 4, 1, D, lens, new, window=5000, slopes=True))
    check(Inputs(9, dtype, 4, 1, D, lens[:2], new[:2], window=5000, cap=10.0, first=[30000, 5]))


def test_rules_off_is_the_plain_attention():
    x = Inputs(10, BF, 28, 4, 128, [700, 300, 90], [100, 1, 90])
    args, rules = x.args()
    c = H.ctx()
    a, b = c.attn(*args), c.attn_rules(*args)
    ref, bar = x.reference()
    assert bool(((a.double() - b.double()).abs().cpu() <= 2 * bar).all())


def test_softmax_scale_is_taken():
    check(Inputs(11, BF, 8, 2, 128, [200, 100], [30, 1], cap=4.0), scale=0.31)


def test_bad_lengths_give_rows_of_zeros():
    b = _binding()
    for dtype, D in ((BF, 128), (BF, 64), (F32, 64)):
        for bad in (0, 5, 10 ** 6):
            x = Inputs(12, dtype, 4, 2, D, [100, 40, 60], [1, 20, 30], window=50)
            args, rules = x.args()
            args[4][1] = bad
            out = H.ctx().attn_rules(*args, **rules)
            assert H.ctx().poll_status() == b.DEV_BAD_SEQ_LEN
            assert not bool(out[1:21].any()) and bool(out[0].any()) and bool(out[21:].any())
            x = Inputs(12, dtype, 4, 2, D, [100, 40], [1, 1], cap=5.0)
            args, rules = x.args()
            args[4][0] = 0 if bad == 5 else bad
            out = H.ctx().attn_rules(*args, **rules)
            assert H.ctx().poll_status() == b.DEV_BAD_SEQ_LEN and not bool(out[0].any()) and bool(out[1].any())


def test_bad_pages_are_reported_and_other_sequences_keep_their_rows():
    b = _binding()
    for dtype, new in ((BF, 1), (BF, 30), (F32, 1), (F32, 30)):
        x = Inputs(13, dtype, 4, 2, 128, [200, 150], [new, new], cap=5.0)
        ref, bar = x.reference()
        args, rules = x.args()
        args[3][0, 3] = x.pages + 5
        args[3][0, 5] = -9
        out = H.ctx().attn_rules(*args, **rules)
        assert H.ctx().poll_status() == b.DEV_BAD_PAGE
        assert bool(((out[new:].double().cpu() - ref[new:]).abs() <= bar[new:]).all()) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64)])
def test_more_rows_on_the_device_than_there_are(dtype, D):
    """q_lens that add up to more than total_q: rows beyond it are neither read nor written."""
    x = Inputs(17, dtype, 4, 2, D, [100, 90, 80, 0 + 70], [1, 1, 1, 1], window=30, cap=5.0)
    ref, bar = x.reference()
    args, rules = x.args()
    c = H.ctx()
    for first in (None, torch.zeros(2, dtype=torch.int32, device="cuda")):
        buf = torch.full((6, 4, D), 333.0, dtype=dtype, device="cuda")
        c.attn_rules(args[0][:2].contiguous(), *args[1:], cap=5.0, window=30, first_keys=first, out=buf[2:4])
        assert c.poll_status() == 0
        assert bool((buf[:2] == 333).all()) and bool((buf[4:] == 333).all())
        assert bool(((buf[2:4].double().cpu() - ref[:2]).abs() <= bar[:2]).all())
    y = Inputs(18, dtype, 4, 2, D, [100, 90, 80], [20, 30, 1], window=30)
    args, rules = y.args()
    buf = torch.full((30, 4, D), 333.0, dtype=dtype, device="cuda")
    c.attn_rules(args[0][:25].contiguous(), *args[1:6], 20, window=30, out=buf[2:27])   # the second step has rows for five
    c.poll_status()
    assert bool((buf[:2] == 333).all()) and bool((buf[27:] == 333).all())


def test_two_contexts_two_streams_and_a_graph():
    b = _binding()
    x = Inputs(14, BF, 28, 4, 128, [900, 3000, 400], [60, 1, 100], cap=9.0, window=700, slopes=True)
    args, rules = x.args()
    ctxs, streams = [b.Context(0) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = ctxs[0].attn_rules(*args, **rules)
    torch.cuda.synchronize()
    outs = [[torch.empty_like(want) for _ in range(8)] for _ in range(2)]
    for i in range(8):
        for c, s, o in zip(ctxs, streams, outs):
            c.attn_rules(*args, **rules, out=o[i], stream=s)
    torch.cuda.synchronize()
    for o in outs:
        for t in o:
            assert torch.equal(t, want)                  # the same call gives the same bits
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        for t in outs[0][:3]:
            ctxs[0].attn_rules(*args, **rules, out=t, stream=streams[0])
    for _ in range(2):
        for t in outs[0]:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want) for t in outs[0][:3])
    for c in ctxs:
        assert c.poll_status() == 0
        c.close()


def test_between_other_calls_of_the_context():
    """The workspaces are shared with arb_attn's kernels: calls of both kinds in turn on one stream."""
    c = H.ctx()
    a = Inputs(15, BF, 12, 2, 128, [3000, 5000, 200], [1, 1, 1], window=2000)
    d = Inputs(16, BF, 32, 8, 128, [9000, 700], [20, 130], cap=7.0)
    outs = []
    for _ in range(6):
        for x in (a, d):
            args, rules = x.args()
            outs.append((x, c.attn_rules(*args, **rules)))
            p = c.params_for(args[0], args[1], args[3], args[6], flags=1 if x is a else 0)
            c.attn(*args, params=p)
    assert c.poll_status() == 0
    for x in (a, d):
        ref, bar = x.reference()
        got = [o for y, o in outs if y is x]
        assert all(torch.equal(g, got[0]) for g in got)
        assert bool(((got[0].double().cpu() - ref).abs() <= bar).all())


def test_a_token_from_projection_to_token():
    """The three calls as a loop uses them: rows into the cache, attention with rules, logits to the next token; a step of
    eight tokens one by one equals the step as one chunk."""
    c, hq, hkv, D, B, n, V = H.ctx(), 8, 2, 128, 3, 8, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    start = [40, 7, 200]
    table = torch.arange(B * 16, device="cuda", dtype=torch.int32).view(B, 16)
    pools = [rnd(B * 16, hkv, P, D) for _ in range(2)]
    pools2 = [p.clone() for p in pools]
    qkv = rnd(B, n, (hq + 2 * hkv) * D)
    freq = 10000.0 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float32) * 2 / D)
    head = rnd(hq * D, V) * 0.05
    wq = torch.rand(D, generator=g, device="cuda") + 0.5
    rules = dict(cap=20.0, window=64, slopes=None)

    def split(x):
        return [t.reshape(x.shape[0], -1, D) for t in x.split((hq * D, hkv * D, hkv * D), dim=1)]

    lens, ones = torch.tensor(start, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    rows, tokens = [], []
    for t in range(n):
        q, k, v = split(qkv[:, t].contiguous())
        q = c.rope_append(q, k, v, freq, table, lens, ones, *pools, wq, wq)
        o = c.attn_rules(q, *pools, table, lens, ones, 1, **rules)
        rows.append(o)
        _, token, _ = c.logits(o.reshape(B, -1) @ head, want_out=False)
        tokens.append(token)
    lens2, new = torch.tensor(start, dtype=torch.int32, device="cuda"), torch.full((B,), n, dtype=torch.int32, device="cuda")
    q, k, v = split(qkv.reshape(B * n, -1))
    q = c.rope_append(q, k, v, freq, table, lens2, new, *pools2, wq, wq)
    whole = c.attn_rules(q, *pools2, table, lens2, new, n, **rules).view(B, n, hq, D)
    assert c.poll_status() == 0
    assert torch.equal(lens, lens2) and all(torch.equal(a, b) for a, b in zip(pools, pools2))
    # both sides: weights rounded to bf16 (2^-8 of sum p |v| <= 4.5) and the outputs' own rounding
    assert float((torch.stack(rows, 1).double() - whole.double()).abs().max()) <= 2 * (2.0 ** -8 * 4.5 + 2.0 ** -8 * 4.5)
    assert torch.stack(tokens).shape == (n, B) and bool((torch.stack(tokens) >= 0).all())
