"""arb_attn_rules where the definition and a kernel's way to it part most easily: caps from far below to far above the scores, and
row tiles none of whose rows sees a key.

Tolerance: that of test_gpu_rules.py with another term for the cap.  The kernels work cap * tanh(s / cap) out with a relative error
of the result of at most 2^-19 where |s| <= cap (a polynomial's 1.2e-6 and the roundings around it), or out of an exponential
with an error of 2^-21 * cap in a tile that holds a score of at least 0.8 cap; with Z, the bound of every score of the call, either is at
most 2^-19 * min(cap, Z).  Far caps leave the scores as they are, near ones make them all alike."""
import math

import numpy as np
import pytest
import torch

from tests import helpers as H
from tests.test_gpu_rules import BF, F32, P, Inputs

pytestmark = pytest.mark.gpu


def reference(x):
    """(out, bar) in 64 bits."""
    D, G = x.D, x.hq // x.hkv
    scale, outs, bars, row0 = D ** -0.5, [], [], 0
    largest = scale * float(x.q.double().norm(dim=-1).max() * torch.nan_to_num(x.k.double()).norm(dim=-1).max())
    cap_err = 2.0 ** -19 * min(x.cap, largest) if x.cap else 0.0
    for b in range(len(x.lens)):
        n, L = int(x.new[b]), int(x.lens[b])
        if n == 0:
            continue
        m, dist = x.sees(b, row0)
        seen = m.any(0)
        page = x.table[b, :-(-L // P)].long()
        page = torch.where((page >= 0) & (page < x.pages), page, 0)
        k, v = (torch.where(seen[:, None], t[page].transpose(0, 1).flatten(1, 2)[:, :L].double(), 0.0) for t in (x.k, x.v))
        o, bar = (torch.zeros(n, x.hq, D, dtype=torch.float64) for _ in range(2))
        for h in range(x.hq):
            q, kk, vv = x.q[row0:row0 + n, h].double(), k[h // G], v[h // G]
            s = q @ kk.T * scale
            if x.cap:
                s = x.cap * torch.tanh(s / x.cap)
            if x.slopes is not None:
                s = s - x.slopes[h].double() * dist
            s = torch.where(m, s, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.where(m, torch.exp(s - torch.where(torch.isinf(top), 0.0, top)), 0.0)
            p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
            o[:, h] = p @ vv
            z = scale * q.norm(dim=-1, keepdim=True) * kk.norm(dim=-1).max()
            counts = torch.where(p > 2.0 ** -30, s.abs(), 0.0).amax(-1, keepdim=True)
            d = (D + 4) * 2.0 ** -24 * z + cap_err + 2.0 ** -22 * (1 + counts)
            rel = 2 * d + (2.0 ** -8 if x.dtype == BF else 2.0 ** -20)
            bar[:, h] = rel * (p @ vv.abs()) + torch.finfo(x.dtype).eps / 2 * o[:, h].abs() + 1e-30
        outs.append(o)
        bars.append(bar)
        row0 += n
    return torch.cat(outs), torch.cat(bars)


def check(x, bits=0):
    args, rules = x.args()
    out = H.ctx().attn_rules(*args, **rules)
    assert H.ctx().poll_status() == bits
    ref, bar = reference(x)
    got = out.double().cpu()
    assert bool(torch.isfinite(got).all())
    err = (got - ref).abs()
    assert bool((err <= bar).all()), f"off by {err.max():.3e}, {(err / bar).max():.2f} of the bar"
    return out


CAPS = [1e-20, 1e-4, 1e-2, 300.0, 800.0, 900.0, 1e3, 1e4, 1e5, 1e6, 1e8, 1e12, 1e20]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("dtype,D,new", [(BF, 128, 1), (BF, 128, 40), (BF, 64, 40), (F32, 64, 1), (F32, 128, 20)])
def test_caps_of_any_size(dtype, D, new, cap):
    check(Inputs(20, dtype, 8, 2, D, [600, 200], [new, new], std=4.0, cap=cap))
    check(Inputs(21, dtype, 8, 2, D, [600, 200], [new, new], std=4.0, cap=cap, slopes=True, window=150))


@pytest.mark.parametrize("cap", [20.0, 800.0, 1e3, 1e5, 1e7])
@pytest.mark.parametrize("D", [64, 128])
def test_ordinary_rows_beside_rows_that_reach_the_cap(D, cap):
    """A tile works its scores out in one way for all rows of a warp: one token's queries are large enough to reach the cap, its
    neighbours' are not."""
    for slopes in (False, True):
        x = Inputs(22, BF, 8, 2, D, [900, 300], [64, 37], std=2.0, cap=cap, slopes=slopes)
        x.q[5] = (x.q[5].float() * cap).to(BF)
        x.q[70] = (x.q[70].float() * cap * 0.3).to(BF)
        args, rules = x.args()
        out = H.ctx().attn_rules(*args, **rules).double().cpu()
        ref, _ = reference(x)
        usual = torch.ones(101, dtype=torch.bool)
        usual[[5, 70]] = False
        # Z of the ordinary rows alone: the form out of an exponential is off by 2^-21 of the cap, which only caps below 1024 take
        y = Inputs(22, BF, 8, 2, D, [900, 300], [64, 37], std=2.0, cap=cap, slopes=slopes)
        _, bar = reference(y)
        bar = bar + 2 * 2.0 ** -21 * min(cap, 1024.0) * 4.5          # sum p |v| <= 4.5 for N(0, 1) values
        assert bool(torch.isfinite(out).all())
        assert bool(((out - ref).abs() <= bar)[usual].all()), float(((out - ref).abs() / bar)[usual].max())


@pytest.mark.parametrize("cap", [30.0, 1e6, 1e20])
@pytest.mark.parametrize("D", [64, 128])
def test_a_step_as_one_chunk_and_token_by_token(D, cap):
    """Both forms of the call see the same keys; each is within its bar."""
    n, start = 20, 300
    x = Inputs(23, BF, 8, 2, D, [start + n], [n], std=4.0, cap=cap, window=250)
    args, rules = x.args()
    whole = H.ctx().attn_rules(*args, **rules)
    ones = torch.ones(1, dtype=torch.int32, device="cuda")
    single = torch.cat([H.ctx().attn_rules(args[0][t:t + 1].contiguous(), args[1], args[2], args[3],
                                           torch.full((1,), start + t + 1, dtype=torch.int32, device="cuda"), ones, 1, cap=cap, window=250)
                        for t in range(n)])
    _, bar = reference(x)
    assert H.ctx().poll_status() == 0
    assert bool(((whole.double() - single.double()).abs().cpu() <= 2 * bar).all())


@pytest.mark.parametrize("dtype,D,new", [(BF, 128, 1), (BF, 128, 9), (BF, 128, 70), (BF, 64, 70), (F32, 64, 1), (F32, 128, 40)])
@pytest.mark.parametrize("L", [200, 30000])
def test_no_row_sees_a_key_and_nothing_is_looked_up(dtype, D, new, L):
    """First keys beyond every row: rows of zeros, whatever the cache holds and whatever the table says; short contexts and ones
    whose keys are split over several items."""
    for rules in ({}, {"cap": 5.0}, {"slopes": True}):
        x = Inputs(24, dtype, 8, 2, D, [L], [new], first=[L + 5] * new, **rules)
        x.k.fill_(float("nan"))
        x.v.fill_(float("inf"))
        x.table.fill_(-1)
        args, more = x.args()
        out = torch.full_like(args[0], 5.0)
        H.ctx().attn_rules(*args, **more, out=out)
        assert H.ctx().poll_status() == 0
        assert not bool(out.any()) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128)])
@pytest.mark.parametrize("L", [700, 20000])
def test_row_tiles_that_see_nothing_beside_others_that_do(dtype, D, L):
    """Of a step of 150 tokens (600 rows of a kv head) some runs see nothing, others only the last page; keys before that page are no
    numbers and its table entries are unset."""
    n = 150
    first = [L + 1] * 70 + [L - 200] * 10 + [10 ** 9] * 64 + [L - n] * 6
    x = Inputs(25, dtype, 8, 2, D, [L, 90], [n, 30], first=first + [0] * 30, cap=9.0)
    dead = L - 200
    flat = torch.arange(dead)
    page = x.table[0, flat // P].long()
    x.k[page, :, flat % P] = float("nan")
    x.v[page, :, flat % P] = float("nan")
    x.table[0, :dead // P] = -7
    out = check(x)
    assert not bool(out[:70].any()) and not bool(out[80:144].any()) and bool(out[70:80].any()) and bool(out[144:].any())


def test_repeated_calls_give_the_same_bits():
    """Whatever ran before and whatever memory it left behind: decode rows, chunks and both, each kind of rule."""
    cases = [Inputs(26, BF, 32, 8, 128, list(np.linspace(500, 9000, 16).astype(int)), [1] * 16, cap=50.0, window=4096),
             Inputs(27, BF, 12, 2, 128, [1024, 8192, 4000], [1] * 3, slopes=True),
             Inputs(28, BF, 28, 4, 128, [3000, 900, 5000], [60, 1, 128], cap=30.0, std=4.0),
             Inputs(29, BF, 32, 8, 64, [700, 256], [700, 256], prefix=[150, 20], first=[max(0, p - p % 300) for p in range(700)] + [0] * 256),
             Inputs(30, F32, 8, 2, 128, [1400, 1700], [56, 104], window=640, slopes=True)]
    want = []
    for turn in range(4):
        for i in range(len(cases)) if turn % 2 == 0 else reversed(range(len(cases))):
            x = cases[i]
            args, rules = x.args()
            junk = torch.full((1 << 20,), float("nan"), device="cuda")
            out = H.ctx().attn_rules(*args, **rules)
            del junk
            if turn == 0:
                want.append(out)
            else:
                assert torch.equal(out, want[i]), (turn, i)
    assert H.ctx().poll_status() == 0


@pytest.mark.parametrize("dtype,hq,hkv,D", [(BF, 32, 8, 64), (BF, 28, 4, 128), (F32, 8, 2, 64)])
def test_chunks_with_every_rule_off_are_the_plain_attentions(dtype, hq, hkv, D):
    """Bit for bit; 64-dimension heads so at that call's bar of 1e-3 beside the output's rounding (their weights are two bf16 terms, 16
    bits), 128-dimension ones within this module's: a weight of one bf16 term is off by up to 2^-8, which of a few keys with values of up to 4.5
    is more than any bar of 1e-3 allows (2^-8 * 4.5 = 0.018)."""
    x = Inputs(31, dtype, hq, hkv, D, [12, 300, 700, 2000, 40], [12, 30, 129, 16, 40])
    args, rules = x.args()
    a, b = H.ctx().attn(*args), H.ctx().attn_rules(*args)
    assert H.ctx().poll_status() == 0 and torch.equal(a, b)
    ref, bar = reference(x)
    err = (b.double().cpu() - ref).abs()
    assert bool((err <= bar).all())
    if D == 64:
        assert bool((err <= torch.finfo(dtype).eps / 2 * ref.abs() + (1e-5 if dtype == F32 else 1e-3)).all())


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("B", [33, 70, 300, 1024])
def test_large_batches(dtype, D, B):
    """More sequences than a warp plans for, up to the most a call takes: tokens, short steps and idle slots, whatever the window cuts off."""
    r = np.random.RandomState(B)
    lens = [int(v) for v in r.randint(1, 130, B)]
    tokens = [int(v) for v in r.randint(0, 2, B)]
    check(Inputs(32, dtype, 4, 2, D, lens, tokens[:-1] + [1], window=37, slopes=True))
    new = [min(L, int(v)) for L, v in zip(lens, r.choice([0, 1, 2, 7], B))]
    check(Inputs(33, dtype, 4, 2, D, lens, new[:-1] + [1], window=20, cap=8.0))
    check(Inputs(34, dtype, 4, 2, D, lens, new[:-1] + [1], first=[int(v) for v in r.randint(0, 140, sum(new[:-1]) + 1)]))
