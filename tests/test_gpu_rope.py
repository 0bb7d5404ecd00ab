"""arb_rope_append and its quantising forms against the formulas in 64 bits.

Tolerance.  In fp32 a normed value carries the errors of a 128-term sum of squares (7 levels of adding and the products: 8 units of
2^-24, halved by the root), of rsqrt (2^-22), of three products; a rotated one those of two such values, of sine and cosine (2^-22
each with the reduced angle) and of the sum: together below 2^-19 of |a| + |b| of its pair.  The output's rounding comes on top,
finfo.eps / 2 of the value.  An E4M3 code may be the neighbour where the value lies within the fp32 error of the border of two
codes: the decoded value is off by at most half a step of the format (2^-4 relative, 2^-10 absolute below the smallest normal)
plus that error.  A 4-bit value is off by half a code, scale / 2, and the scale by the error of the row's largest value."""
import numpy as np
import pytest
import torch

from tests import helpers as H

pytestmark = pytest.mark.gpu
P = 16


def _binding():
    from paper_2512_05033_b200 import binding
    return binding


def make(seed, dtype, hq, hkv, D, before, new, rot, pages_extra=3, std=1.0, table_slack=0):
    g = torch.Generator().manual_seed(seed)
    B, T = len(new), sum(new)
    need = [-(-(b + n) // P) for b, n in zip(before, new)]
    pages = sum(need) + pages_extra
    order = torch.randperm(pages, generator=g)
    width = max(max(need), 1) + table_slack
    table, at = torch.full((B, width), -1, dtype=torch.int32), 0
    for b, c in enumerate(need):
        table[b, :c] = order[at:at + c].int()
        at += c
    qkv = (torch.randn(T, (hq + 2 * hkv) * D, generator=g) * std).to(dtype)
    inv_freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) * 2 / max(rot, 1))
    w = lambda: 1 + 0.3 * torch.randn(D, generator=g)  # noqa: E731
    d = dict(qkv=qkv, table=table, before=torch.tensor(before, dtype=torch.int32), new=torch.tensor(new, dtype=torch.int32),
             inv_freq=inv_freq, q_weight=w(), k_weight=w(), pages=pages, hq=hq, hkv=hkv, D=D, rot=rot, dtype=dtype, g=g)
    return d


def views(d, device="cuda", fused=True):
    hq, hkv, D = d["hq"], d["hkv"], d["D"]
    x = d["qkv"].to(device)
    q, k, v = x.split((hq * D, hkv * D, hkv * D), dim=1)
    out = [t.view(t.shape[0], h, D) for t, h in ((q, hq), (k, hkv), (v, hkv))]
    return out if fused else [t.contiguous() for t in out]


def reference(d, norm, inter, eps, positions=None):
    """(q, k) rows in 64 bits, the |a| + |b| of each element's pair, and (sequence, place) of each row."""
    q, k, _ = views(d, "cpu")
    T, rot, D = q.shape[0], d["rot"], d["D"]
    seq = torch.repeat_interleave(torch.arange(len(d["new"])), d["new"].clamp(min=0).long())
    start = torch.cumsum(d["new"].clamp(min=0).long(), 0) - d["new"].clamp(min=0).long()
    place = d["before"].long()[seq] + torch.arange(len(seq)) - start[seq]
    pos = (place if positions is None else positions[:len(seq)].long()).double()
    outs, mags = [], []
    for x, w in ((q, d["q_weight"]), (k, d["k_weight"])):
        x = x[:len(seq)].double()
        if norm:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        angle = pos[:, None, None] * d["inv_freq"].double()
        c, s = torch.cos(angle), torch.sin(angle)
        i = torch.arange(rot // 2)
        ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        y, mag = x.clone(), x.abs().clone()
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
        mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
        outs.append(y)
        mags.append(mag)
    return outs, mags, seq, place


def close(got, ref, mag, dtype):
    err = (got.double().cpu() - ref).abs()
    bar = 2.0 ** -19 * mag + torch.finfo(dtype).eps / 2 * ref.abs() + 1e-30
    assert bool((err <= bar).all()), f"off by {err.max():.3e}, {(err / bar).max():.2f} of the bar"


CASES = [
    # dtype, Hq, Hkv, D, before, new, rot, norm, interleaved
    (torch.bfloat16, 12, 2, 128, [1023, 0, 15, 16], [1, 1, 1, 1], 128, True, False),
    (torch.bfloat16, 28, 4, 128, [5, 0, 100, 31], [17, 0, 1, 130], 128, True, True),
    (torch.bfloat16, 32, 8, 64, [0, 7], [33, 300], 32, False, False),
    (torch.float32, 8, 2, 64, [512], [16], 64, True, False),
    (torch.float32, 5, 3, 128, [3, 0, 1 << 20], [2, 0, 40], 16, True, True),
    (torch.bfloat16, 1, 1, 128, [0], [1], 0, False, False),
    (torch.bfloat16, 7, 7, 64, [9] * 40, [0, 1, 3] * 13 + [5], 48, True, False),
    (torch.bfloat16, 32, 8, 128, [0, 0, 0], [700, 1, 900], 96, True, True),
]


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_rows_and_cache(case, fused):
    dtype, hq, hkv, D, before, new, rot, norm, inter = case
    d = make(1, dtype, hq, hkv, D, before, new, rot)
    q, k, v = views(d, fused=fused)
    c = H.ctx()
    kp = torch.randn(d["pages"], hkv, P, D, device="cuda").to(dtype)
    vp = torch.randn(d["pages"], hkv, P, D, device="cuda").to(dtype)
    k0, v0 = kp.clone(), vp.clone()
    lens = d["before"].cuda()
    wq, wk = (d["q_weight"].cuda(), d["k_weight"].cuda()) if norm else (None, None)
    buf = torch.full((q.shape[0] + 2, hq, D), 777.0, dtype=dtype, device="cuda")
    out = c.rope_append(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), lens, d["new"].cuda(), kp, vp, wq, wk, 1e-5, inter,
                        q_out=buf[1:-1])
    assert c.poll_status() == 0
    (rq, rk), (mq, mk), seq, place = reference(d, norm, inter, 1e-5)
    close(out, rq, mq, dtype)
    assert bool((buf[0] == 777).all()) and bool((buf[-1] == 777).all())
    page = d["table"][seq, place // P].long()
    close(kp[page.cuda(), :, (place % P).cuda()], rk, mk, dtype)
    assert torch.equal(vp[page.cuda(), :, (place % P).cuda()], v)
    # everything else of the pools is as it was
    kp[page.cuda(), :, (place % P).cuda()] = k0[page.cuda(), :, (place % P).cuda()]
    vp[page.cuda(), :, (place % P).cuda()] = v0[page.cuda(), :, (place % P).cuda()]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    assert lens.tolist() == [b + n for b, n in zip(before, new)]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [(torch.bfloat16, 128, 128), (torch.float32, 64, 32), (torch.float32, 128, 16), (torch.bfloat16, 64, 64)])
def test_e4m3_cache(dtype, D, rot, inter):
    d = make(2, dtype, 6, 2, D, [0, 40, 17], [30, 1, 77], rot, std=2.0)
    q, k, v = views(d)
    c = H.ctx()
    kc = torch.randint(0, 100, (d["pages"], 2, P, D), dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    lens = d["before"].cuda()
    out = c.rope_append_e4m3(q, k, v, d["inv_freq"].cuda(), 30.0, 12.0, d["table"].cuda(), lens, d["new"].cuda(), kc, vc,
                             d["q_weight"].cuda(), d["k_weight"].cuda(), 1e-6, inter, update_lens=False)
    assert c.poll_status() == 0
    (rq, rk), (mq, mk), seq, place = reference(d, True, inter, 1e-6)
    close(out, rq, mq, dtype)
    page, slot = d["table"][seq, place // P].long().cuda(), (place % P).cuda()
    got = kc[page, :, slot].view(torch.float8_e4m3fn).double().cpu()
    want = (rk * 30.0).clamp(-448, 448)
    assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 + 30.0 * 2.0 ** -18 * mk).all())
    codes = (v.float() * 12.0).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(vc[page, :, slot], codes)          # values: bit for bit
    assert lens.tolist() == d["before"].tolist()


@pytest.mark.parametrize("rot,inter", [(128, False), (128, True), (64, False), (16, False), (32, True), (0, False)])
def test_i4_cache(rot, inter):
    from oracle import oracle
    d = make(3, torch.bfloat16, 4, 2, 128, [0, 33], [50, 20], rot)
    d["qkv"][7] = 0                                          # a token of zeros: scale 0
    q, k, v = views(d)
    c = H.ctx()
    kc, vc = (torch.zeros(d["pages"], 2, P, 64, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((d["pages"], 2, P), -1.0, device="cuda") for _ in range(2))
    wk = d["k_weight"].cuda()
    c.rope_append_i4(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), d["before"].cuda(), d["new"].cuda(), kc, vc, ks, vs, None, wk,
                     1e-6, inter)
    assert c.poll_status() == 0
    d2 = dict(d, q_weight=torch.ones(128))
    (_, rk), (_, mk), seq, place = reference(d2, True, inter, 1e-6)
    page, slot = d["table"][seq, place // P].long().cuda(), (place % P).cuda()
    # values: the format's own encoder, bit for bit (the append's)
    kc2, vc2, ks2, vs2 = kc.clone(), vc.clone(), ks.clone(), vs.clone()
    c.kv_append_i4(k.contiguous(), v.contiguous(), d["table"].cuda(), d["before"].cuda(), d["new"].cuda(), kc2, vc2, ks2, vs2)
    assert torch.equal(vc, vc2) and torch.equal(vs, vs2)
    # keys: unpack the words and compare with the rotated keys
    words = kc[page, :, slot].cpu().numpy().view(np.uint32)                  # [T, 2, 16]
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    vals = np.zeros(words.shape + (8,))
    for nib, dim in enumerate(order):
        vals[..., dim] = ((words >> (4 * nib)) & 15).astype(np.int64) - 8
    scale = ks[page, :, slot].double().cpu()
    got = torch.from_numpy(vals).reshape(len(seq), 2, 128) * scale[..., None]
    big = rk.abs().amax(-1)
    assert bool(((scale - big / 7).abs() <= 2.0 ** -18 * mk.amax(-1) + 2.0 ** -24 * big).all())
    assert bool(((got - rk).abs() <= scale[..., None] * 0.5 * (1 + 2.0 ** -20) + 2.0 ** -16 * mk.amax(-1, keepdim=True)).all())
    assert bool((scale[7] == 0).all()) and not bool(got[7].any())


def test_far_positions_keep_their_angles():
    """Positions near 2^30 by the `positions` argument, neighbours apart by one: an angle worked out in fp32 would be off by radians."""
    d = make(4, torch.float32, 2, 1, 64, [0], [4], 64)
    q, k, v = views(d)
    pos = torch.tensor([0, (1 << 30) - 1, 1 << 30, -5], dtype=torch.int32)
    kp, vp = (torch.zeros(d["pages"], 1, P, 64, device="cuda") for _ in range(2))
    c = H.ctx()
    out = c.rope_append(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), d["before"].cuda(), d["new"].cuda(), kp, vp,
                        positions=pos.cuda())
    d["q_weight"] = d["k_weight"] = torch.ones(64)
    (rq, _), (mq, _), _, _ = reference(d, False, False, 0, pos)
    close(out, rq, mq, torch.float32)


def test_refused_sequences_are_left_alone():
    b = _binding()
    for kind, bits in (("fit", b.DEV_BAD_SEQ_LEN), ("page", b.DEV_BAD_PAGE), ("page_below", b.DEV_BAD_PAGE), ("negative", b.DEV_BAD_SEQ_LEN)):
        d = make(5, torch.bfloat16, 4, 2, 128, [10, 20, 30], [5, 6, 7], 128)
        if kind == "fit":
            d["before"][1] = d["table"].shape[1] * P - 5
        elif kind == "negative":
            d["before"][1] = -1
        else:
            d["table"][1, 1] = d["pages"] if kind == "page" else -7
        q, k, v = views(d)
        c = H.ctx()
        kp, vp = (torch.full((d["pages"], 2, P, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lens = d["before"].cuda()
        out = c.rope_append(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), lens, d["new"].cuda(), kp, vp)
        assert c.poll_status() == bits
        assert lens.tolist() == [15, int(d["before"][1]), 37]
        assert not bool(out[5:11].any()) and bool(out[:5].any()) and bool(out[11:].any())
        written = {int(d["table"][s, (int(d["before"][s]) + j) // P]) * P + (int(d["before"][s]) + j) % P for s, n in ((0, 5), (2, 7)) for j in range(n)}
        touched = (kp != 3).any(-1).any(1).reshape(-1).nonzero().flatten().tolist()
        assert set(touched) <= written and len(touched) == 12
        assert c.poll_status() == 0


def test_lengths_that_add_up_to_more_than_there_is():
    """Lengths on the device whose sum passes 32 bits, and total_new: refused where they do not fit, never read past the rows."""
    b = _binding()
    d = make(9, torch.bfloat16, 4, 2, 64, [0, 0, 0, 0], [3, 4, 2, 3], 64)
    q, k, v = views(d)
    c = H.ctx()
    for new in ([2 ** 31 - 1, 5, 2 ** 31 - 1, 7], [2 ** 30] * 4, [3, 2 ** 31 - 1, 2, 3]):
        kp, vp = (torch.zeros(d["pages"], 2, P, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        buf = torch.full((q.shape[0] + 2, 4, 64), 777.0, dtype=torch.bfloat16, device="cuda")
        c.rope_append(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), d["before"].cuda(), torch.tensor(new, dtype=torch.int32, device="cuda"),
                      kp, vp, q_out=buf[1:-1], update_lens=False)
        assert c.poll_status() == b.DEV_BAD_SEQ_LEN
        assert bool((buf[0] == 777).all()) and bool((buf[-1] == 777).all())
        first = 0 if new[0] > 100 else new[0]
        assert not bool(buf[1 + first:-1].any())            # rows of the refused sequence, up to the last there is
        assert first == 0 or bool(buf[1:1 + first].any())


def test_rows_behind_the_last_sequence_stay():
    d = make(6, torch.bfloat16, 4, 2, 64, [3, 0], [2, 3], 64)
    q, k, v = (torch.cat((t, t)) for t in views(d))
    c = H.ctx()
    kp, vp = (torch.zeros(d["pages"], 2, P, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.full(tuple(q.shape), 9.0, dtype=torch.bfloat16, device="cuda")
    c.rope_append(q, k, v, d["inv_freq"].cuda(), d["table"].cuda(), d["before"].cuda(), d["new"].cuda(), kp, vp, q_out=out)
    assert bool((out[5:] == 9).all()) and not bool((out[:5] == 9).all())


def test_in_place_and_a_stream_of_its_own_and_a_graph():
    d = make(7, torch.bfloat16, 12, 2, 128, [100, 3], [1, 1], 128)
    c = _binding().Context(0)
    q, k, v = views(d, fused=False)
    table, new, freq, wq = d["table"].cuda(), d["new"].cuda(), d["inv_freq"].cuda(), d["q_weight"].cuda()
    kp, vp = (torch.zeros(d["pages"], 2, P, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    want = c.rope_append(q, k, v, freq, table, d["before"].cuda(), new, kp, vp, wq)
    k1 = kp.clone()
    torch.cuda.synchronize()
    # in place
    q2, lens = q.clone(), d["before"].cuda()
    c.rope_append(q2, k, v, freq, table, lens, new, kp, vp, wq, q_out=q2)
    assert torch.equal(q2, want)
    # on another stream than the current one, then captured and replayed: lengths advance with every replay
    s = torch.cuda.Stream()
    lens = d["before"].cuda()
    kp.zero_()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    c.rope_append(q, k, v, freq, table, lens, new, kp, vp, wq, q_out=out, update_lens=False, stream=s)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(kp, k1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            c.rope_append(q, k, v, freq, table, lens, new, kp, vp, wq, q_out=out)
    for i in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert lens.tolist() == [103, 6] and c.poll_status() == 0
    c.close()


def test_the_attention_reads_what_was_written():
    """rope_append then attn equals norm, rotation and kv_append done apart, bit for bit where the rows agree."""
    d = make(8, torch.bfloat16, 8, 2, 128, [0, 0], [40, 70], 128)
    q, k, v = views(d)
    c = H.ctx()
    kp, vp = (torch.zeros(d["pages"], 2, P, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens, table, new = d["before"].cuda(), d["table"].cuda(), d["new"].cuda()
    qo = c.rope_append(q, k, v, d["inv_freq"].cuda(), table, lens, new, kp, vp, d["q_weight"].cuda(), d["k_weight"].cuda())
    out = c.attn(qo, kp, vp, table, lens, new, 70)
    (rq, rk), _, seq, _ = reference(d, True, False, 1e-6)
    for b, rows in enumerate((range(0, 40), range(40, 110))):
        rows = list(rows)
        for h in (0, 5):
            s = rq[rows, h] @ rk[rows, h // 4].T / 128 ** 0.5
            s = s.masked_fill(torch.triu(torch.ones(len(rows), len(rows), dtype=torch.bool), 1), -np.inf)
            want = torch.softmax(s, -1) @ v[rows, h // 4].double().cpu()
            # q, k and the weights rounded to bf16: 2^-8 each of scores up to |q| |k| / sqrt(D) <= 40 and of weights
            assert float((out[rows, h].double().cpu() - want).abs().max()) < 6e-2


@pytest.mark.parametrize("kind", ["rope", "rope_e4m3", "rope_i4", "append", "append_e4m3", "append_i4"])
def test_sequences_whose_rows_are_not_there_are_refused(kind):
    """new_lens on the device that fit the block table but add up to more than the rows of the call: sequences that end behind the last
    row keep their pools and lengths and raise the bad-length bit, the others are written."""
    b, c = _binding(), H.ctx()
    for new, total, okay in (([3, 4, 2, 3], 12, 4), ([3, 4, 5, 3], 12, 3), ([3, 4, 5, 0], 11, 2), ([13, 0, 1, 0], 12, 0), ([12, 1, 0, 0], 12, 1)):
        d = make(10, torch.bfloat16, 4, 2, 128, [0, 17, 5, 20], [14] * 4, 128)
        q, k, v = (t[:total].contiguous() for t in views(d))
        table, lens, n = d["table"].cuda(), d["before"].cuda(), torch.tensor(new, dtype=torch.int32, device="cuda")
        bf = dict(dtype=torch.bfloat16, device="cuda")
        pools = [torch.full((d["pages"], 2, P, 128), 3.0, **bf) for _ in range(2)]
        codes = [torch.full((d["pages"], 2, P, 64 if kind.endswith("i4") else 128), 7, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.full((d["pages"], 2, P), 7.0, device="cuda") for _ in range(2)]
        freq = d["inv_freq"].cuda()
        if kind == "rope":
            out = c.rope_append(q, k, v, freq, table, lens, n, *pools)
        elif kind == "rope_e4m3":
            out = c.rope_append_e4m3(q, k, v, freq, 16.0, 16.0, table, lens, n, *codes)
        elif kind == "rope_i4":
            out = c.rope_append_i4(q, k, v, freq, table, lens, n, *codes, *scales)
        elif kind == "append":
            c.kv_append(k, v, table, lens, n, *pools)
        elif kind == "append_e4m3":
            c.kv_append_e4m3(k, v, 16.0, 16.0, table, lens, n, *codes)
        else:
            c.kv_append_i4(k, v, table, lens, n, *codes, *scales)
        rows, ends = [], np.cumsum(new)
        for s in range(4):
            rows.append(int(d["before"][s]) + (new[s] if ends[s] <= total else 0))
        short = [s for s in range(4) if new[s] and ends[s] > total]
        assert c.poll_status() == (b.DEV_BAD_SEQ_LEN if short else 0)
        assert lens.tolist() == rows
        pool = pools[0] if kind in ("rope", "append") else codes[0]
        base = 3 if kind in ("rope", "append") else 7
        touched = set((pool != base).any(-1).any(1).reshape(-1).nonzero().flatten().tolist())
        written = {int(d["table"][s, p // P]) * P + p % P for s in range(4) if s not in short for p in range(int(d["before"][s]), int(d["before"][s]) + new[s])}
        assert touched == written
        if kind.startswith("rope"):
            full = int(ends[max((s for s in range(4) if ends[s] <= total), default=0)]) if ends[0] <= total else 0
            assert not bool(out[full:].any()) if short else bool(out[:full].any())
