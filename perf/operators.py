"""What one token needs around and inside the attention, in a plain form and as the library's calls.

Every case is a dict of plain values; `op` names the operator:

  rope_append  queries and keys normed per head and rotated, keys and values written into the paged cache
               (Context.rope_append, Context.rope_append_e4m3)
  attn_rules   attention over the paged cache with capped scores, a bias by distance, a window, a two-sided prefix and
               documents (Context.attn_rules)
  logits       penalties, biases and an allowed-token mask on a batch of logits, the next token and its log-probability
               (Context.logits)

Lengths are spread evenly over a case's range, so that the work of a case does not depend on the seed; the seed gives the
order of the sequences, the pages and every value.
"""
import math
import random

import torch

PAGE = 16
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
DTYPES = {"bf16": BF16, "fp32": F32}
GEOMETRIES = ((12, 2), (28, 4), (32, 8))   # query / KV heads: draft-, router- and target-shaped
E4M3_MAX = 448.0
own = False

_ctx = None


def _context():
    global _ctx
    if _ctx is None:
        from paper_2512_05033_b200 import binding
        _ctx = binding.Context(0)
    return _ctx


# ---- the cases ----------------------------------------------------------------------------------------------------

def _rope(name, kv, dtype, B, heads, lo, hi, n_lo, n_hi, head_dim=128, rot=128, interleaved=False, norm=True):
    return {"name": name, "op": "rope_append", "kv": kv, "dtype": dtype, "batch": B, "hq": heads[0], "hkv": heads[1],
            "head_dim": head_dim, "rot": rot, "interleaved": interleaved, "norm": norm,
            "lo": lo, "hi": hi, "n_lo": n_lo, "n_hi": n_hi}


def _rules(name, dtype, B, heads, lo, hi, n_lo, n_hi, head_dim=128, cap=0.0, window=0, slopes=False, prefix=0, document=0):
    return {"name": name, "op": "attn_rules", "dtype": dtype, "batch": B, "hq": heads[0], "hkv": heads[1],
            "head_dim": head_dim, "lo": lo, "hi": hi, "n_lo": n_lo, "n_hi": n_hi, "cap": cap, "window": window,
            "slopes": slopes, "prefix": prefix, "document": document}


def _logits(name, dtype, rows, vocab, history, penalties=True, biases=0, mask=False, sampled=False):
    return {"name": name, "op": "logits", "dtype": dtype, "rows": rows, "vocab": vocab, "history": history,
            "penalties": penalties, "biases": biases, "mask": mask, "sampled": sampled}


def listed():
    return [
        # a draft token's queries, keys and values on their way to the cache: once per token and layer, latency alone
        _rope("token_write", "same", "bf16", 8, (12, 2), 1024, 8192, 1, 1),
        # the prompts of a batch: as much as one call of this loop writes
        _rope("prompt_write", "same", "bf16", 16, (32, 8), 0, 0, 256, 2048),
        # finished steps absorbed by a quantised draft's cache; neighbouring dimensions rotate together, half of them
        _rope("step_write_e4m3", "e4m3", "bf16", 32, (28, 4), 2048, 16384, 16, 128, rot=64, interleaved=True, norm=False),
        # a target token with capped scores and a window over long contexts
        _rules("target_token_windowed", "bf16", 16, (32, 8), 4096, 32768, 1, 1, cap=50.0, window=4096),
        # a draft token whose scores fall off with distance
        _rules("draft_token_slopes", "bf16", 8, (12, 2), 1024, 8192, 1, 1, slopes=True),
        # the smallest call: one sequence, fp32, 64-dimension heads
        _rules("tiny_token", "fp32", 1, (8, 2), 513, 513, 1, 1, head_dim=64, cap=30.0, slopes=True),
        # a batch of steps scored by a model with capped scores
        _rules("step_scoring_capped", "bf16", 32, (28, 4), 2048, 16384, 16, 128, cap=30.0),
        # prompts of several documents behind a prefix that reads both ways, 64-dimension heads
        _rules("prompt_documents", "bf16", 16, (32, 8), 0, 0, 256, 2048, head_dim=64, prefix=200, document=700),
        # fp32 steps in a window with a bias by distance
        _rules("step_window_fp32", "fp32", 2, (8, 2), 1300, 1800, 56, 104, window=640, slopes=True),
        # one greedy row of a small vocabulary
        _logits("logits_greedy", "bf16", 1, 32000, 500),
        # a batch of sampled rows with everything a request can ask for
        _logits("logits_sampled", "bf16", 64, 128001, 4096, biases=64, mask=True, sampled=True),
        # a batch in fp32 under a grammar
        _logits("logits_grammar", "fp32", 24, 50003, 300, penalties=False, biases=16, mask=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        case.pop("name")
        if _cost(case) <= most and _plain_bytes(case) <= 16e9:
            return case


def _draw(rng):
    op = rng.choice(("rope_append", "attn_rules", "attn_rules", "logits"))
    if op == "logits":
        return _logits("", rng.choice(("bf16", "fp32")), _log_int(rng, 1, 128), _log_int(rng, 2000, 160000),
                       _log_int(rng, 1, 6000), rng.random() < 0.7, rng.choice((0, 1, 40, 300)), rng.random() < 0.5,
                       rng.random() < 0.5)
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    head_dim = rng.choice((64, 128, 128))
    hkv = rng.choice((1, 2, 4, 8))
    heads = rng.choice(GEOMETRIES + ((hkv * rng.randint(1, 8), hkv),))
    B = _log_int(rng, 1, 48)
    lo = _log_int(rng, 1, 16000)
    hi = _log_int(rng, lo, 32000)
    chunk = rng.random() < 0.6
    n_lo = _log_int(rng, 1, 400) if chunk else 1
    n_hi = _log_int(rng, n_lo, 2000) if chunk else 1
    if op == "rope_append":
        return _rope("", rng.choice(("same", "same", "e4m3")), dtype, B, heads, lo, hi, n_lo, n_hi, head_dim,
                     rng.choice((16, head_dim // 2, head_dim)), rng.random() < 0.4, rng.random() < 0.7)
    return _rules("", dtype, B, heads, lo, hi, n_lo, n_hi, head_dim, rng.choice((0.0, 0.0, 20.0, 50.0)),
                  rng.choice((0, 0, _log_int(rng, 16, 8000))), rng.random() < 0.4,
                  rng.choice((0, 0, _log_int(rng, 1, 3000))), rng.choice((0, 0, _log_int(rng, 50, 4000))))


# ---- what a case moves and computes ---------------------------------------------------------------------------------

def _spread(lo, hi, count):
    if count == 1:
        return [hi]
    return [lo + round(i * (hi - lo) / (count - 1)) for i in range(count)]


def _lengths(case):
    """(tokens before the call, new tokens) of each sequence; the longest prefix meets the shortest step."""
    return _spread(case["lo"], case["hi"], case["batch"]), _spread(case["n_lo"], case["n_hi"], case["batch"])[::-1]


def _visible(case):
    """(keys that have to be read, query-key pairs) per KV head and per query head, over the batch."""
    keys = pairs = 0
    for before, n in zip(*_lengths(case)):
        L, first = before + n, before
        reach = L if not case["window"] else min(L, case["window"] + n - 1)
        if case["document"]:
            reach = min(reach, case["document"] + n - 1)
        keys += max(1, reach)
        row = lambda pos: min(pos + 1, case["window"] or pos + 1, (case["document"] + 1) // 2 if case["document"] else pos + 1)  # noqa: E731
        steps = 16
        pairs += n * sum(row(first + (2 * i + 1) * n // (2 * steps)) for i in range(steps)) / steps
        ahead = max(0, min(case["prefix"], L) - first)
        pairs += ahead * (ahead - 1) / 2
    return keys, pairs


def work(case):
    if case["op"] == "logits":
        S, V, elt = case["rows"], case["vocab"], 2 if case["dtype"] == "bf16" else 4
        per = elt + 4 + (4 if case["sampled"] else 0) + (0.125 if case["mask"] else 0)
        return {"bytes": S * V * per + 4 * S * case["history"] * case["penalties"], "flops": 8 * S * V}
    elt = 2 if case["dtype"] == "bf16" else 4
    new = sum(_lengths(case)[1])
    hq, hkv, D = case["hq"], case["hkv"], case["head_dim"]
    if case["op"] == "rope_append":
        kv_out = elt if case["kv"] == "same" else 1
        return {"bytes": new * D * ((hq + 2 * hkv) * elt + hq * elt + 2 * hkv * kv_out), "flops": new * (hq + hkv) * D * 8}
    keys, pairs = _visible(case)
    return {"bytes": 2 * keys * hkv * D * elt + 2 * new * hq * D * elt, "flops": 4 * pairs * hq * D}


def _cost(case):
    w = work(case)
    rate = 1.4e15 if case["dtype"] == "bf16" else 4e13
    return max(w["bytes"] / 6.5e12, w["flops"] / rate, 2e-6)


def _plain_bytes(case):
    if case["op"] != "attn_rules":
        return 0
    before, n = _lengths(case)
    L = max(b + k for b, k in zip(before, n))
    return 4 * case["batch"] * L * (case["hq"] * max(n) + 4 * case["hkv"] * case["head_dim"])


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=I32, device="cuda")


def _cache(case, rng, before, n):
    """A block table of shuffled pages (unused entries -1) and the number of pages of the pool."""
    need = [-(-(b + k) // PAGE) for b, k in zip(before, n)]
    order = list(range(sum(need)))
    rng.shuffle(order)
    width, rows, at = max(need), [], 0
    for c in need:
        rows.append(order[at:at + c] + [-1] * (width - c))
        at += c
    return _ints(rows), sum(need)


def prepare(case, seed):
    rng, g = random.Random(seed), _generator(seed)
    normal = lambda *shape, std=1.0, dtype=F32: (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    if case["op"] == "logits":
        return _prepare_logits(case, rng, g, normal)
    before, n = _lengths(case)
    both = list(zip(before, n))
    rng.shuffle(both)
    before, n = [b for b, _ in both], [k for _, k in both]
    table, pages = _cache(case, rng, before, n)
    B, hq, hkv, D, dtype = case["batch"], case["hq"], case["hkv"], case["head_dim"], DTYPES[case["dtype"]]
    T = sum(n)
    s = {"case": case, "block_table": table, "total": T, "new_lens": _ints(n)}
    if case["op"] == "rope_append":
        # a projection's output: the queries', keys' and values' rows of a token side by side
        s["qkv"] = normal(T, (hq + 2 * hkv) * D, dtype=dtype)
        s["seq_lens"] = _ints(before)
        s["inv_freq"] = 10000.0 ** (-torch.arange(case["rot"] // 2, device="cuda", dtype=F32) * 2 / case["rot"])
        s["q_weight"], s["k_weight"] = ((1 + normal(D, std=0.2), 1 + normal(D, std=0.2)) if case["norm"] else (None, None))
        pool = (pages, hkv, PAGE, D)
        if case["kv"] == "same":
            s["k_pages"], s["v_pages"] = normal(*pool, dtype=dtype), normal(*pool, dtype=dtype)
        else:
            s["k_pages"], s["v_pages"] = (torch.randint(0, 120, pool, generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        s["q_out"] = torch.empty(T, hq, D, dtype=dtype, device="cuda")
        return s
    s["q"] = normal(T, hq, D, std=4.0 if case["cap"] else 1.0, dtype=dtype)
    s["k_pages"], s["v_pages"] = normal(pages, hkv, PAGE, D, dtype=dtype), normal(pages, hkv, PAGE, D, dtype=dtype)
    s["seq_lens"], s["max_q"] = _ints([b + k for b, k in zip(before, n)]), max(n)
    s["slopes"] = 2.0 ** (-8.0 * (torch.arange(hq, device="cuda", dtype=F32) + 1) / hq) if case["slopes"] else None
    s["prefix_lens"] = _ints([rng.randint(0, case["prefix"]) for _ in range(B)]) if case["prefix"] else None
    s["first_keys"] = None
    if case["document"]:
        first = []
        for b, k in both:
            shift = rng.randrange(case["document"])
            first += [max(0, p - (p + shift) % case["document"]) for p in range(b, b + k)]
        s["first_keys"] = _ints(first)
    s["out"] = torch.empty_like(s["q"])
    return s


def _prepare_logits(case, rng, g, normal):
    S, V, H = case["rows"], case["vocab"], case["history"]
    s = {"case": case, "logits": normal(S, V, std=3.0, dtype=DTYPES[case["dtype"]])}
    uniform = lambda lo, hi: lo + (hi - lo) * torch.rand(S, generator=g, device="cuda")  # noqa: E731
    s["history"] = s["history_lens"] = s["repetition"] = s["presence"] = s["frequency"] = None
    if case["penalties"]:
        # a generated text repeats itself: most tokens come from a small part of the vocabulary
        few = torch.randint(0, max(1, V // 50), (S, H), generator=g, device="cuda", dtype=I32)
        any_ = torch.randint(0, V, (S, H), generator=g, device="cuda", dtype=I32)
        s["history"] = torch.where(torch.rand(S, H, generator=g, device="cuda") < 0.8, few, any_).contiguous()
        s["history_lens"] = _ints(_spread(max(1, H // 2), H, S))
        s["repetition"], s["presence"], s["frequency"] = uniform(1.0, 1.4), uniform(0.0, 0.6), uniform(0.0, 0.3)
    s["bias_offsets"] = s["bias_tokens"] = s["bias_values"] = None
    if case["biases"]:
        counts = [rng.randint(0, min(V, case["biases"])) for _ in range(S)]
        s["bias_offsets"] = _ints([sum(counts[:i]) for i in range(S + 1)])
        s["bias_tokens"] = _ints([t for c in counts for t in rng.sample(range(V), c)] or [0])
        s["bias_values"] = normal(len(s["bias_tokens"]), std=4.0)
    s["mask"] = None
    if case["mask"]:
        s["mask"] = torch.randint(-2 ** 31, 2 ** 31, (S, -(-V // 32)), generator=g, device="cuda", dtype=torch.int64).to(I32)
    s["temperature"] = uniform(0.3, 1.5) if case["sampled"] else None
    s["noise"] = None
    if case["sampled"]:
        s["noise"] = -torch.log(-torch.log(torch.rand(S, V, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)))
    s["out"] = torch.empty(S, V, dtype=F32, device="cuda")
    s["tokens"], s["logprobs"] = torch.empty(S, dtype=I32, device="cuda"), torch.empty(S, dtype=F32, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(state):
    return {"rope_append": _run_rope, "attn_rules": _run_rules, "logits": _run_logits}[state["case"]["op"]](state)


def _split_rows(s):
    c = s["case"]
    hq, hkv, D, T = c["hq"], c["hkv"], c["head_dim"], s["total"]
    q, k, v = s["qkv"].split((hq * D, hkv * D, hkv * D), dim=1)
    return q.view(T, hq, D), k.view(T, hkv, D), v.view(T, hkv, D)


def _scales(case):
    return 16.0, 20.0   # 1 / scale of keys and of values: N(0, 1) rows use the middle of the code range


def _places(s):
    """Sequence and position of every new token (rows packed by sequence)."""
    T, lens = s["total"], s["new_lens"].long()
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens, output_size=T)
    start = torch.cumsum(lens, 0) - lens
    return seq, torch.arange(T, device="cuda") - start[seq]


def _run_rope(s):
    c = s["case"]
    q, k, v = _split_rows(s)
    e4m3 = c["kv"] == "e4m3"
    ki, vi = _scales(c)
    if own:
        more = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], interleaved=c["interleaved"], q_out=s["q_out"], update_lens=False)
        where = (s["block_table"], s["seq_lens"], s["new_lens"], s["k_pages"], s["v_pages"])
        if e4m3:
            _context().rope_append_e4m3(q, k, v, s["inv_freq"], ki, vi, *where, **more)
        else:
            _context().rope_append(q, k, v, s["inv_freq"], *where, **more)
    else:
        seq, j = _places(s)
        pos = s["seq_lens"].long()[seq] + j
        angle = pos.double()[:, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

        def turned(x, w):
            x = x.float()
            if w is not None:
                x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
            r = c["rot"]
            a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
            y, z = a * cos - b * sin, a * sin + b * cos
            first = torch.stack((y, z), -1).flatten(-2) if c["interleaved"] else torch.cat((y, z), -1)
            return torch.cat((first, x[..., r:]), -1)

        s["q_out"].copy_(turned(q, s["q_weight"]))
        rows, values = turned(k, s["k_weight"]), v
        if e4m3:
            rows = (rows * ki).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
            values = (v.float() * vi).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        page = s["block_table"][seq, pos // PAGE].long()
        s["k_pages"][page, :, pos % PAGE] = rows.to(s["k_pages"].dtype)
        s["v_pages"][page, :, pos % PAGE] = values
    held = torch.float8_e4m3fn if e4m3 else s["k_pages"].dtype
    return {"q": s["q_out"], "k": s["k_pages"].view(held), "v": s["v_pages"].view(held)}


def _run_rules(s):
    c = s["case"]
    if own:
        return _context().attn_rules(s["q"], s["k_pages"], s["v_pages"], s["block_table"], s["seq_lens"], s["new_lens"], s["max_q"],
                                     cap=c["cap"], window=c["window"], slopes=s["slopes"], prefix_lens=s["prefix_lens"],
                                     first_keys=s["first_keys"], out=s["out"])
    B, hq, hkv, D, g = c["batch"], c["hq"], c["hkv"], c["head_dim"], c["hq"] // c["hkv"]
    n, width = s["max_q"], s["block_table"].shape[1] * PAGE
    seq, j = _places(s)
    pages = s["block_table"].clamp(min=0).long()
    keys = s["k_pages"][pages].permute(0, 2, 1, 3, 4).reshape(B, hkv, width, D).float()
    values = s["v_pages"][pages].permute(0, 2, 1, 3, 4).reshape(B, hkv, width, D).float()
    q = torch.zeros(B, n, hq, D, device="cuda")
    q[seq, j] = s["q"].float()
    q = q.view(B, n, hkv, g, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, g * n, D)
    x = torch.matmul(q, keys.transpose(2, 3)).mul_(D ** -0.5).view(B, hkv, g, n, width)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    pos = (s["seq_lens"] - s["new_lens"])[:, None] + torch.arange(n, device="cuda", dtype=I32)   # [B, n]
    key = torch.arange(width, device="cuda", dtype=I32)
    last, first = pos, torch.zeros_like(pos)
    if s["prefix_lens"] is not None:
        prefix = torch.minimum(s["prefix_lens"], s["seq_lens"])[:, None]
        last = torch.where(pos < prefix, torch.maximum(pos, prefix - 1), pos)
    if c["window"]:
        first = torch.maximum(first, pos - c["window"] + 1)
    if s["first_keys"] is not None:
        starts = torch.zeros_like(pos)
        starts[seq, j] = s["first_keys"]
        first = torch.maximum(first, starts)
    hidden = (key < first[..., None]) | (key > last[..., None])                                    # [B, n, width]
    if s["slopes"] is not None:
        distance = (pos[..., None] - key).abs().float()
        x -= s["slopes"].view(1, hkv, g, 1, 1) * distance[:, None, None]
    x.masked_fill_(hidden[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hkv, g * n, width), values).view(B, hkv, g, n, D) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, D)
    return o[seq, j].to(s["q"].dtype)


def _run_logits(s):
    if own:
        out, tokens, logprobs = _context().logits(
            s["logits"], history=s["history"], history_lens=s["history_lens"], repetition=s["repetition"], presence=s["presence"],
            frequency=s["frequency"], bias_offsets=s["bias_offsets"], bias_tokens=s["bias_tokens"], bias_values=s["bias_values"],
            mask=s["mask"], temperature=s["temperature"], noise=s["noise"], out=s["out"], tokens=s["tokens"], logprobs=s["logprobs"])
        return {"logits": out, "tokens": tokens, "logprobs": logprobs}
    x = s["logits"].float()
    S, V = x.shape
    if s["history"] is not None:
        there = torch.arange(s["history"].shape[1], device="cuda") < s["history_lens"][:, None]
        count = torch.zeros(S, V, device="cuda").scatter_add_(1, s["history"].long(), there.float())
        rep = s["repetition"][:, None]
        seen = torch.where(x > 0, x / rep, x * rep) - s["presence"][:, None] - s["frequency"][:, None] * count
        x = torch.where(count > 0, seen, x)
    if s["bias_offsets"] is not None:
        total = int(s["bias_tokens"].numel())
        row = torch.searchsorted(s["bias_offsets"][1:].contiguous(), torch.arange(total, device="cuda", dtype=I32), right=True)
        bias = torch.zeros(S + 1, V, device="cuda")
        bias[row, s["bias_tokens"].long()] = s["bias_values"]
        x = x + bias[:S]
    if s["temperature"] is not None:
        x = x / s["temperature"][:, None]
    if s["mask"] is not None:
        bit = torch.arange(V, device="cuda")
        allowed = (s["mask"][:, bit // 32] >> (bit % 32).to(I32)) & 1
        x = torch.where(allowed != 0, x, -math.inf)
    y = x if s["noise"] is None else x + s["noise"]
    best = y.amax(-1, keepdim=True)
    tokens = torch.where(y == best, torch.arange(V, device="cuda"), V).amin(-1)
    m = x.amax(-1, keepdim=True)
    logprobs = x.gather(1, tokens[:, None]) - m - (x - m).exp().sum(-1, keepdim=True).log()
    return {"logits": x, "tokens": tokens.to(I32), "logprobs": logprobs[:, 0]}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope_append": _exact_rope, "attn_rules": _exact_rules, "logits": _exact_logits}[case["op"]](s)


def _exact_rope(s):
    c = s["case"]
    q, k, v = (x.double() for x in _split_rows(s))
    e4m3 = c["kv"] == "e4m3"
    if c["norm"]:
        q = q / (q.pow(2).sum(-1, keepdim=True) / q.shape[-1] + 1e-6).sqrt() * s["q_weight"].double()
        k = k / (k.pow(2).sum(-1, keepdim=True) / k.shape[-1] + 1e-6).sqrt() * s["k_weight"].double()
    lens, at = s["new_lens"].tolist(), 0
    pools = [p.view(torch.float8_e4m3fn).double() if e4m3 else p.double() for p in (s["k_pages"], s["v_pages"])]
    ki, vi = _scales(c) if e4m3 else (1.0, 1.0)
    r, outs = c["rot"], []
    for b, n in enumerate(lens):
        pos = int(s["seq_lens"][b]) + torch.arange(n, device="cuda")
        turn = torch.polar(torch.ones(n, r // 2, dtype=torch.float64, device="cuda"), pos.double()[:, None] * s["inv_freq"].double())[:, None]

        def turned(x):
            pair = x[..., :r].unflatten(-1, (r // 2, 2)) if c["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            z = z if c["interleaved"] else z.transpose(-1, -2)
            return torch.cat((z.flatten(-2), x[..., r:]), -1)

        rows = slice(at, at + n)
        outs.append(turned(q[rows]))
        page = s["block_table"][b].long()[pos // PAGE]
        for pool, row, scale in ((pools[0], turned(k[rows]), ki), (pools[1], v[rows], vi)):
            row = row * scale
            pool[page, :, pos % PAGE] = row.clamp(-E4M3_MAX, E4M3_MAX) if e4m3 else row
        at += n
    return {"q": torch.cat(outs), "k": pools[0], "v": pools[1]}


def _exact_rules(s):
    c = s["case"]
    D, g, outs, at = c["head_dim"], c["hq"] // c["hkv"], [], 0
    slopes = None if s["slopes"] is None else s["slopes"].double()
    for b, n in enumerate(s["new_lens"].tolist()):
        L = int(s["seq_lens"][b])
        page = s["block_table"][b, :-(-L // PAGE)].long()
        k, v = (p[page].transpose(0, 1).flatten(1, 2)[:, :L].double().repeat_interleave(g, 0) for p in (s["k_pages"], s["v_pages"]))
        pos, key = torch.arange(L - n, L, device="cuda"), torch.arange(L, device="cuda")
        sees = key <= pos[:, None]
        if s["prefix_lens"] is not None:
            P = int(s["prefix_lens"][b])
            sees |= (pos[:, None] < P) & (key < P)
        if c["window"]:
            sees &= key > pos[:, None] - c["window"]
        if s["first_keys"] is not None:
            sees &= key >= s["first_keys"][at:at + n, None]
        rows = []
        for h in range(c["hq"]):   # one head at a time: the scores of a long prompt in 64 bits
            x = s["q"][at:at + n, h].double() @ k[h].T / math.sqrt(D)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if slopes is not None:
                x = x - slopes[h] * (pos[:, None] - key).abs()
            x = torch.where(sees, x, -math.inf)
            p = torch.exp(x - x.amax(-1, keepdim=True)).nan_to_num(0.0)
            rows.append((p @ v[h]) / p.sum(-1, keepdim=True).clamp(min=1e-300))
        outs.append(torch.stack(rows, 1))
        at += n
    return torch.cat(outs)


def _exact_logits(s):
    x = s["logits"].double()
    S, V = x.shape
    for i in range(S):
        if s["history"] is not None:
            token, count = s["history"][i, :int(s["history_lens"][i])].long().unique(return_counts=True)
            old, rep = x[i, token], s["repetition"][i].double()
            x[i, token] = torch.where(old > 0, old / rep, old * rep) - s["presence"][i].double() - s["frequency"][i].double() * count
        if s["bias_offsets"] is not None:
            part = slice(int(s["bias_offsets"][i]), int(s["bias_offsets"][i + 1]))
            x[i].index_add_(0, s["bias_tokens"][part].long(), s["bias_values"][part].double())
        if s["temperature"] is not None:
            x[i] /= s["temperature"][i].double()
        if s["mask"] is not None:
            bits = ((s["mask"][i].long()[:, None] >> torch.arange(32, device="cuda")) & 1).flatten()[:V]
            x[i, bits == 0] = -math.inf
    y = x if s["noise"] is None else x + s["noise"].double()
    return {"logits": x, "tokens": None, "logprobs": torch.log_softmax(x, -1).gather(1, y.argmax(-1, keepdim=True))[:, 0]}
