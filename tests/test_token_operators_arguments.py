"""What arb_rope_append*, arb_attn_rules and arb_logits refuse before any launch, in the C ABI and in the Python binding.  No GPU is
needed: a call whose arguments are right ends at the check that its tensors lie on the device."""
import ctypes

import pytest
import torch

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
B, HQ, HKV, D, PAGES, P, V = 2, 4, 2, 128, 5, 16, 70
RIGHT = "CUDA tensor"


def _binding():
    from paper_2512_05033_b200 import build
    build.build()
    from paper_2512_05033_b200 import binding
    return binding


def _context():
    c = _binding().Context.__new__(_binding().Context)   # no arb_ctx: nothing gets as far as using one
    c._h = c._p = None
    return c


def _t(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def _calls():
    q, rows, freq = _t(3, HQ, D), _t(3, HKV, D), _t(D // 2, dtype=F32)
    pool, codes, half = _t(PAGES, HKV, P, D), _t(PAGES, HKV, P, D, dtype=U8), _t(PAGES, HKV, P, D // 2, dtype=U8)
    sc, table, lens = _t(PAGES, HKV, P, dtype=F32), _t(B, 3, dtype=I32), _t(B, dtype=I32)
    rope = dict(q=q, k_new=rows, v_new=rows, inv_freq=freq, block_table=table, seq_lens=lens, new_lens=lens)
    return {
        "rope_append": dict(rope, k_pages=pool, v_pages=pool),
        "rope_append_e4m3": dict(rope, k_inv_scale=1.0, v_inv_scale=1.0, k_codes=codes, v_codes=codes),
        "rope_append_i4": dict(rope, k_codes=half, v_codes=half, k_scales=sc, v_scales=sc),
        "attn_rules": dict(q=q, k_pages=pool, v_pages=pool, block_table=table, seq_lens=lens, q_lens=lens, max_q_len=2),
        "logits": dict(logits=_t(3, V)),
    }


BAD = [
    ("rope_append", "q", _t(HQ, D), "dimensions"), ("rope_append", "k_new", _t(2, HKV, D), "has to be"),
    ("rope_append", "v_new", _t(3, 1, D), "has to be"), ("rope_append", "v_new", _t(3, HKV, 64), "has to be"),
    ("rope_append", "inv_freq", _t(D, dtype=F32), "more than head_dim"), ("rope_append", "block_table", _t(B, dtype=I32), "dimensions"),
    ("rope_append", "k_pages", _t(PAGES, HKV + 1, P, D), "do not match"), ("rope_append", "v_pages", _t(PAGES - 1, HKV, P, D), "shape"),
    ("rope_append_i4", "k_codes", _t(PAGES, HKV, P, D, dtype=U8), "do not match"),
    ("rope_append_e4m3", "v_codes", _t(PAGES, HKV, P, D // 2, dtype=U8), "shape"),
    ("attn_rules", "q", _t(3, HQ * D), "dimensions"), ("attn_rules", "k_pages", _t(PAGES, HKV, P, 64), "shape|different head"),
    ("attn_rules", "v_pages", _t(PAGES, 1, P, D), "shape"),
    ("logits", "logits", _t(V), "dimensions"),
]


@pytest.mark.parametrize("name", list(_calls()))
def test_right_arguments_end_at_the_device_check(name):
    with pytest.raises(ValueError, match=RIGHT):
        getattr(_context(), name)(**_calls()[name])


@pytest.mark.parametrize("name,arg,value,message", BAD)
def test_wrong_shapes_are_refused(name, arg, value, message):
    with pytest.raises(ValueError, match=message):
        getattr(_context(), name)(**{**_calls()[name], arg: value})


# ---- the C ABI: a block of memory stands in for the context, pointers are numbers that are never followed

PTR = 1 << 20


def _ctx_memory():
    return (ctypes.c_char * (1 << 16))()


def _attn_params(binding, **more):
    p = binding.attn_params(binding.ARB_BF16, B, HQ, HKV, D, PAGES, 3, 3, 2)
    for k, v in more.items():
        setattr(p, k, v)
    return p


def _rope(form, total=3, rope=None, params=None, null=None, off=None, scales=(1.0, 1.0), **fields):
    b = _binding()
    r = b.RopeParams(rot_dim=D, eps=1e-6, inv_freq=PTR, **(rope or {}))
    p = _attn_params(b, **(params or {}))
    names = ["q", "k_new", "v_new"] + (["ki", "vi"] if form == 1 else []) + ["block_table", "seq_lens", "new_lens", "update", "q_out", "k", "v"]
    names += ["k_scales", "v_scales"] if form == 2 else []
    args = []
    for n in names:
        args.append(scales[n == "vi"] if n in ("ki", "vi") else 1 if n == "update" else None if n == null else PTR + (8 if n == off else 0))
    call = (b.lib.arb_rope_append, b.lib.arb_rope_append_e4m3, b.lib.arb_rope_append_i4)[form]
    return call(ctypes.addressof(_ctx_memory()), ctypes.byref(p), ctypes.byref(r), total, *args, None)


INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("form", [0, 1, 2])
def test_rope_append_refusals(form):
    for n in ("q", "k_new", "v_new", "block_table", "seq_lens", "new_lens", "q_out", "k", "v") + (("k_scales", "v_scales") if form == 2 else ()):
        assert _rope(form, null=n) == INVALID, n
    for n in ("q", "k_new", "v_new", "q_out", "k", "v"):
        assert _rope(form, off=n) == INVALID, n
    assert _rope(form, total=-1) == INVALID
    for rope in ({"eps": -1.0}, {"eps": float("nan")}, {"reserved": 1}, {"rot_dim": -16}, {"inv_freq": None}, {"inv_freq": PTR + 4},
                 {"q_weight": PTR + 8}, {"k_weight": PTR + 8}, {"q_stride": HQ * D - 8}, {"k_stride": 8}, {"v_stride": HKV * D + 4},
                 {"q_stride": -8}):
        b = _binding()
        r = {"rot_dim": D, "eps": 1e-6, "inv_freq": PTR, **rope}
        assert _rope_raw(b, form, r) == INVALID, rope
    for rope in ({"rot_dim": D + 16}, {"rot_dim": 8}, {"rot_dim": 100}):
        assert _rope_raw(_binding(), form, {"rot_dim": D, "eps": 1e-6, "inv_freq": PTR, **rope}) == UNSUPPORTED, rope
    for params in ({"dtype": 7}, {"head_dim": 96}, {"page_size": 32}, {"batch": 1025}, {"max_pages_per_seq": 1 << 27}):
        assert _rope(form, params=params) == UNSUPPORTED, params
    for params in ({"batch": 0}, {"num_q_heads": 0}, {"num_kv_heads": 0}, {"num_pages": 0}, {"max_pages_per_seq": 0}):
        assert _rope(form, params=params) == INVALID, params
    assert _rope(form, total=1 << 29) == UNSUPPORTED          # rows of all heads beyond 2^31 - 1
    assert _rope(form, total=0) == 0                          # nothing to do


def _rope_raw(b, form, fields):
    r = b.RopeParams(**fields)
    p = _attn_params(b)
    mem = _ctx_memory()
    head = [ctypes.addressof(mem), ctypes.byref(p), ctypes.byref(r), 3, PTR, PTR, PTR]
    tail = [PTR, PTR, PTR, 1, PTR, PTR, PTR]
    if form == 1:
        return b.lib.arb_rope_append_e4m3(*head, 1.0, 1.0, *tail, None)
    if form == 2:
        return b.lib.arb_rope_append_i4(*head, *tail, PTR, PTR, None)
    return b.lib.arb_rope_append(*head, *tail, None)


def test_rope_append_quantised_refusals():
    for scales in ((0.0, 1.0), (1.0, -1.0), (float("nan"), 1.0)):
        assert _rope(1, scales=scales) == INVALID
    assert _rope(2, params={"dtype": 0}) == UNSUPPORTED
    assert _rope(2, params={"head_dim": 64}) == UNSUPPORTED


def _rules(null=None, off=None, rules=None, params=None):
    b = _binding()
    r, p = b.ScoreRules(**(rules or {})), _attn_params(b, **(params or {}))
    mem = _ctx_memory()
    args = [None if n == null else PTR + (8 if n == off else 0) for n in ("q", "k", "v", "table", "seq_lens", "q_lens", "out")]
    return b.lib.arb_attn_rules(ctypes.addressof(mem), ctypes.byref(p), ctypes.byref(r), *args, None)


def test_attn_rules_refusals():
    for n in ("q", "k", "v", "table", "seq_lens", "q_lens", "out"):
        assert _rules(null=n) == INVALID, n
    for n in ("q", "k", "v", "out"):
        assert _rules(off=n) == INVALID, n
    for rules in ({"cap": -1.0}, {"cap": float("nan")}, {"cap": float("inf")}, {"window": -1}):
        assert _rules(rules=rules) == INVALID, rules
    for params in ({"flags": 1}, {"flags": 2}, {"head_dim": 96}, {"num_q_heads": 18}, {"dtype": 2}, {"page_size": 8}, {"batch": 1025}):
        assert _rules(params=params) == UNSUPPORTED, params
    for params in ({"num_q_heads": 5}, {"batch": 0}, {"max_q_len": 4}, {"total_q": -1}):
        assert _rules(params=params) == INVALID, params
    assert _rules(params={"total_q": 0, "max_q_len": 0}) == 0
    b = _binding()
    p = _attn_params(b)
    assert b.lib.arb_attn_rules(None, ctypes.byref(p), ctypes.byref(b.ScoreRules()), *[PTR] * 7, None) == INVALID
    assert b.lib.arb_attn_rules(ctypes.addressof(_ctx_memory()), ctypes.byref(p), None, *[PTR] * 7, None) == INVALID


def _logits(**fields):
    b = _binding()
    p = b.LogitsParams(**{**dict(dtype=1, rows=3, vocab=V, logits=PTR, out=PTR + 4096), **fields})
    return b.lib.arb_logits(ctypes.addressof(_ctx_memory()), ctypes.byref(p), None)


def test_logits_refusals():
    for f in ({"rows": -1}, {"vocab": 0}, {"logits": None}, {"logits": PTR + 1}, {"out": PTR + 2}, {"noise": PTR + 1}, {"out": None}, {"logits": PTR, "out": PTR},
              {"logits_stride": V - 1}, {"history": PTR}, {"history_lens": PTR}, {"mask": PTR, "mask_stride": 2},
              {"bias_tokens": PTR}, {"bias_values": PTR}, {"bias_offsets": PTR, "bias_total": 3},
              {"bias_offsets": PTR, "bias_total": -1, "bias_tokens": PTR, "bias_values": PTR}):
        assert _logits(**f) == INVALID, f
    for f in ({"dtype": 3}, {"rows": 65536}, {"vocab": (1 << 24) + 1}):
        assert _logits(**f) == UNSUPPORTED, f
    assert _logits(rows=0) == 0
    b = _binding()
    assert b.lib.arb_logits(None, ctypes.byref(b.LogitsParams()), None) == INVALID


def test_the_records_match_the_header():
    b = _binding()
    assert ctypes.sizeof(b.RopeParams) == 72 and ctypes.sizeof(b.ScoreRules) == 32 and ctypes.sizeof(b.LogitsParams) == 152


def test_lists_beyond_32_bits_are_refused():
    """In the C ABI, whose kernels step through a list with 32-bit numbers, and in the binding, where a longer tensor's length would wrap."""
    long_list = {"bias_offsets": PTR, "bias_tokens": PTR, "bias_values": PTR}
    assert _logits(**long_list, bias_total=1 << 30) == UNSUPPORTED and _logits(**long_list, bias_total=2 ** 31 - 1) == UNSUPPORTED
    assert _logits(history=PTR, history_stride=1 << 24) == UNSUPPORTED
