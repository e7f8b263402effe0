"""The fusion scorer's operators without a GPU: the library exports what their header declares, bad
arguments are refused before any HIP call, the angle tables, and the 64-bit forms that the GPU tests use."""

import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2603_14002_amd as lbm
from paper_2603_14002_amd import scorer
from tests import scorer_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 4096  # an address that is never touched


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "lightbeam_scorer.h")).read()
    names = set(re.findall(r"^lb_status (lb_\w+)\s*\(", text, re.M))
    assert names == set(lbm.SCORER_EXPORTED)
    for n in names:
        assert hasattr(lbm.lib(), n) and hasattr(lbm, n)


def test_struct_sizes_match_header_layout():
    assert ctypes.sizeof(scorer.lb_kv_cache) == 40 and ctypes.sizeof(scorer.lb_kv_batch) == 40
    assert ctypes.sizeof(scorer.lb_rope) == 32 and ctypes.sizeof(scorer.lb_logit_rules) == 72


def cache(**over):
    d = dict(pages=AT, n_pages=8, page_tokens=16, kv_heads=2, head_dim=64, reserved=0, flags=None)
    d.update(over)
    return scorer.lb_kv_cache(**d)


def batch(**over):
    d = dict(starts=AT, lengths=AT, pages=AT, n_seqs=2, n_rows=3, max_pages=4, max_new=2)
    d.update(over)
    return scorer.lb_kv_batch(**d)


def rope(**over):
    d = dict(cos=AT, sin=AT, positions=64, rot_dim=64, layout=0, reserved=0)
    d.update(over)
    return scorer.lb_rope(**d)


def by(x):
    return None if x is None else ctypes.addressof(x)


def append(c=None, b=None, r=None, dtype=0, hq=4, q=AT, qs=256, k=AT, ks=128, v=AT, vs=128, o=2 * AT, os_=256):
    c, b = cache() if c is None else c, batch() if b is None else b
    return lbm.lib().lb_kv_append(by(c), by(b), by(r), dtype, hq, q, qs, k, ks, v, vs, o, os_, None)


def attend(c=None, b=None, dtype=0, hq=4, q=AT, qs=256, scale=1.0, window=0, o=2 * AT, os_=256, ws=AT, nb=1 << 40):
    c, b = cache() if c is None else c, batch() if b is None else b
    return lbm.lib().lb_kv_attend(by(c), by(b), dtype, hq, q, qs, scale, window, o, os_, None, ws, nb, None)


def refused(st):
    return st == lbm.LB_ERR_INVALID_ARG and lbm.lb_last_error() != ""


@pytest.mark.parametrize("over", [dict(head_dim=96), dict(head_dim=0), dict(kv_heads=0), dict(kv_heads=2000), dict(page_tokens=8),
                                  dict(page_tokens=48), dict(page_tokens=512), dict(pages=None), dict(pages=AT + 8), dict(n_pages=-1),
                                  dict(flags=AT + 2)])
def test_caches_that_are_refused(over):
    assert refused(append(cache(**over)))
    assert refused(attend(cache(**over)))
    assert refused(lbm.lib().lb_kv_read(by(cache(**over)), by(batch()), 0, AT, 8192, AT, 8192, None))
    n = ctypes.c_int64()
    assert refused(lbm.lib().lb_kv_attend_workspace(by(cache(**over)), by(batch()), 4, ctypes.addressof(n)))


@pytest.mark.parametrize("over", [dict(starts=None), dict(lengths=None), dict(pages=None), dict(n_seqs=-1), dict(n_rows=-1),
                                  dict(max_pages=0), dict(max_pages=1 << 27), dict(max_new=0), dict(n_rows=(1 << 28) + 1),
                                  dict(n_seqs=(1 << 24) + 1), dict(n_rows=(1 << 24) + 1), dict(n_seqs=(1 << 22) + 1)])
def test_batches_that_are_refused(over):
    assert refused(append(b=batch(**over)))
    assert refused(attend(b=batch(**over)))


@pytest.mark.parametrize("over", [dict(dtype=3), dict(dtype=-1), dict(hq=-1), dict(q=None), dict(k=None), dict(v=None), dict(o=None),
                                  dict(qs=255), dict(ks=127), dict(vs=129), dict(os_=258), dict(q=AT + 4), dict(k=AT + 8),
                                  dict(o=AT, os_=512), dict(dtype=1, ks=132), dict(r=rope(rot_dim=8)), dict(r=rope(rot_dim=24)),
                                  dict(r=rope(rot_dim=80)), dict(r=rope(layout=2)), dict(r=rope(cos=None)), dict(r=rope(sin=AT + 4)),
                                  dict(r=rope(positions=0)), dict(r=rope(rot_dim=-16))])
def test_appends_that_are_refused(over):
    assert refused(append(**over))


@pytest.mark.parametrize("over", [dict(dtype=5), dict(hq=0), dict(hq=3), dict(q=None), dict(o=None), dict(qs=200), dict(os_=257),
                                  dict(o=AT + 2), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(scale=3e38),
                                  dict(c=cache(kv_heads=1024), hq=1024, qs=65536, os_=65536, b=batch(n_seqs=1 << 20, n_rows=1 << 20)),
                                  dict(c=cache(page_tokens=256), b=batch(max_pages=4096), ws=None),
                                  dict(c=cache(page_tokens=256), b=batch(max_pages=4096), nb=64),
                                  dict(c=cache(page_tokens=256), b=batch(max_pages=4096), ws=AT + 4)])
def test_attends_that_are_refused(over):
    assert refused(attend(**over))


def test_empty_batches_are_nothing_to_do():
    L = lbm.lib()
    for b in (batch(n_seqs=0), batch(n_rows=0), batch(n_seqs=0, n_rows=0, starts=None, lengths=None, pages=None, max_pages=0, max_new=0)):
        assert append(b=b, q=None, k=None, v=None, o=None) == lbm.LB_OK
        assert attend(b=b, q=None, o=None, ws=None, nb=0) == lbm.LB_OK
        assert L.lb_kv_read(by(cache()), by(b), 0, None, 0, None, 0, None) == lbm.LB_OK
        n = ctypes.c_int64(5)
        assert L.lb_kv_attend_workspace(by(cache()), by(b), 4, ctypes.addressof(n)) == lbm.LB_OK and n.value == 0
    assert L.lb_lora_add(0, 0, 8, 8, 8, 0, None, 8, None, 8, None, None, None, None, None, 8, None, 0, None) == lbm.LB_OK
    assert L.lb_logits_adjust(0, 0, 5, None, 5, None, None, None, 5, None, None, None, 0, None) == lbm.LB_OK
    assert refused(L.lb_kv_append(None, by(batch()), None, 0, 0, None, 0, AT, 128, AT, 128, None, 0, None))
    assert refused(L.lb_kv_attend(by(cache()), None, 0, 4, AT, 256, 1.0, 0, AT, 256, None, None, 0, None))


@pytest.mark.parametrize("at,value", [(0, 4), (1, -1), (1, 1 << 29), (2, 12), (2, 0), (3, 4), (4, 12), (4, 136), (4, 0), (5, -1), (6, None),
                                      (6, AT + 4), (7, 63), (7, 65), (8, None), (9, 8), (10, None), (11, AT + 8), (12, None),
                                      (14, None), (15, 60), (16, None), (16, AT + 8), (17, 100)])
def test_lora_that_is_refused(at, value):
    a = [0, 300, 64, 64, 16, 2, AT, 64, AT, 64, AT, AT, AT, None, 2 * AT, 64, AT, 1 << 20, None]
    a[at] = value
    assert refused(lbm.lib().lb_lora_add(*a))


def test_lora_in_place_needs_the_same_stride():
    assert refused(lbm.lib().lb_lora_add(0, 4, 64, 64, 16, 2, AT, 64, AT, 64, AT, AT, AT, None, AT, 72, AT, 1 << 20, None))
    n = ctypes.c_int64()
    for bad in ((-1, 64, 64, 16), (4, 63, 64, 16), (4, 64, 0, 16), (4, 64, 64, 200)):
        assert refused(lbm.lib().lb_lora_workspace(*bad, ctypes.addressof(n)))
    assert refused(lbm.lib().lb_lora_workspace(4, 64, 64, 16, None))
    for rows, d_out, rank, some in ((4, 64, 16, False), (300, 64, 16, True), (4, 2048, 16, True), (4, 64, 64, True)):
        assert lbm.lib().lb_lora_workspace(rows, 64, d_out, rank, ctypes.addressof(n)) == lbm.LB_OK and (n.value > 0) == some


def rules(**over):
    d = dict(temperature=1.0, repetition=1.0, presence=0.0, frequency=0.0, history=None, bias_ids=None, bias_values=None, mask=None,
             mask_row=None, history_width=0, bias_width=0, bias_per_row=0, mask_rows=0)
    d.update(over)
    return scorer.lb_logit_rules(**d)


@pytest.mark.parametrize("over", [dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(repetition=0.0),
                                  dict(repetition=math.inf), dict(temperature=1e-39), dict(repetition=1e-40), dict(presence=math.nan), dict(frequency=math.inf),
                                  dict(history=AT, history_width=-1), dict(history=AT, history_width=4097),
                                  dict(bias_ids=AT, bias_width=4), dict(bias_ids=AT, bias_values=AT, bias_width=2049, history=AT, history_width=2048),
                                  dict(mask=AT), dict(mask=AT, mask_rows=2)])
def test_rules_that_are_refused(over):
    r = rules(**over)
    assert refused(lbm.lib().lb_logits_adjust(0, 3, 50, AT, 50, by(r), None, 2 * AT, 50, None, None, None, 0, None))


@pytest.mark.parametrize("at,value", [(0, 7), (1, -1), (2, 0), (3, None), (3, AT + 2), (4, 49), (8, 40), (9, AT), (7, AT)])
def test_logits_that_are_refused(at, value):
    a = [0, 3, 50, AT, 50, None, None, 2 * AT, 50, None, None, None, 0, None]
    a[at] = value
    if at == 7:
        a[8] = 64  # over the logits with another stride
    assert refused(lbm.lib().lb_logits_adjust(*a))


def test_logits_workspace_is_checked():
    a = [0, 1, 100000, AT, 100000, None, None, None, 0, None, AT, None, 0, None]
    assert refused(lbm.lib().lb_logits_adjust(*a))
    n = ctypes.c_int64()
    assert lbm.lib().lb_logits_workspace(1, 100000, ctypes.addressof(n)) == lbm.LB_OK and n.value > 0
    assert refused(lbm.lib().lb_logits_workspace(1, 0, ctypes.addressof(n)))


def test_binding_refuses_tensors_that_do_not_fit():
    """Types, shapes, layouts and devices that the C side cannot see."""
    pages = torch.zeros(3, 2, 16 * 68, dtype=torch.uint8)
    with pytest.raises(lbm.LBError):
        lbm.KVCache(pages, 32, 2, 64)
    with pytest.raises(lbm.LBError):
        lbm.KVCache(pages.to(torch.int8), 16, 2, 64)
    c = lbm.KVCache(pages, 16, 2, 64)
    i32 = dict(dtype=torch.int32)
    with pytest.raises(lbm.LBError):
        lbm.KVBatch(torch.zeros(2, **i32), torch.zeros(2, **i32), torch.zeros(2, 4, **i32), 2, 1)
    with pytest.raises(lbm.LBError):
        lbm.KVBatch(torch.zeros(3, dtype=torch.int64), torch.zeros(2, **i32), torch.zeros(2, 4, **i32), 2, 1)
    b = lbm.KVBatch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 4, **i32), 2, 1)
    k = torch.zeros(2, 2, 64)
    for q, kk, v in ((None, k, k[:, :1]), (None, k.double(), k.double()), (k[:, :, :32], k, k), (k.half(), k, k),
                     (None, k.transpose(0, 1), k), (None, k, torch.zeros(2, 2, 128)[:, :, ::2]), (None, k, k)):
        with pytest.raises(lbm.LBError):  # the last one: not on a GPU
            lbm.lb_kv_append(c, b, q, kk, v)
    with pytest.raises(lbm.LBError):
        lbm.lb_kv_attend(c, b, k, 1.0, lse=torch.zeros(2, 3))
    with pytest.raises(lbm.LBError):
        lbm.lb_kv_read(c, b, torch.float64)
    with pytest.raises(lbm.LBError):
        lbm.Rope(torch.zeros(4, 8), torch.zeros(4, 16))
    y, x, a, bb = torch.zeros(4, 16), torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(2, 16, 8)
    ids = torch.zeros(4, **i32)
    for args in ((y, x, a, bb.half(), ids), (y, x[:3], a, bb, ids), (y, x, a, bb[:, :8], ids), (y, x, a, bb, ids.long()),
                 (y, x, a, bb, ids, torch.zeros(3)), (y, x, a, bb, ids)):
        with pytest.raises(lbm.LBError):
            lbm.lb_lora_add(*args)
    z = torch.zeros(4, 50)
    for kw in (dict(rules=lbm.LogitRules(history=torch.zeros(3, 2, **i32))), dict(rules=lbm.LogitRules(mask=torch.zeros(1, 1, **i32))),
               dict(target=torch.zeros(3, **i32)), dict(logprobs=torch.zeros(4, 50).half()), dict()):
        with pytest.raises(lbm.LBError):
            lbm.lb_logits_adjust(z, **kw)
    for kw in (dict(bias_ids=torch.zeros(1, 2, **i32)), dict(mask_row=torch.zeros(1, **i32)), dict(history=torch.zeros(4, **i32))):
        with pytest.raises(lbm.LBError):
            lbm.LogitRules(**kw)


@pytest.mark.parametrize("scaling,kw", [(lbm.LB_ROPE_PLAIN, {}), (lbm.LB_ROPE_LINEAR, dict(factor=4.0)),
                                        (lbm.LB_ROPE_BLEND, dict(factor=8.0, trained=8192.0, low=1.0, high=4.0))])
def test_rope_table(scaling, kw):
    n, rot, base = 131072, 32, 500000.0
    cos, sin = lbm.lb_rope_table(n, rot, base, scaling, **kw)
    f = base ** (-2 * np.arange(rot // 2, dtype=np.float64) / rot)
    if scaling == lbm.LB_ROPE_LINEAR:
        f = f / 4
    if scaling == lbm.LB_ROPE_BLEND:
        wavelength = 2 * math.pi / f
        w = np.clip((8192.0 / wavelength - 1.0) / 3.0, 0, 1)
        f = w * f + (1 - w) * f / 8
        assert (w == 0).any() and (w == 1).any() and ((w > 0) & (w < 1)).any()
    p = np.array([0, 1, 2, 777, 65537, n - 1], dtype=np.float64)
    a = p[:, None] * f
    # one rounding to 32 bits, and the angle's own to 64 (at most 2^-53 of 131071)
    tol = 2.0 ** -25 + 2.0 ** -53 * n * 2
    assert np.abs(cos.numpy()[p.astype(int)] - np.cos(a)).max() < tol
    assert np.abs(sin.numpy()[p.astype(int)] - np.sin(a)).max() < tol


@pytest.mark.parametrize("args", [(0, 32), (4, 31), (4, 0), (4, 32, 0.0), (4, 32, math.inf), (4, 32, 1e4, 3), (4, 32, 1e4, 1, 0.0),
                                  (4, 32, 1e4, 2, 2.0, 0.0), (4, 32, 1e4, 2, 2.0, 100.0, 4.0, 1.0)])
def test_rope_tables_that_are_refused(args):
    with pytest.raises(lbm.LBError):
        lbm.lb_rope_table(*args)


def test_reference_blocks_by_hand():
    """The rounding of a block on worked values: scale 1 (largest 5 or 6), ties to the even code, clipping."""
    x = torch.zeros(32, dtype=torch.float64)
    x[:10] = torch.tensor([6.0, -0.25, 0.26, 0.75, 1.25, 1.26, 2.5, -3.5, 5.0, 5.01])
    code, scale = ref.encode(x)
    assert scale.tolist() == [127]
    assert ref.decode(code, scale)[:10].tolist() == [6.0, 0.0, 0.5, 1.0, 1.0, 1.5, 2.0, -4.0, 4.0, 6.0]
    assert ref.encode(x * 2 ** 0.001)[1].tolist() == [128]  # 6.004 needs the next scale
    assert ref.encode(x * 0)[1].tolist() == [3]
    assert ref.encode(x + math.inf)[1].tolist() == [255]


def test_reference_attention_by_hand():
    """Two tokens of scores 0 and ln 3: weights 1/4 and 3/4."""
    k = torch.zeros(2, 1, 32, dtype=torch.float64)
    k[1, 0, 0] = math.log(3)
    v = torch.zeros(2, 1, 32, dtype=torch.float64)
    v[0, 0, 1], v[1, 0, 1] = 4.0, 8.0
    q = torch.zeros(1, 1, 32, dtype=torch.float64)
    q[0, 0, 0] = 1.0
    out, lse, _, _ = ref.attend(q, k, v, 1.0, 1, 0)
    assert abs(float(out[0, 0, 1]) - 7.0) < 1e-12 and abs(float(lse[0, 0]) - math.log(4)) < 1e-12
    assert abs(float(ref.attend(q, k, v, 1.0, 1, 1)[0][0, 0, 1]) - 8.0) < 1e-12


def test_attend_workspace_refuses_what_attend_refuses():
    """Batches of more work than a call takes, and those that the header says are taken."""
    n = ctypes.c_int64()

    def workspace(**over):
        c, b = cache(kv_heads=over.pop("kv_heads")), batch(**over)
        return lbm.lib().lb_kv_attend_workspace(by(c), by(b), c.kv_heads, ctypes.addressof(n))

    big = dict(kv_heads=1024, n_seqs=1 << 20, n_rows=1 << 20)
    b = dict(big)
    assert refused(attend(c=cache(kv_heads=b.pop("kv_heads")), hq=1024, qs=65536, os_=65536, b=batch(**b)))
    assert refused(workspace(**big))
    # kv_heads * (n_seqs + n_rows / 16) below 2^24, with any max_new
    for heads, seqs, rows, new in ((8, 8192, 8192, 8192), (3, 20000, 25000, 5000), (1, 60000, 70000, 10000), (1, 1 << 22, 1 << 24, 1 << 24),
                                   (15, 1 << 20, 1 << 20, 1), (15, 1 << 20, 1 << 20, 1 << 20)):
        assert heads * (seqs + rows / 16) < 1 << 24
        assert workspace(kv_heads=heads, n_seqs=seqs, n_rows=rows, max_new=new) == lbm.LB_OK


@pytest.mark.parametrize("d_in,d_out", [((1 << 30) + 8, 64), (64, (1 << 30) + 8), (2 ** 31 - 8, 64), (64, 2 ** 31 - 8)])
def test_lora_widths_past_what_kernels_count(d_in, d_out):
    a = [1, 1, d_in, d_out, 8, 2, AT, d_in, AT, d_out, AT, AT, AT, None, 2 * AT, d_out, AT, 1 << 20, None]
    assert refused(lbm.lib().lb_lora_add(*a))
    n = ctypes.c_int64()
    assert refused(lbm.lib().lb_lora_workspace(1, d_in, d_out, 8, ctypes.addressof(n)))
    assert lbm.lib().lb_lora_workspace(1, 1 << 30, 1 << 30, 8, ctypes.addressof(n)) == lbm.LB_OK


def test_lora_over_its_own_input_needs_a_workspace():
    """A call of one launch would write rows of x that its other workgroups still read."""
    L = lbm.lib()
    n = ctypes.c_int64()
    assert L.lb_lora_workspace(4, 512, 512, 16, ctypes.addressof(n)) == lbm.LB_OK and n.value == 0
    for x, xs, out, os_ in ((AT, 512, AT, 512), (AT, 512, AT + 64, 512), (AT + 512 * 4 * 3, 512, AT, 512), (AT, 2048, AT + 511 * 4 + 4 - 16, 2048),
                            (AT + 1600 * 4, 2048, AT, 2048), (AT, 1024, AT + 600 * 4, 1032)):
        for nb in (0, 4 * 16 * 4 - 1):
            assert refused(L.lb_lora_add(0, 4, 512, 512, 16, 2, x, xs, out, os_, AT, AT, AT, None, out, os_, AT if nb else None, nb, None))


def test_attend_takes_the_workspace_that_the_library_says(monkeypatch):
    """Whatever the table's width: the rule for parts of the keys is the library's alone."""
    asked, got = [], []

    def workspace(c, b, heads):
        asked.append((b.max_pages, heads))
        return 1024 * b.max_pages + heads

    monkeypatch.setattr(scorer, "lb_kv_attend_workspace", workspace)
    monkeypatch.setattr(scorer, "_call", lambda g, stream, name, *a: got.append(a[-1]))
    monkeypatch.setattr(scorer, "_attend_bytes", {})
    c = lbm.KVCache(torch.zeros(3, 2, 16 * 68, dtype=torch.uint8), 16, 2, 64)
    i32 = dict(dtype=torch.int32)
    for width, heads in ((4, 2), (1, 4), (70, 2), (4, 4)):
        for _ in range(2):  # asked once for each size
            b = lbm.KVBatch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, width, **i32), 2, 1)
            lbm.lb_kv_attend(c, b, torch.zeros(2, heads, 64), 1.0)
            assert got.pop() == 1024 * width + heads
    assert len(asked) == len(set(asked)) == 4


def small():
    """A call of every function of the binding: its tensors by name, which of them it writes to, and the call."""
    i32 = dict(dtype=torch.int32)
    c = lbm.KVCache(torch.zeros(3, 2, 16 * 68, dtype=torch.uint8), 16, 2, 64)
    b = lbm.KVBatch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 4, **i32), 2, 1)
    z = lambda *shape: torch.zeros(*shape)
    return [
        (dict(q=z(2, 4, 64), k=z(2, 2, 64), v=z(2, 2, 64), q_out=z(2, 4, 64), cos=z(9, 32), sin=z(9, 32)), ["q_out"], [c.pages],
         lambda q, k, v, q_out, cos, sin: lbm.lb_kv_append(c, b, q, k, v, rope=lbm.Rope(cos, sin), q_out=q_out)),
        (dict(k_out=z(2, 2, 64), v_out=z(2, 2, 64)), ["k_out", "v_out"], [], lambda **t: lbm.lb_kv_read(c, b, **t)),
        (dict(q=z(2, 4, 64), out=z(2, 4, 64), lse=z(2, 4)), ["out", "lse"], [], lambda q, out, lse: lbm.lb_kv_attend(c, b, q, 1.0, out=out, lse=lse)),
        (dict(y=z(4, 16), x=z(4, 8), a=z(2, 8, 8), b=z(2, 16, 8), scale=z(2), out=z(4, 16)), ["out"], [],
         lambda y, x, a, b, scale, out: lbm.lb_lora_add(y, x, a, b, z(4).int(), scale, out=out)),
        (dict(y=z(4, 16), x=z(4, 8), a=z(2, 8, 8), b=z(2, 16, 8)), ["y"], [], lambda y, x, a, b: lbm.lb_lora_add(y, x, a, b, z(4).int())),
        (dict(logits=z(4, 50), logprobs=z(4, 50), bias_values=z(1, 3)), ["logprobs"], [],
         lambda logits, logprobs, bias_values: lbm.lb_logits_adjust(
             logits, lbm.LogitRules(bias_ids=torch.zeros(1, 3, **i32), bias_values=bias_values), logprobs=logprobs)),
    ]


def test_binding_refuses_tensors_that_require_gradients(monkeypatch):
    monkeypatch.setattr(scorer, "_call", lambda *a: None)
    for tensors, _, _, call in small():
        call(**tensors)
        for name in tensors:
            tensors[name].requires_grad_(True)
            with pytest.raises(lbm.LBError, match=f"^LB_ERR_INVALID_ARG: {name} requires a gradient"):
                call(**tensors)
            with torch.no_grad():
                call(**tensors)
            tensors[name].requires_grad_(False)


def test_binding_counts_what_it_writes_as_changed(monkeypatch):
    """Torch's autograd refuses a backward pass over a saved tensor that was written since."""
    monkeypatch.setattr(scorer, "_call", lambda *a: None)
    for tensors, out, more, call in small():
        before = {n: t._version for n, t in tensors.items()}
        pages = [t._version for t in more]
        call(**tensors)
        for n, t in tensors.items():
            assert (t._version > before[n]) == (n in out)
        assert all(t._version > v for t, v in zip(more, pages))
        with torch.inference_mode():
            call(**{n: torch.zeros_like(t) for n, t in tensors.items()})
    y, w = torch.ones(4, 16), torch.ones(4, 16, requires_grad=True)
    loss = (y * w).sum()
    lbm.lb_lora_add(y, torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(2, 16, 8), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_binding_refuses_numbers_past_32_bits(monkeypatch):
    """ctypes would take them modulo 2^32.  Tensors of such sizes are on the meta device, without memory."""
    monkeypatch.setattr(scorer, "_call", lambda *a: None)
    big, i32 = 2 ** 32, dict(dtype=torch.int32)
    c = lbm.KVCache(torch.zeros(3, 2, 16 * 68, dtype=torch.uint8), 16, 2, 64)
    tables = torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 4, **i32)
    b = lbm.KVBatch(*tables, 2, 1)
    meta = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")
    calls = [lambda: lbm.KVBatch(*tables, 2, big + 1), lambda: lbm.KVBatch(*tables, big + 2, 1), lambda: lbm.KVBatch(*tables, 2, -1),
             lambda: lbm.KVBatch(meta(big + 3, **i32), meta(big + 2, **i32), meta(big + 2, 4, **i32), 2, 1),
             lambda: lbm.KVBatch(tables[0], tables[1], meta(2, big + 4, **i32), 2, 1),
             lambda: lbm.KVCache(meta(3, 2, (big + 16) * 68, dtype=torch.uint8), big + 16, 2, 64),
             lambda: lbm.KVCache(meta(1, big + 2, 16 * 68, dtype=torch.uint8), 16, big + 2, 64),
             lambda: lbm.Rope(meta(big + 8, 8), meta(big + 8, 8)), lambda: lbm.Rope(torch.zeros(4, 8), torch.zeros(4, 8), big),
             lambda: lbm.LogitRules(history=meta(1, big + 2, **i32)), lambda: lbm.LogitRules(mask=meta(big + 1, 2, **i32)),
             lambda: lbm.LogitRules(bias_ids=meta(1, big + 2, **i32), bias_values=meta(1, big + 2)),
             lambda: lbm.lb_rope_table(big + 4, 16), lambda: lbm.lb_rope_table(4, big + 16), lambda: lbm.lb_rope_table(4, 16, 1e4, big),
             lambda: lbm.lb_kv_attend_workspace(c, b, big + 2), lambda: lbm.lb_kv_attend(c, b, torch.zeros(2, 2, 64), 1.0, window=big),
             lambda: lbm.lb_kv_attend(c, b, torch.zeros(2, 2, 64), 1.0, window=big + 5),
             lambda: lbm.lb_lora_workspace(4, big + 8, 8, 8), lambda: lbm.lb_lora_workspace(4, 8, big + 8, 8), lambda: lbm.lb_lora_workspace(4, 8, 8, big + 8),
             lambda: lbm.lb_lora_add(meta(1, 8), meta(1, big + 8), meta(1, 8, big + 8), meta(1, 8, 8), meta(1, **i32)),
             lambda: lbm.lb_lora_add(meta(1, big + 8), meta(1, 8), meta(1, 8, 8), meta(1, big + 8, 8), meta(1, **i32)),
             lambda: lbm.lb_logits_workspace(1, big + 41), lambda: lbm.lb_logits_adjust(meta(1, big + 41), target=meta(1, **i32))]
    for k, call in enumerate(calls):
        with pytest.raises(lbm.LBError, match=r"must be in 0\.\.2\^31 - 1"):
            call()
            print("not refused:", k)
