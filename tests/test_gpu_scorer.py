"""The fusion scorer's operators on the GPU against plain 64-bit forms (tests/scorer_ref.py)."""

import math

import numpy as np
import pytest
import torch

import paper_2603_14002_amd as lbm
from tests import scorer_ref as ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    lbm.lib()


def dev(t):
    return t.to("cuda:0")


def randn(rng, *shape, dtype=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape)).to(dtype)


def handles(R, flags=True):
    """The cache and batch of a Ragged on the GPU."""
    word = torch.zeros(1, dtype=torch.int32, device="cuda:0") if flags else None
    cache = lbm.KVCache(dev(R.pages), R.P, R.H, R.D, flags=word)
    return cache, lbm.KVBatch(dev(R.starts), dev(R.lengths), dev(R.table), R.n_rows, max([1] + R.new))


def close(got, want, bound, what):
    """|got - want| <= bound, and the same infinities and NaN."""
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    same_nan = torch.equal(torch.isnan(got), torch.isnan(want))
    assert same_nan, f"{what}: {int(torch.isnan(got).sum())} NaN, {int(torch.isnan(want).sum())} expected"
    inf = ~fine & ~torch.isnan(want)
    same_inf = torch.equal(got[inf], want[inf])
    assert same_inf, f"{what}: other infinities"
    d = (got - want).abs()[fine]
    b = bound.expand_as(want)[fine] if isinstance(bound, torch.Tensor) else torch.full_like(d, bound)
    within = bool((d <= b).all())
    assert within, f"{what}: off by {float(d.max())}, {float((d / b).nan_to_num(0).max())} of the bound, at {int((d > b).sum())} of {d.numel()}"


# ------------------------------------------------------------------ append and read


def angles(R, rot, seed=0, positions=None):
    n = positions or max([1] + R.length)
    cos, sin = lbm.lb_rope_table(n, rot, 10000.0)
    return cos, sin


APPEND = [  # new, length, page, q heads, kv heads, D, rot, interleaved, type, extra row stride, padding rows
    ([1], [1], 16, 4, 4, 64, 64, False, "f32", 0, 0),
    ([1, 1, 1], [5, 16, 17], 16, 4, 2, 64, 32, True, "bf16", 0, 2),
    ([3, 0, 1, 70], [3, 9, 40, 71], 16, 6, 2, 128, 128, False, "bf16", 64, 3),
    ([5, 33, 2], [130, 33, 64], 32, 8, 1, 128, 16, True, "f16", 0, 0),
    ([4, 8, 6], [4, 12, 9], 64, 7, 7, 256, 64, False, "f16", 8, 1),
    ([17], [4000], 128, 1, 1, 64, 48, False, "f32", 4, 0),
    ([9, 2], [11, 300], 256, 2, 2, 256, 0, False, "bf16", 0, 0),
    ([1] * 70 + [2], [3 * i + 2 for i in range(71)], 16, 2, 1, 64, 64, True, "f32", 0, 0),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_writes_the_rotated_blocks(case):
    """Codes and scales byte for byte as the 64-bit form has them, every other byte as it was, and the
    rotated queries to the rounding of their type."""
    new, length, P, Hq, H, D, rot, inter, t, extra, pad = APPEND[case]
    say(f"[case] append {case}")
    rng = np.random.default_rng(case)
    R = ref.Ragged(new, length, P, H, D, seed=case, pad_rows=pad)
    n, dt = R.n_rows, DT[t]
    width = (Hq + 2 * H) * D + extra
    packed = randn(rng, n, width, dtype=dt)
    packed[:, ::7] *= 40.0
    on = dev(packed)
    q, k, v = (on[:, a:b].unflatten(1, (-1, D)) for a, b in ((0, Hq * D), (Hq * D, (Hq + H) * D), ((Hq + H) * D, (Hq + 2 * H) * D)))
    cache, batch = handles(R)
    rope = cos = sin = None
    if rot:
        cos, sin = angles(R, rot)
        rope = lbm.Rope(dev(cos), dev(sin), lbm.LB_ROPE_INTERLEAVED if inter else lbm.LB_ROPE_HALF)
    q_out = torch.full((n, Hq, D), 7.0, dtype=dt, device="cuda:0")
    assert lbm.lb_kv_append(cache, batch, q, k, v, rope=rope, q_out=q_out) is q_out
    torch.cuda.synchronize()
    assert cache.status() == 0
    rows = R.rows()
    m = len(rows)
    pos = torch.tensor([p for _, p in rows])
    qh, kh, vh = (x.cpu()[:m].double() for x in (q, k, v))
    if rot:
        c, s = cos[pos], sin[pos]
        qw, kw = ref.rotate(qh, c, s, inter), ref.rotate(kh, c, s, inter)
        parts = ref.rotate(qh.abs(), c.abs(), -s.abs(), inter).abs() + ref.rotate(qh.abs(), c.abs(), s.abs(), inter).abs()
    else:
        qw, kw, parts = qh, kh, qh.abs()
    # two products and a sum in 32 bits, then the type's rounding
    close(q_out[:m], qw, ref.EPS[dt] * qw.abs() + 3 * 2.0 ** -24 * parts + 2.0 ** -25 * (dt == torch.float16), "q")
    assert bool((q_out[m:] == 7.0).all())
    want = ref.Ragged(new, length, P, H, D, seed=case, pad_rows=pad)
    kc, ks = ref.encode(kw)
    vc, vs = ref.encode(vh)
    for i, (sq, p) in enumerate(rows):
        mem, slot = want.pages[int(R.table[sq, p // P])], p % P
        mem[:, slot * (D // 2):(slot + 1) * (D // 2)] = kc[i, :, 0::2] | kc[i, :, 1::2] << 4
        mem[:, P * D // 2 + ((slot // 4) * (D // 2) + torch.arange(D // 2)) * 4 + slot % 4] = vc[i, :, 0::2] | vc[i, :, 1::2] << 4
        mem[:, P * D + slot * (D // 32):P * D + (slot + 1) * (D // 32)] = ks[i]
        mem[:, P * D + P * D // 32 + ((slot // 4) * (D // 32) + torch.arange(D // 32)) * 4 + slot % 4] = vs[i]
    assert torch.equal(cache.pages.cpu(), want.pages)
    # and back
    for rt in (torch.float32, torch.bfloat16, torch.float16):
        kr, vr = (torch.full((n, H, D), 7.0, dtype=rt, device="cuda:0") for _ in range(2))
        lbm.lb_kv_read(cache, batch, k_out=kr, v_out=vr)
        for got, (code, scale) in ((kr, (kc, ks)), (vr, (vc, vs))):
            assert torch.equal(got[:m].cpu(), ref.decode(code, scale).to(rt))
            assert bool((got[m:] == 7.0).all())


def test_append_in_place_and_without_queries():
    rng = np.random.default_rng(3)
    for inter in (False, True):
        R = ref.Ragged([6, 1], [30, 9], 16, 2, 64, seed=1)
        cos, sin = angles(R, 32)
        rope = lbm.Rope(dev(cos), dev(sin), int(inter))
        q, k, v = (dev(randn(rng, 7, h, 64, dtype=torch.bfloat16)) for h in (4, 2, 2))
        a, b = handles(R), handles(R)
        apart = lbm.lb_kv_append(*a, q.clone(), k, v, rope=rope)
        same = q.clone()
        assert lbm.lb_kv_append(*b, same, k, v, rope=rope, q_out=same) is same
        assert torch.equal(apart, same) and torch.equal(a[0].pages, b[0].pages)
        c = handles(R)
        assert lbm.lb_kv_append(*c, None, k, v, rope=rope) is None
        assert torch.equal(a[0].pages, c[0].pages)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_append_at_the_limits_of_a_block(t):
    """Zeros, the smallest and largest numbers, values on every border of the codes, infinities and NaN."""
    dt = DT[t]
    big, tiny = torch.finfo(dt).max, torch.finfo(dt).smallest_normal
    rows = torch.zeros(10, 64, dtype=torch.float64)
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    rows[1, :32] = torch.cat([borders, -borders, borders * 0.5, borders * 1.5])
    rows[1, 32:] = 2.0 ** -12 * rows[1, :32]
    rows[2, 0], rows[2, 33] = big, -big
    rows[2, 1:32] = big / 3
    rows[3] = tiny
    rows[4] = torch.finfo(dt).smallest_normal * 2.0 ** -3  # subnormal
    rows[5, 5], rows[5, 40] = math.inf, -1.0
    rows[6, 31], rows[6, 63] = math.nan, -math.inf
    rows[7] = -0.0
    rows[8, :32], rows[8, 32:] = 1.5, 1.5000001 if t == "f32" else 1.5078125
    rows[9, :8] = 1e-30 if t != "f16" else 6e-8
    x = rows.to(dt).view(10, 1, 64)
    R = ref.Ragged([10], [10], 16, 1, 64, seed=4)
    cache, batch = handles(R)
    say(f"[case] limits {t}")
    lbm.lb_kv_append(cache, batch, None, dev(x), dev(x))
    k, v = lbm.lb_kv_read(cache, batch)
    code, scale = ref.encode(x)
    want = ref.decode(code, scale)
    for got in (k, v):
        close(got, want, 0.0, t)
    assert bool(torch.isnan(k[5, 0, :32]).all()) and not bool(torch.isnan(k[5, 0, 32:]).any())


def test_append_leaves_out_what_does_not_fit():
    """Pages outside the pool, lengths past the table, more new tokens than tokens, positions past the
    angles: flagged, nothing else is written, no neighbour is touched."""
    rng = np.random.default_rng(5)
    base = ref.Ragged([2, 2], [20, 30], 16, 1, 64, seed=6)
    k, v = (dev(randn(rng, 4, 1, 64)) for _ in range(2))

    def run(change, rope=None):
        R = ref.Ragged([2, 2], [20, 30], 16, 1, 64, seed=6)
        change(R)
        cache, batch = handles(R)
        lbm.lb_kv_append(cache, batch, None, k, v, rope=rope)
        out, _ = lbm.lb_kv_attend(cache, batch, k, 1.0)
        assert bool(torch.isfinite(out).all() | torch.isnan(out).any())
        return cache.status(), cache.pages.cpu()

    say("[case] bad batches")
    st, pages = run(lambda R: None)
    assert st == 0
    good = pages.clone()
    for page in (-1, base.n_pages, 2 ** 31 - 1, -2 ** 31):
        def bad_page(R):
            R.table[0, 1] = page
        st, pages = run(bad_page)
        assert st & lbm.LB_KV_BAD_PAGE
        changed = [i for i in range(base.n_pages) if not torch.equal(pages[i], base.pages[i])]
        assert changed == [int(base.table[1, 1])] and torch.equal(pages[changed[0]], good[changed[0]])
    for value in (33, 10 ** 9, -1, 1):
        def bad_length(R):
            R.lengths[0] = value
        st, pages = run(bad_length)
        assert st & lbm.LB_KV_BAD_LENGTH
        assert torch.equal(pages[int(base.table[1, 1])], good[int(base.table[1, 1])])
    for starts in ([0, 2, 9], [0, -5, 4], [7, 2, 4], [0, 3, 2]):
        def bad_starts(R):
            R.starts[:] = torch.tensor(starts, dtype=torch.int32)
        st, pages = run(bad_starts)
        assert st & lbm.LB_KV_BAD_LENGTH
    cos, sin = lbm.lb_rope_table(29, 16)
    st, pages = run(lambda R: None, lbm.Rope(dev(cos), dev(sin)))
    assert st == lbm.LB_KV_BAD_LENGTH  # positions 28, 29 of the second sequence: the last has no angle


# ------------------------------------------------------------------ attention


ATTEND = [  # new, length, page, q heads, kv heads, D, window, type, padding rows
    ([1], [1], 16, 4, 4, 64, 0, "f32", 0),
    ([1], [200], 16, 4, 4, 64, 0, "f32", 0),
    ([1, 1, 1, 1], [16, 17, 33, 250], 16, 8, 2, 128, 0, "bf16", 0),
    ([1, 0, 1], [700, 5, 1], 32, 4, 1, 128, 100, "f16", 2),
    ([5, 40, 1], [5, 77, 130], 16, 6, 2, 64, 0, "bf16", 1),
    ([33, 2], [64, 2], 64, 3, 3, 256, 9, "f32", 0),
    ([70], [70], 16, 16, 1, 64, 0, "f16", 0),
    ([20, 20], [300, 21], 128, 7, 1, 128, 33, "bf16", 0),
    ([1] * 3, [1, 500, 31], 256, 2, 2, 256, 0, "bf16", 0),
    ([130], [400], 32, 4, 2, 128, 1, "f32", 0),
    ([1, 9], [3000, 1800], 64, 8, 8, 64, 0, "bf16", 0),
    # prompts and single tokens in one batch: each by the kernel for its number of rows, the single ones by parts of their keys
    ([1, 90, 0, 1, 33, 1], [2100, 200, 9, 40, 33, 1], 16, 4, 1, 128, 0, "bf16", 3),
    ([200, 1, 17], [210, 1300, 17], 32, 4, 2, 256, 0, "bf16", 0),
    ([17, 64, 65, 129, 1, 2, 3], [17, 70, 65, 500, 1, 64, 30], 64, 2, 2, 64, 40, "f16", 1),
    ([150, 1], [333, 700], 16, 3, 1, 128, 64, "f32", 0),
    ([70, 3], [90, 5], 16, 2, 1, 256, 2 ** 31 - 1, "f32", 0),
    ([66, 1], [70, 1], 128, 5, 1, 256, 0, "f16", 0),
    # enough rows for the kernel that takes many, with sequences of few rows beside and without
    ([700], [800], 32, 112, 16, 64, 0, "bf16", 1),
    ([650, 1, 3, 0, 40], [650, 1500, 64, 7, 300], 16, 128, 8, 64, 0, "bf16", 2),
    ([310, 300], [330, 333], 64, 128, 4, 128, 90, "bf16", 0),
    ([301, 1], [320, 900], 16, 256, 8, 64, 0, "f16", 0),
    ([300, 2], [300, 400], 32, 260, 4, 128, 17, "f32", 0),
    ([305], [306], 128, 256, 2, 256, 0, "bf16", 0),
    ([160, 140, 2], [160, 200, 200], 16, 256, 4, 256, 0, "f32", 3),
]
# What the probabilities' pieces leave: bf16 has 8 significant bits, so a piece is off by at most half a step, 2^-8 of
# what it stands for, and 1, 2 and 3 pieces by 2^-8, 2^-16 and 2^-24.
PIECE = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -16, torch.float32: 2.0 ** -24}


def bounds(want, lse, mass, reach, dt, D, n):
    """Error of an attention row: the output's rounding; the probabilities' rounding to bf16 pieces; scores summed
    in 32 bits over D channels (off by at most D 2^-23 of the sum of magnitudes, which moves a probability by
    twice that), the exponential's and the sums' own roundings."""
    delta = (D + 8) * 2.0 ** -23 * reach + 2.0 ** -21 * (1 + reach)
    out = ref.EPS[dt] * want.abs() + (PIECE[dt] + 4 * delta + n * 2.0 ** -24).unsqueeze(-1) * mass + 2.0 ** -25 * (dt == torch.float16)
    return out, 2 * delta + n * 2.0 ** -24 + 2.0 ** -22 * torch.where(torch.isfinite(lse), lse.abs(), 0.0)


def check_attend(R, q, got, lse, scale, window, skip=()):
    m = 0
    for s, n in enumerate(R.new):
        if n and s not in skip:
            k, v = R.get(s, R.length[s])
            want, wl, mass, reach = ref.attend(q.cpu()[m:m + n].double(), k, v, scale, R.length[s] - n, window)
            b, bl = bounds(want, wl, mass, reach, q.dtype, R.D, R.length[s])
            close(got[m:m + n], want, b, f"sequence {s}")
            if lse is not None:
                close(lse[m:m + n], wl, bl, f"lse of sequence {s}")
        m += n


@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attend(case):
    new, length, P, Hq, H, D, window, t, pad = ATTEND[case]
    say(f"[case] attend {case}")
    rng = np.random.default_rng(100 + case)
    R = ref.Ragged(new, length, P, H, D, seed=case, pad_rows=pad)
    for s, n in enumerate(length):
        R.put(s, randn(rng, n, H, D, dtype=torch.float64) + 2 * randn(rng, 1, H, D, dtype=torch.float64), randn(rng, n, H, D, dtype=torch.float64))
    dt = DT[t]
    q = dev(randn(rng, R.n_rows, Hq, D, dtype=dt))
    cache, batch = handles(R)
    out = torch.full((R.n_rows, Hq, D), 7.0, dtype=dt, device="cuda:0")
    lse = torch.full((R.n_rows, Hq), 7.0, dtype=torch.float32, device="cuda:0")
    lbm.lb_kv_attend(cache, batch, q, D ** -0.5, window=window, out=out, lse=lse)
    torch.cuda.synchronize()
    assert cache.status() == 0
    check_attend(R, q, out, lse, D ** -0.5, window)
    m = sum(new)
    assert bool((out[m:] == 7.0).all()) and bool((lse[m:] == 7.0).all())
    # the same without lse, with strided rows, bit for bit
    wide = torch.zeros(R.n_rows, Hq * D + 64, dtype=dt, device="cuda:0")
    wide[:, :Hq * D] = q.view(R.n_rows, -1)
    again = torch.full((R.n_rows, Hq * D + 8 * 4), 7.0, dtype=dt, device="cuda:0")
    lbm.lb_kv_attend(cache, batch, wide[:, :Hq * D].unflatten(1, (Hq, D)), D ** -0.5, window=window, out=again[:, :Hq * D].unflatten(1, (Hq, D)))
    assert torch.equal(again[:, :Hq * D], out.view(R.n_rows, -1)) and bool((again[:, Hq * D:] == 7.0).all())


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("new,D,Hq", [(1, 64, 4), (12, 128, 4), (40, 64, 4), (48, 128, 4), (45, 256, 4),
                                      (310, 64, 256), (310, 128, 256), (310, 256, 256)])
def test_attend_unseen_tokens_have_no_effect(t, new, D, Hq):
    """NaN keys and values past a row's position reach no row before them; those a row sees make it NaN."""
    rng = np.random.default_rng(8)
    n = max(50, new + 7)
    G = Hq // 2
    R = ref.Ragged([new, 1], [n, 20], 16, 2, D, seed=9)
    k, v = randn(rng, n, 2, D, dtype=torch.float64), randn(rng, n, 2, D, dtype=torch.float64)
    if new > 1:
        k[n - 5, 0, 3] = math.nan    # head 0: keys from position n - 5 on
        v[n - 4, 1, 40] = math.inf   # head 1: one block of values from n - 4 on
    else:
        v[3, 1, 40] = math.nan
    R.put(0, k, v)
    R.put(1, randn(rng, 20, 2, D, dtype=torch.float64), randn(rng, 20, 2, D, dtype=torch.float64))
    q = dev(randn(rng, new + 1, Hq, D, dtype=DT[t]))
    cache, batch = handles(R)
    say(f"[case] unseen {t} {new} {D}")
    out, lse = lbm.lb_kv_attend(cache, batch, q, 0.2, want_lse=True)
    check_attend(R, q, out, None, 0.2, 0)
    o = out.cpu()
    if new > 1:
        assert bool(torch.isfinite(o[:new - 5]).all())
        assert bool(torch.isnan(o[new - 5:new, :G]).all()) and bool(torch.isnan(o[new - 4:new, G:, 32:64]).all())
        assert bool(torch.isfinite(o[:new, G:, :32]).all()) and bool(torch.isfinite(lse[:new, G:]).all())
    else:
        assert bool(torch.isnan(o[0, G:, 32:64]).all()) and bool(torch.isfinite(o[0, :, :32]).all())
    assert bool(torch.isfinite(o[new:]).all())


def test_attend_rows_that_see_nothing():
    """A missing page masks its tokens; where nothing is left out = 0 and lse = -infinity."""
    rng = np.random.default_rng(10)
    R = ref.Ragged([1, 1], [10, 40], 16, 1, 64, seed=11)
    for s in range(2):
        R.put(s, randn(rng, R.length[s], 1, 64, dtype=torch.float64), randn(rng, R.length[s], 1, 64, dtype=torch.float64))
    R.table[0, 0] = -1
    R.table[1, 1] = -1
    q = dev(randn(rng, 2, 3, 64))
    cache, batch = handles(R)
    say("[case] empty rows")
    out, lse = lbm.lb_kv_attend(cache, batch, q, 1.0, want_lse=True)
    assert cache.status() == lbm.LB_KV_BAD_PAGE
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())
    R.table[1, 1] = 0
    k, v = R.get(1, 40)
    keep = [t for t in range(40) if not 16 <= t < 32]
    want, wl, mass, reach = ref.attend(q.cpu()[1:2].double(), k[keep], v[keep], 1.0, len(keep) - 1, 0)
    b, bl = bounds(want, wl, mass, reach, torch.float32, 64, 40)
    close(out[1:2], want, b, "out")
    close(lse[1:2], wl, bl, "lse")


def test_thousands_of_ragged_sequences():
    """Each workgroup finds its sequence among 5000 of 0 to 5 new tokens: appended blocks, what is read back, and
    attention by both kernels (5 tokens of 16 heads are many rows, fewer are few)."""
    rng = np.random.default_rng(17)
    new = [int(x) for x in rng.integers(0, 6, 5000)]
    length = [n + int(x) for n, x in zip(new, rng.integers(0, 20, 5000))]
    R = ref.Ragged(new, length, 16, 1, 64, seed=18)
    rows, n = R.rows(), R.n_rows
    k, v = randn(rng, n, 1, 64, dtype=torch.bfloat16), randn(rng, n, 1, 64, dtype=torch.bfloat16)
    # the tokens before the new ones: the same for all
    old = [randn(rng, 20, 1, 64, dtype=torch.float64) for _ in range(2)]
    for s, (m, ln) in enumerate(zip(new, length)):
        R.put(s, old[0][:ln - m], old[1][:ln - m])
    cache, batch = handles(R)
    say("[case] thousands")
    lbm.lb_kv_append(cache, batch, None, dev(k), dev(v))
    kr, vr = lbm.lb_kv_read(cache, batch)
    for got, x in ((kr, k), (vr, v)):
        assert torch.equal(got.cpu().double(), ref.decode(*ref.encode(x)))
    q = dev(randn(rng, n, 16, 64, dtype=torch.bfloat16))
    out, lse = lbm.lb_kv_attend(cache, batch, q, 0.125, want_lse=True)
    assert cache.status() == 0 and n * 16 >= 128 * 600 and max(new) == 5
    R.pages = cache.pages.cpu()
    check_attend(R, q, out, lse, 0.125, 0, skip=set(range(5000)) - set(range(0, 5000, 7)) - set(range(4900, 5000)))


def test_attend_leaves_rows_out_that_no_sequence_has():
    """Starts that do not fit: the rows between the sequences, and those past max_new, stay as they were, with one
    part of the keys and with several."""
    rng = np.random.default_rng(15)
    for length in (40, 2000):
        R = ref.Ragged([2, 2], [length, 30], 16, 1, 64, seed=16)
        for s in range(2):
            R.put(s, randn(rng, R.length[s], 1, 64, dtype=torch.float64), randn(rng, R.length[s], 1, 64, dtype=torch.float64))
        q = dev(randn(rng, 6, 2, 64))
        for starts, fine, bad in (([0, 2, 6], [0, 1, 2, 3], True), ([1, 3, 5], [1, 2, 3, 4], False), ([0, -5, 4], [0, 1], True)):
            word = torch.zeros(1, dtype=torch.int32, device="cuda:0")
            cache = lbm.KVCache(dev(R.pages), 16, 1, 64, flags=word)
            batch = lbm.KVBatch(dev(torch.tensor(starts, dtype=torch.int32)), dev(R.lengths), dev(R.table), 6, 2)
            say(f"[case] rows left out {length} {starts}")
            out, lse = torch.full((6, 2, 64), 7.0, device="cuda:0"), torch.full((6, 2), 7.0, device="cuda:0")
            lbm.lb_kv_attend(cache, batch, q, 1.0, out=out, lse=lse)
            rest = [i for i in range(6) if i not in fine]
            assert bool((out[rest] == 7.0).all()) and bool((lse[rest] == 7.0).all())
            assert not bool((lse[fine] == 7.0).any())
            assert cache.status() == (lbm.LB_KV_BAD_LENGTH if bad else 0)


@pytest.mark.parametrize("starts", [[0, -5, 4], [7, 2, 4], [0, 3, 2], [0, 2, 9], [-2 ** 31, 2, 4]])
def test_append_alone_reports_starts_that_do_not_fit(starts):
    R = ref.Ragged([2, 2], [20, 30], 16, 1, 64, seed=6)
    R.starts[:] = torch.tensor(starts, dtype=torch.int32)
    cache, batch = handles(R)
    k = torch.zeros(4, 1, 64, device="cuda:0")
    say(f"[case] append starts {starts}")
    lbm.lb_kv_append(cache, batch, None, k, k)
    assert cache.status() == lbm.LB_KV_BAD_LENGTH


def test_attend_large_scores():
    """Scores of many thousands: the softmax is a choice of one token."""
    rng = np.random.default_rng(12)
    R = ref.Ragged([1], [100], 16, 1, 64, seed=13)
    R.put(0, 100 * randn(rng, 100, 1, 64, dtype=torch.float64), randn(rng, 100, 1, 64, dtype=torch.float64))
    q = dev(100 * randn(rng, 1, 1, 64, dtype=torch.bfloat16))
    cache, batch = handles(R)
    out, lse = lbm.lb_kv_attend(cache, batch, q, 1.0, want_lse=True)
    k, v = R.get(0, 100)
    s = k[:, 0] @ q.cpu().double()[0, 0]
    top = s.sort().values
    assert float(top[-1] - top[-2]) > 50
    close(out[0, 0], v[int(s.argmax()), 0], 2.0 ** -8 * v[int(s.argmax()), 0].abs(), "out")
    close(lse[0], s.max()[None], 2.0 ** -15 * float(s.max()), "lse")


# ------------------------------------------------------------------ adapters


LORA = [  # rows, d_in, d_out, rank, adapters, ids, type
    (1, 8, 8, 8, 1, "runs", "f32"),
    (1, 256, 768, 16, 3, "each", "bf16"),
    (17, 264, 776, 16, 5, "each", "f32"),
    (40, 2048, 520, 24, 4, "runs", "bf16"),
    (33, 1000, 264, 64, 7, "each", "f16"),
    (16, 512, 4096, 128, 2, "runs", "f16"),
    (50, 136, 64, 96, 60, "each", "bf16"),
    (300, 72, 40, 32, 3, "none", "f32"),
    (5, 4096, 8, 8, 2, "each", "f16"),
    # one launch or two, the rank's tiles side by side or not, a rank that ends inside a tile
    (256, 200, 1024, 16, 9, "each", "f32"),
    (257, 200, 1024, 16, 9, "each", "bf16"),
    (70, 2048, 1032, 32, 5, "runs", "bf16"),
    (21, 2040, 600, 32, 5, "each", "f32"),
    (9, 64, 2000, 120, 3, "each", "f16"),
    (1030, 96, 272, 56, 4, "runs", "f16"),
]


@pytest.mark.parametrize("case", range(len(LORA)))
def test_lora_add(case):
    rows, d_in, d_out, r, n, ids, t = LORA[case]
    say(f"[case] lora {case}")
    rng = np.random.default_rng(200 + case)
    dt = DT[t]
    x, y = randn(rng, rows, d_in, dtype=dt), randn(rng, rows, d_out, dtype=dt)
    a, b = (randn(rng, n, r, d_in) / d_in ** 0.5).to(dt), (randn(rng, n, d_out, r) / r ** 0.5).to(dt)
    scale = torch.from_numpy(rng.uniform(-2, 2, n)).float()
    if ids == "each":
        adapter = torch.from_numpy(rng.integers(-2, n + 2, rows).astype(np.int32))  # some outside 0..n-1
    elif ids == "runs":
        adapter = torch.arange(rows, dtype=torch.int32) // 7 % n
    else:
        adapter = torch.full((rows,), -1, dtype=torch.int32)
        adapter[::16] = 1
    out = torch.full((rows, d_out), 7.0, dtype=dt, device="cuda:0")
    ins = [dev(v) for v in (y, x, a, b, adapter, scale)]
    assert lbm.lb_lora_add(*ins, out=out) is out
    want, bound = y.double(), torch.zeros(rows, d_out, dtype=torch.float64)
    piece = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21}[dt]
    for i in range(rows):
        k = int(adapter[i])
        if 0 <= k < n:
            h, hm = a[k].double() @ x[i].double(), a[k].double().abs() @ x[i].double().abs()
            s = float(scale[k])
            want[i] += s * (b[k].double() @ h)
            # h summed in 32 bits over d_in and then taken in two pieces; the products with B summed over 2 rank entries
            dh = (d_in + 8) * 2.0 ** -24 * hm + piece * h.abs().max()
            bound[i] = abs(s) * (b[k].double().abs() @ (dh + (2 * r + 4) * 2.0 ** -24 * (h.abs() + dh)))
    bound += (ref.EPS[dt] + 2.0 ** -23) * want.abs() + ref.EPS[dt] * bound + 2.0 ** -25 * (dt == torch.float16)
    close(out, want, bound, "out")
    none = (adapter < 0) | (adapter >= n)
    assert torch.equal(out.cpu()[none], y[none])
    # in place, strided, with a scale of one for all: the same rows
    wide = torch.full((rows, d_out + 16), 7.0, dtype=dt, device="cuda:0")
    wide[:, :d_out] = ins[0]
    xw = torch.zeros((rows, d_in + 8), dtype=dt, device="cuda:0")
    xw[:, :d_in] = ins[1]
    lbm.lb_lora_add(wide[:, :d_out], xw[:, :d_in], ins[2], ins[3], ins[4], ins[5])
    assert torch.equal(wide[:, :d_out], out) and bool((wide[:, d_out:] == 7.0).all())
    one = lbm.lb_lora_add(*ins[:5], None, out=torch.empty_like(out))
    assert torch.equal(one, lbm.lb_lora_add(*ins[:5], torch.ones(n, device="cuda:0"), out=torch.empty_like(out)))


def test_lora_rows_do_not_mix():
    """A NaN or infinite row, and a NaN adapter, stay in their own rows."""
    rng = np.random.default_rng(14)
    for dt in DT.values():
        x, y = randn(rng, 32, 64, dtype=dt), randn(rng, 32, 48, dtype=dt)
        a, b = randn(rng, 4, 16, 64, dtype=dt), randn(rng, 4, 48, 16, dtype=dt)
        x[3, 5], x[20, 0] = math.nan, math.inf
        a[2, 1, 1] = math.nan
        adapter = torch.tensor([0, 1, 3, 0] * 4 + [0, 1, 2, 3] * 4, dtype=torch.int32)
        say(f"[case] lora mix {dt}")
        out = lbm.lb_lora_add(*(dev(v) for v in (y, x, a, b, adapter)), out=torch.empty(32, 48, dtype=dt, device="cuda:0")).cpu()
        bad = [3, 20] + [i for i in range(32) if adapter[i] == 2]
        good = [i for i in range(32) if i not in bad]
        assert bool(torch.isfinite(out[good]).all())
        assert not bool(torch.isfinite(out[bad]).any())


def test_lora_f16_products_past_the_type():
    """h beyond fp16's range and far below it: the result is what 32 bits give."""
    for big in (2.0 ** 11, 2.0 ** -14):
        x = torch.full((1, 64), big, dtype=torch.float16)
        a = torch.full((1, 8, 64), 2.0, dtype=torch.float16)       # h = 128 * big: 2^18, or 2^-7
        b = torch.full((1, 8, 8), 2.0 ** -10, dtype=torch.float16)
        y = torch.zeros(1, 8, dtype=torch.float16)
        out = lbm.lb_lora_add(*(dev(v) for v in (y, x, a, b, torch.zeros(1, dtype=torch.int32))))
        assert bool((out == 8 * 128 * big * 2.0 ** -10).all())


# ------------------------------------------------------------------ logits


def bit_mask(rng, rows, classes, keep):
    words = -(-classes // 32)
    bits = rng.random((rows, words * 32)) < keep
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).reshape(rows, words).copy())


LOGITS = [  # rows, classes, history, biases, bias rows, masks, mask rows named, type, temperature
    (1, 1, 0, 0, 0, 0, False, "f32", 1.0),
    (7, 41, 5, 3, 1, 1, False, "f32", 1.3),
    (300, 41, 0, 4, 1, 0, False, "bf16", 1.0),
    (9, 64, 70, 64, 9, 3, True, "f16", 0.7),
    (33, 129, 3, 0, 0, 33, False, "f32", 2.0),
    (2, 5000, 200, 100, 2, 5, True, "f32", 1.0),
    (1, 70001, 300, 50, 1, 1, False, "bf16", 1.1),
    (3, 131073, 40, 7, 3, 2, True, "f16", 1.0),
    (600, 1025, 2, 2, 600, 0, False, "f32", 1.0),
    (1, 4000, 3000, 1096, 1, 0, False, "f32", 1.0),
]


@pytest.mark.parametrize("case", range(len(LOGITS)))
def test_logits_adjust(case):
    R, C, H, W, wrows, masks, named, t, temp = LOGITS[case]
    say(f"[case] logits {case}")
    rng = np.random.default_rng(300 + case)
    dt = DT[t]
    x = (3 * randn(rng, R, C)).to(dt)
    rules = dict(temperature=temp, repetition=1.3, presence=0.25, frequency=0.125)
    if H:
        rules["history"] = torch.from_numpy(rng.integers(-3, min(C + 3, 60), (R, H)).astype(np.int32))
    if W:
        rules["bias_ids"] = torch.from_numpy(rng.integers(-2, C + 2, (wrows, W)).astype(np.int32))
        rules["bias_values"] = randn(rng, wrows, W)
    if masks:
        rules["mask"] = bit_mask(rng, masks, C, 0.6)
        if named:
            rules["mask_row"] = torch.from_numpy(rng.integers(-1, masks + 1, R).astype(np.int32))
    if masks == R and not named:
        rules["mask"][0] = 0  # a row with nothing left
    target = torch.from_numpy(rng.integers(0, C, R).astype(np.int32))
    if R > 3:
        target[1], target[2] = -1, C
    z = ref.logits_rules(x, **rules)
    logp, lse = ref.log_softmax(z)
    on = lbm.LogitRules(**{k: dev(v) if isinstance(v, torch.Tensor) else v for k, v in rules.items()})
    xd = dev(x)
    got, score, gl = lbm.lb_logits_adjust(xd, on, target=dev(target))
    # four roundings of the rules at the logit's size, and those of at most 2 C / 256 + 64 sums of positive terms
    zmax = torch.where(torch.isfinite(z), z.abs(), 0.0)
    rule = 6 * 2.0 ** -24 * (zmax + x.abs().double().amax(1, keepdim=True) * 2 + 40)
    summed = (2 * C / 256 + 64) * 2.0 ** -24 + 2.0 ** -21
    bl = rule.amax(1) + summed + 2.0 ** -22 * torch.where(torch.isfinite(lse), lse.abs(), 0.0)
    close(gl, lse, bl, "lse")
    close(got, logp, rule + bl[:, None] + 2.0 ** -23 * torch.where(torch.isfinite(logp), logp.abs(), 0.0), "logprobs")
    want = torch.zeros(R, dtype=torch.float64)
    for r in range(R):
        w = int(target[r])
        want[r] = 0.0 if w < 0 else math.nan if w >= C else float(got[r, w])
    close(score, want, 0.0, "score")
    # without log-probabilities, strided and unaligned rows: the same numbers
    wide = torch.zeros(R, C + 3, dtype=dt, device="cuda:0")
    wide[:, 1:C + 1] = xd
    none, s2, l2 = lbm.lb_logits_adjust(wide[:, 1:C + 1], on, target=dev(target), want_logprobs=False)
    assert none is None
    close(s2, score.cpu().double(), 2 * float(bl.max()), "score alone")
    close(l2, gl.cpu().double(), 2 * bl, "lse alone")
    if t == "f32":
        lbm.lb_logits_adjust(xd, on, logprobs=xd)
        close(xd, got.cpu().double(), 2 * float(bl.max()), "in place")


@pytest.mark.parametrize("C", [41, 3000, 20000])
def test_logits_with_infinities_and_nan(C):
    x = torch.zeros(8, C)
    x[0, 3] = -math.inf
    x[1] = torch.finfo(torch.float32).min
    x[2, 5] = math.nan
    x[3, 6] = math.inf
    x[4] = -math.inf
    x[5, 7], x[6, 7] = math.nan, math.inf
    keep = torch.ones(8, C, dtype=torch.bool)
    keep[5:7, 7] = False  # masked: no effect
    keep[7] = False
    words = -(-C // 32)
    bits = torch.zeros(8, words * 32, dtype=torch.bool)
    bits[:, :C] = keep
    mask = torch.from_numpy(np.packbits(bits.numpy(), axis=1, bitorder="little").view(np.int32).reshape(8, words).copy())
    say(f"[case] logits inf nan {C}")
    got, _, lse = lbm.lb_logits_adjust(dev(x), lbm.LogitRules(mask=dev(mask)))
    got, lse = got.cpu().double(), lse.cpu().double()
    ln = math.log(C)
    tol = (2 * C / 256 + 64) * 2.0 ** -24 * (1 + ln)
    assert got[0, 3] == -math.inf and abs(float(got[0, 0]) + math.log(C - 1)) < tol
    assert float((got[1] + ln).abs().max()) < tol
    assert bool(torch.isnan(got[2]).all()) and bool(torch.isnan(lse[2]))
    assert lse[3] == math.inf and bool(torch.isnan(got[3, 6])) and got[3, 0] == -math.inf
    assert bool((got[4] == -math.inf).all()) and lse[4] == -math.inf
    for r in (5, 6):
        assert got[r, 7] == -math.inf and abs(float(lse[r]) - math.log(C - 1)) < tol
    assert bool((got[7] == -math.inf).all()) and lse[7] == -math.inf


# ------------------------------------------------------------------ streams and graphs


def _pass(n, seed):
    """Inputs of one scorer step over all four operators, and the step."""
    rng = np.random.default_rng(seed)
    R = ref.Ragged([3, 1, 5], [700, 40, 5], 16, 2, 64, seed=seed)
    for s, ln in enumerate(R.length):
        R.put(s, randn(rng, ln, 2, 64, dtype=torch.float64), randn(rng, ln, 2, 64, dtype=torch.float64))
    cache, batch = handles(R)
    cos, sin = angles(R, 64)
    rope = lbm.Rope(dev(cos), dev(sin))
    x = dev(randn(rng, 9, 128, dtype=torch.bfloat16))
    base = dev(randn(rng, 9, 512, dtype=torch.bfloat16))
    a, b = dev(randn(rng, 2, 16, 128, dtype=torch.bfloat16) * 0.1), dev(randn(rng, 2, 512, 16, dtype=torch.bfloat16) * 0.1)
    adapter = dev(torch.tensor([0, 0, 0, 1, -1, -1, -1, -1, -1], dtype=torch.int32))
    head = dev(randn(rng, 5000, 256))
    target = dev(torch.arange(9, dtype=torch.int32) * 7)
    qkv, q = torch.empty_like(base), torch.empty(9, 4, 64, dtype=torch.bfloat16, device="cuda:0")
    out = torch.empty_like(q)
    logp = torch.empty(9, 5000, device="cuda:0")
    logits = torch.empty(9, 5000, device="cuda:0")
    lse = torch.empty(9, 4, device="cuda:0")
    ws = [torch.empty(max(16, nb), dtype=torch.uint8, device="cuda:0") for nb in (
        lbm.lb_lora_workspace(9, 128, 512, 16), lbm.lb_kv_attend_workspace(cache, batch, 4), lbm.lb_logits_workspace(9, 5000))]
    res = {}

    def step(stream=None):
        lbm.lb_lora_add(base, x, a, b, adapter, out=qkv, workspace=ws[0], stream=stream)
        parts = [qkv[:, i:j].unflatten(1, (-1, 64)) for i, j in ((0, 256), (256, 384), (384, 512))]
        lbm.lb_kv_append(cache, batch, *parts, rope=rope, q_out=q, stream=stream)
        lbm.lb_kv_attend(cache, batch, q, 0.125, out=out, lse=lse, workspace=ws[1], stream=stream)
        torch.matmul(out.view(9, 256).float(), head.t(), out=logits)
        res["logits"] = lbm.lb_logits_adjust(logits, None, target=target, logprobs=logp, workspace=ws[2], stream=stream)

    return step, lambda: [qkv, q, out, lse, cache.pages, logp, res["logits"][1], res["logits"][2]], [x, base]


def test_a_scorer_step_captured_and_replayed():
    """Two graphs of whole steps, replayed in turn with new inputs and eager work between: every replay gives the
    eager result bit for bit."""
    say("[case] graphs")
    steps = [_pass(9, 20), _pass(9, 21)]
    side = torch.cuda.Stream()
    graphs = []
    for step, outs, ins in steps:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append((g, outs()))
    for k in range(4):
        for (g, got), (step, outs, ins) in zip(graphs, steps):
            for t in ins:
                t.mul_(1.25 if k % 2 else -0.8)
            g.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in got]
            step()
            torch.cuda.synchronize()
            for a, b in zip(replayed, outs()):
                assert torch.equal(a, b)


def test_a_stream_of_the_callers():
    """A call on another stream than torch's current one, outputs and workspaces made by the call."""
    say("[case] streams")
    step, outs, ins = _pass(9, 22)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs()]
    side = torch.cuda.Stream()
    rng = np.random.default_rng(1)
    R = ref.Ragged([1, 1], [900, 30], 16, 1, 64, seed=3)
    for s in range(2):
        R.put(s, randn(rng, R.length[s], 1, 64, dtype=torch.float64), randn(rng, R.length[s], 1, 64, dtype=torch.float64))
    cache, batch = handles(R)
    q = dev(randn(rng, 2, 4, 64))
    plain, _ = lbm.lb_kv_attend(cache, batch, q, 0.1)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got, _ = lbm.lb_kv_attend(cache, batch, q, 0.1, stream=stream)
        torch.empty(1 << 20, device="cuda:0").fill_(3.0)  # memory that a freed workspace would be given to
        side.synchronize()
        assert torch.equal(got, plain)
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    for a, b in zip(want, outs()):
        assert torch.equal(a, b)


def test_new_memory_belongs_to_the_call_s_stream():
    """A block that torch's current stream has just let go of may still be in use by work queued there: a call on
    another stream does not get it."""
    side = torch.cuda.Stream()
    logits, target = torch.zeros(64, 50000, device="cuda:0"), torch.zeros(64, dtype=torch.int32, device="cuda:0")
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        held = [torch.empty(64 * 50000, device="cuda:0"), torch.empty(64, device="cuda:0"), torch.empty(64, device="cuda:0")]
        old = {t.data_ptr() for t in held}
        del held
        new = lbm.lb_logits_adjust(logits, target=target, stream=stream)
        assert not old & {t.data_ptr() for t in new}
        side.synchronize()
        close(new[2], torch.full((64,), math.log(50000), dtype=torch.float64), 2.0 ** -18, "lse")
    null = lbm.lb_logits_adjust(logits, target=target, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(null[2], new[2])


# ------------------------------------------------------------------ the cached word LM


def lm64(lm, cached, key, adapters=None):
    """The model in 64 bits on the keys and values that the cache holds of a sequence: its score, and how far these
    are from the model's own, as a part of their block's largest."""
    which, words = key
    n, hd = len(words), lm.d // lm.h
    pages = cached.held[key][0]
    R = ref.Ragged([], [], cached.P, lm.h, hd)
    R.table = torch.tensor([pages], dtype=torch.int32)
    norm = lambda x: (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, keepdim=True, unbiased=False) + 1e-5)
    W = lambda p: p.detach().cpu().double()
    z = W(lm.emb)[[lm.bos] + list(words[:-1])] + W(lm.pos)[:n]
    off = 0.0
    for i, m in enumerate(lm.layers):
        k, v = R.get(0, n, cached.caches[i].pages.cpu())
        a = norm(z)
        qkv = a @ W(m.qkv).t()
        if adapters is not None and 0 <= which < adapters[i][0].shape[0]:
            qkv = qkv + a @ W(adapters[i][0][which]).t() @ W(adapters[i][1][which]).t()
        q, kk, vv = (x.reshape(n, lm.h, hd) for x in qkv.split(lm.d, dim=1))
        for got, own in ((k, kk), (v, vv)):
            most = own.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
            off = max(off, float(((got - own).unflatten(-1, (-1, 32)).abs() / most).max()))
        o = ref.attend(q, k, v, 1 / math.sqrt(hd), 0, 0)[0]
        z = z + o.reshape(n, lm.d) @ W(m.proj).t()
        h = norm(z) @ W(m.up).t()
        z = z + (h * 0.5 * (1 + torch.erf(h / math.sqrt(2)))) @ W(m.down).t()
    lp = torch.log_softmax(norm(z) @ W(lm.emb).t() * lm.out_scale, 1)
    return float(lp[torch.arange(n), list(words)].sum()), off


def test_cached_lm_scores():
    """Sequences that grow over several calls, branch inside a page, repeat and come back after they made room: each
    score is the 64-bit one on the cache's contents, whose keys and values are the model's to half a step of 4 bits."""
    from workloads.fusion_lm import CachedWordLM, CausalWordLM
    V, BOS, d = 600, 599, 128
    lm = CausalWordLM(V, BOS, d_model=d, n_layers=2, n_heads=2, max_len=64, seed=5).to("cuda:0")
    g = torch.Generator().manual_seed(3)
    adapters = [(torch.randn(3, 8, d, generator=g).to("cuda:0") * 0.05, torch.randn(3, 3 * d, 8, generator=g).to("cuda:0") * 0.05)
                for _ in range(2)]
    rng = np.random.default_rng(4)
    word = lambda n: [int(x) for x in rng.integers(0, V, n)]
    a, b = word(13), word(30)
    calls = [[a[:5], b, [], a[:5]],
             [a, a[:5] + word(14), b + word(9), b[:16] + word(3), a[:5] + word(1)],
             [a + word(20), a, word(1), b],
             [word(40), word(47), word(33), word(50), word(44), word(61), word(17)],
             [a[:5] + word(2), b]]
    for use in (None, adapters):
        cached = CachedWordLM(lm, n_pages=26, adapters=use)
        for k, seqs in enumerate(calls):
            say(f"[case] cached lm {use is not None} call {k}")
            L = max(1, max(map(len, seqs)))
            rows = torch.full((len(seqs), L), -1, dtype=torch.int32)
            for i, s in enumerate(seqs):
                rows[i, :len(s)] = torch.tensor(s, dtype=torch.int32)
            lens = torch.tensor([len(s) for s in seqs])
            ids = None if use is None else torch.tensor([(i % 4) - 1 for i in range(len(seqs))])
            got = cached.score(rows.to("cuda:0"), lens.to("cuda:0"), ids)
            assert [c.status() for c in cached.caches] == [0, 0]
            for i, s in enumerate(seqs):
                if not s:
                    assert float(got[i]) == 0.0
                    continue
                want, off = lm64(lm, cached, (-1 if ids is None else int(ids[i]), tuple(s)), use)
                # each word's log-probability: sums over d channels in 32 bits, through a dozen products and norms
                assert abs(float(got[i]) - want) < len(s) * 64 * d * 2.0 ** -24
                # half the widest step (4 to 6) is one scale, the scale less than a third of the largest value
                assert off < (1 + 2.0 ** -10) / 3
            in_use = sorted(p for pages, _ in cached.held.values() for p in set(pages))
            assert all(cached.uses[p] == in_use.count(p) for p in range(26))
            assert sorted(cached.free) == [p for p in range(26) if cached.uses[p] == 0]
        before = dict(cached.held)
        too_many = torch.randint(0, V, (8, 60), generator=g)
        with pytest.raises(ValueError):
            cached.score(too_many.to("cuda:0"), torch.full((8,), 60))
        assert all(cached.uses[p] == sum(p in pages for pages, _ in cached.held.values()) for p in range(26))
        assert set(cached.held) <= set(before)
        with pytest.raises(ValueError):
            cached.score(torch.zeros(1, 64, dtype=torch.int32), torch.tensor([64]))
        cached.reset()
        assert not cached.held and len(cached.free) == 26


def test_cached_lm_answers_a_request():
    """An exported request scored through the cached model: each asked sub-beam's score is the 64-bit one on the
    cache's contents, the others get 0."""
    from workloads.fusion_lm import CachedWordLM, CausalWordLM, score_requests
    V, BOS, d = 200, 199, 256
    lm = CausalWordLM(V, BOS, seed=2).to("cuda:0")
    cached = CachedWordLM(lm, n_pages=512)
    rng = np.random.default_rng(7)
    words = torch.from_numpy(rng.integers(0, V, (2, 4, 2, 16)).astype(np.int32))
    for n in (3, 6, 11):  # the same words, more of them each time
        counts = torch.from_numpy(rng.integers(-1, n + 1, (2, 4, 2)).astype(np.int32))
        say(f"[case] request {n}")
        got = score_requests(words.to("cuda:0"), counts.to("cuda:0"), cached.score, batch=3).cpu()
        for at in np.ndindex(*counts.shape):
            m = int(counts[at])
            want = lm64(lm, cached, (-1, tuple(words[at][:m].tolist())))[0] if m > 0 else 0.0
            assert abs(float(got[at]) - want) <= max(m, 0) * 64 * d * 2.0 ** -24


def _three(seed):
    """Inputs of calls that need workspaces, and the calls with all memory their own."""
    rng = np.random.default_rng(seed)
    R = ref.Ragged([1, 2], [1900, 1400], 16, 2, 64, seed=seed)
    for s, ln in enumerate(R.length):
        R.put(s, randn(rng, ln, 2, 64, dtype=torch.float64), randn(rng, ln, 2, 64, dtype=torch.float64))
    cache, batch = handles(R)
    q, logits = dev(randn(rng, 3, 8, 64)), dev(randn(rng, 2, 30000))
    x, y = dev(randn(rng, 300, 64)), dev(randn(rng, 300, 96))
    a, b = dev(randn(rng, 4, 16, 64)), dev(randn(rng, 4, 96, 16))
    ids = dev(torch.arange(300, dtype=torch.int32) % 5)
    target = dev(torch.tensor([3, 29999], dtype=torch.int32))

    def calls(stream=None):
        out, lse = lbm.lb_kv_attend(cache, batch, q, 0.2, want_lse=True, stream=stream)
        z = lbm.lb_lora_add(y, x, a, b, ids, out=torch.empty_like(y), stream=stream)
        return [out, lse, z, *lbm.lb_logits_adjust(logits, target=target, stream=stream)]

    assert lbm.lb_kv_attend_workspace(cache, batch, 8) > 0 and lbm.lb_lora_workspace(300, 64, 96, 16) > 0 \
        and lbm.lb_logits_workspace(2, 30000) > 0
    return calls, [q, x, logits]


def test_captured_calls_with_workspaces_of_their_own():
    calls, ins = _three(30)
    say("[case] graph, own workspaces")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = calls()
    for k in range(4):
        for t in ins:
            t.mul_(-0.75 if k % 2 else 1.25)
        g.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in got]
        for a, b in zip(replayed, calls()):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    """Each has outputs and workspaces of its own: the results are those of one after the other."""
    sets = [_three(31), _three(32)]
    want = [[t.clone() for t in calls()] for calls, _ in sets]
    torch.cuda.synchronize()
    say("[case] two streams at once")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(10):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got.append((k, sets[k][0]()))
    torch.cuda.synchronize()
    for k, outs in got:
        for a, b in zip(outs, want[k]):
            assert torch.equal(a, b)
