"""The fusion scorer's operators on the GPU where they were once wrong, each against a 64-bit form
or against the same call made again."""

import numpy as np
import pytest
import torch

import paper_2603_14002_amd as lbm
from tests import scorer_ref as ref
from tests.gpu_util import say
from tests.test_gpu_scorer import DT, bounds, close, dev, handles, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    lbm.lib()


# ------------------------------------------------------------------ attention in bf16

BF16 = [  # new, length, page, q heads, kv heads, D, window: each of the kernels, and the parts' join
    ([1, 3], [200, 40], 16, 8, 2, 64, 0),
    ([1], [1500], 64, 4, 1, 128, 0),
    ([2], [400], 32, 2, 1, 256, 90),
    ([1] * 530, [1 + i % 40 for i in range(530)], 16, 4, 4, 64, 0),
    ([650], [700], 16, 128, 8, 64, 0),
    ([310, 300], [330, 333], 64, 128, 4, 128, 90),
    ([305], [306], 128, 256, 2, 256, 0),
]


@pytest.mark.parametrize("case", range(len(BF16)))
def test_attend_bf16_rounds_the_output_alone(case):
    """With bf16 activations an output is off by its own rounding to bf16, and beside that by no more than 2^-16 of
    the probabilities (two pieces of 8 significant bits) and the 32-bit sums' errors."""
    new, length, P, Hq, H, D, window = BF16[case]
    say(f"[case] attend bf16 {case}")
    rng = np.random.default_rng(500 + case)
    R = ref.Ragged(new, length, P, H, D, seed=case)
    for s, n in enumerate(length):
        R.put(s, randn(rng, n, H, D, dtype=torch.float64) + 2 * randn(rng, 1, H, D, dtype=torch.float64), randn(rng, n, H, D, dtype=torch.float64))
    q = dev(randn(rng, R.n_rows, Hq, D, dtype=torch.bfloat16))
    cache, batch = handles(R)
    out, _ = lbm.lb_kv_attend(cache, batch, q, D ** -0.5, window=window)
    m = 0
    for s, n in enumerate(new):
        if s < 4 or s % 40 == 0:
            k, v = R.get(s, length[s])
            want, _, mass, reach = ref.attend(q.cpu()[m:m + n].double(), k, v, D ** -0.5, length[s] - n, window)
            # scores summed in 32 bits over D channels move a probability by twice their error; the exponential's and
            # the sums' own roundings; the output's half step on top
            delta = (D + 8) * 2.0 ** -23 * reach + 2.0 ** -21 * (1 + reach)
            rest = (2.0 ** -16 + 4 * delta + length[s] * 2.0 ** -24).unsqueeze(-1) * mass
            close(out[m:m + n], want, ref.EPS[torch.bfloat16] * (want.abs() + rest) + rest, f"sequence {s}")
        m += n


# ------------------------------------------------------------------ batches whose max_new is a loose bound


def filled(R, rng, shared=False):
    """R with keys and values for all tokens (shared: the same ones for every sequence)."""
    most = max(R.length)
    k, v = (randn(rng, most, R.H, R.D, dtype=torch.float64) for _ in range(2))
    for s, n in enumerate(R.length):
        if not shared:
            k, v = (randn(rng, n, R.H, R.D, dtype=torch.float64) for _ in range(2))
        R.put(s, k[:n], v[:n])
    return R


def check_some(R, q, out, lse, scale, window, which):
    at = np.cumsum([0] + R.new)
    for s in which:
        m, n = int(at[s]), R.new[s]
        if n == 0:
            continue
        k, v = R.get(s, R.length[s])
        want, wl, mass, reach = ref.attend(q.cpu()[m:m + n].double(), k, v, scale, R.length[s] - n, window)
        b, bl = bounds(want, wl, mass, reach, q.dtype, R.D, R.length[s])
        close(out[m:m + n], want, b, f"sequence {s}")
        close(lse[m:m + n], wl, bl, f"lse of sequence {s}")


def batch_of(R, max_new):
    word = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    cache = lbm.KVCache(dev(R.pages), R.P, R.H, R.D, flags=word)
    return cache, lbm.KVBatch(dev(R.starts), dev(R.lengths), dev(R.table), R.n_rows, max_new)


@pytest.mark.parametrize("seqs,heads,max_new,window", [(8192, 8, 8192, 0), (600, 3, 300, 5), (70, 2, 1 << 20, 0), (3, 1, 3, 0)])
def test_attend_single_tokens_under_a_loose_bound(seqs, heads, max_new, window):
    """max_new is a bound: a large one gives what the exact one gives, bit for bit where no key range has parts."""
    say(f"[case] loose {seqs} {heads} {max_new}")
    rng = np.random.default_rng(40)
    R = filled(ref.Ragged([1] * seqs, [1 + i % 23 for i in range(seqs)], 16, heads, 64, seed=41), rng, shared=True)
    q = dev(randn(rng, seqs, heads, 64, dtype=torch.bfloat16))
    exact = lbm.lb_kv_attend(*batch_of(R, 1), q, 0.3, window=window, want_lse=True)
    cache, batch = batch_of(R, max_new)
    loose = lbm.lb_kv_attend(cache, batch, q, 0.3, window=window, want_lse=True)
    assert cache.status() == 0
    for a, b in zip(exact, loose):
        assert torch.equal(a, b)
    check_some(R, q, *loose, 0.3, window, range(0, seqs, max(1, seqs // 40)))


@pytest.mark.parametrize("new,length,P,Hq,H,D,window,t", [
    ([1] * 40 + [200, 0, 3], [5 + i for i in range(40)] + [260, 9, 70], 16, 8, 2, 64, 0, "bf16"),
    ([200] + [1] * 7, [300] + [3000 + i for i in range(7)], 64, 2, 2, 128, 0, "f32"),          # parts of the keys
    ([90, 0, 0, 1, 1, 1, 17, 1], [90, 0, 40, 1100, 2, 1, 17, 1200], 32, 4, 1, 256, 50, "f16"),  # parts, empty sequences
    ([1] * 1500 + [33], [1 + i % 30 for i in range(1500)] + [500], 16, 16, 4, 64, 0, "bf16"),   # jobs by wavefront
    ([0] * 20 + [100] + [0] * 20, [3] * 20 + [120] + [7] * 20, 16, 1, 1, 128, 0, "bf16"),
])
def test_attend_short_sequences_beside_a_long_one(new, length, P, Hq, H, D, window, t):
    say(f"[case] mixed {len(new)} {Hq} {H} {D}")
    rng = np.random.default_rng(42)
    R = filled(ref.Ragged(new, length, P, H, D, seed=43, pad_rows=2), rng, shared=len(new) > 100)
    q = dev(randn(rng, R.n_rows, Hq, D, dtype=DT[t]))
    cache, batch = batch_of(R, max(new))
    out = torch.full((R.n_rows, Hq, D), 7.0, dtype=DT[t], device="cuda:0")
    lse = torch.full((R.n_rows, Hq), 7.0, device="cuda:0")
    lbm.lb_kv_attend(cache, batch, q, D ** -0.5, window=window, out=out, lse=lse)
    assert cache.status() == 0
    assert bool((out[sum(new):] == 7.0).all()) and bool((lse[sum(new):] == 7.0).all())
    which = list(range(len(new))) if len(new) < 100 else list(range(0, len(new), 37)) + [len(new) - 1]
    check_some(R, q, out, lse, D ** -0.5, window, which)


def test_attend_mixed_batches_report_starts_and_lengths_that_do_not_fit():
    """Flagged whichever sequence it is; where the starts are in order, the other sequences get theirs, and no row
    outside the sequences is written."""
    rng = np.random.default_rng(44)
    new, length = [1] * 30 + [40] + [1] * 9, [20] * 30 + [60] + [30] * 9
    R = filled(ref.Ragged(new, length, 16, 1, 64, seed=45, pad_rows=3), rng)
    q = dev(randn(rng, R.n_rows, 2, 64))
    n, S = sum(new), len(new)

    def run(starts=None, lengths=None):
        T = ref.Ragged(new, length, 16, 1, 64, seed=45, pad_rows=3)
        T.pages = R.pages
        if starts is not None:
            T.starts = torch.tensor(starts, dtype=torch.int32)
        if lengths is not None:
            T.lengths = torch.tensor(lengths, dtype=torch.int32)
        cache, batch = batch_of(T, 40)
        out, lse = torch.full((R.n_rows, 2, 64), 7.0, device="cuda:0"), torch.full((R.n_rows, 2), 7.0, device="cuda:0")
        lbm.lb_kv_attend(cache, batch, q, 0.2, out=out, lse=lse)
        return out, lse, cache.status()

    say("[case] mixed, bad starts and lengths")
    out, lse, st = run()
    assert st == 0
    check_some(R, q, out, lse, 0.2, 0, range(S))
    good = R.starts.tolist()
    for s in (0, 7, 30, S - 1):
        for value in (-1, 10 ** 9):
            bad = list(length)
            bad[s] = value
            o, l, st = run(lengths=bad)
            rest = [i for i in range(R.n_rows) if not good[s] <= i < good[s + 1]]
            assert st & lbm.LB_KV_BAD_LENGTH  # beside it LB_KV_BAD_PAGE, where the length reaches the table's end
            assert torch.equal(o[rest], out[rest]) and torch.equal(l[rest], lse[rest])
    # the last sequences past the rows
    o, l, st = run(starts=good[:-1] + [R.n_rows + 5])
    assert st == lbm.LB_KV_BAD_LENGTH and torch.equal(o[:n - 1], out[:n - 1])
    # out of order, far outside
    for s, value in ((1, -5), (20, -2 ** 31), (20, 2 ** 31 - 1), (31, 2), (0, 9), (S, 3)):
        starts = list(good)
        starts[s] = value
        o, l, st = run(starts=starts)
        assert st & lbm.LB_KV_BAD_LENGTH
        assert bool(torch.isfinite(o).all())
    zero = run(starts=[0] * (S + 1))
    assert zero[2] == 0 and bool((zero[0] == 7.0).all()) and bool((zero[1] == 7.0).all())


# ------------------------------------------------------------------ adapters


def test_lora_rows_past_one_launch():
    """2^27 rows and more are several launches: the rows are those of a call on each half."""
    half = 2 ** 26 + 16
    rows = 2 * half
    say("[case] lora 2^27 rows")
    g = torch.Generator(device="cuda:0").manual_seed(50)
    x, y = (torch.randn(rows, 8, generator=g, device="cuda:0", dtype=torch.bfloat16) for _ in range(2))
    a, b = (torch.randn(3, 8, 8, generator=g, device="cuda:0", dtype=torch.bfloat16) for _ in range(2))
    adapter = torch.randint(-1, 3, (rows,), generator=g, device="cuda:0", dtype=torch.int32)
    out = torch.empty_like(y)
    lbm.lb_lora_add(y, x, a, b, adapter, out=out)
    for at in (0, 16 * (2 ** 23 - 1) - 8, rows - 30):
        rest = slice(at, at + 30)
        ids = adapter[rest].long()
        h = torch.bmm(a.float()[ids.clamp_min(0)], x[rest].float().unsqueeze(2))
        add = torch.bmm(b.float()[ids.clamp_min(0)], h).squeeze(2)
        want = y[rest].float() + torch.where(ids[:, None] >= 0, add, 0.0)
        # the output's half step; sums of 8 terms in 32 bits and h in two pieces (2^-16) within |b| |a| |x|
        size = torch.bmm(b.float().abs()[ids.clamp_min(0)], torch.bmm(a.float().abs()[ids.clamp_min(0)], x[rest].float().abs().unsqueeze(2))).squeeze(2)
        close(out[rest], want.cpu().double(), (ref.EPS[torch.bfloat16] * want.abs() + 2.0 ** -14 * size).cpu().double(), f"rows {at}")
    for part in (slice(0, half), slice(half, rows)):
        lbm.lb_lora_add(y[part], x[part], a, b, adapter[part])  # in place
    assert torch.equal(out, y)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d,r", [(8, 512, 16), (40, 1024, 8), (256, 264, 8), (20, 512, 64), (600, 272, 16)])
def test_lora_over_its_own_input(rows, d, r, t):
    """x is y, or lies across the result: as if x had been copied first, in one launch's sizes and in two's."""
    say(f"[case] lora over x {rows} {d} {r} {t}")
    rng = np.random.default_rng(51)
    dt = DT[t]
    wide = dev(randn(rng, rows, 2 * d, dtype=dt))
    a, b = dev(randn(rng, 5, r, d, dtype=dt) * 0.1), dev(randn(rng, 5, d, r, dtype=dt) * 0.1)
    adapter = dev(torch.from_numpy(rng.integers(-1, 5, rows).astype(np.int32)))
    for off in (0, 8, d - 8, d):  # out lies `off` channels into x: the same, overlapping, beside it
        apart = lbm.lb_lora_add(wide[:, off:off + d].clone(), wide[:, :d].clone(), a, b, adapter)
        for _ in range(8):
            one = wide.clone()
            lbm.lb_lora_add(one[:, off:off + d], one[:, :d], a, b, adapter)
            # one launch sums h's parts of 4 wavefronts, two of 8: the same up to 32-bit sums' order
            bound = 2.0 ** -20 * apart.abs().amax() + 2 * ref.EPS[dt] * apart.abs()
            close(one[:, off:off + d], apart.cpu().double(), bound.cpu().double(), f"offset {off}")
            assert torch.equal(one[:, off + d:], wide[:, off + d:]) and torch.equal(one[:, :off], wide[:, :off])
    # rows over other rows
    tall = dev(randn(rng, rows + 16, d, dtype=dt))
    for x0, y0 in ((0, 16), (16, 0)):
        apart = lbm.lb_lora_add(tall[y0:y0 + rows].clone(), tall[x0:x0 + rows].clone(), a, b, adapter)
        one = tall.clone()
        lbm.lb_lora_add(one[y0:y0 + rows], one[x0:x0 + rows], a, b, adapter)
        bound = 2.0 ** -20 * apart.abs().amax() + 2 * ref.EPS[dt] * apart.abs()
        close(one[y0:y0 + rows], apart.cpu().double(), bound.cpu().double(), f"rows {x0} {y0}")


# ------------------------------------------------------------------ logits


@pytest.mark.parametrize("R,C,H,W,t", [(64, 125002, 300, 200, "bf16"), (1, 125002, 3000, 1000, "f32"), (400, 700, 60, 68, "f32"), (5, 20000, 1, 4095, "f16")])
def test_logits_of_long_rows_repeat_bit_for_bit(R, C, H, W, t):
    """The named classes are added in an order that does not depend on which wavefront came first."""
    say(f"[case] repeat {R} {C}")
    rng = np.random.default_rng(60)
    x = dev((3 * randn(rng, R, C)).to(DT[t]))
    x += 4.0  # most of a row's sum can lie in the named classes
    rules = lbm.LogitRules(temperature=0.9, repetition=1.1, presence=0.1, frequency=0.1,
                           history=dev(torch.from_numpy(rng.integers(0, C, (R, H)).astype(np.int32))),
                           bias_ids=dev(torch.from_numpy(rng.integers(0, C, (R, W)).astype(np.int32))),
                           bias_values=dev(randn(rng, R, W) + 9))
    first = None
    for _ in range(60):
        logp, _, lse = lbm.lb_logits_adjust(x, rules)
        if first is None:
            first = logp, lse
        assert torch.equal(lse, first[1]) and torch.equal(logp, first[0])


# ------------------------------------------------------------------ the largest numbers of a type


def test_attend_queries_of_the_lowest_value():
    """fp32 queries past bf16's largest number are finite: 0 times one is 0, and a small key's score is what 32 bits give."""
    rng = np.random.default_rng(70)
    low = torch.finfo(torch.float32).min
    for new, length in ((1, 50), (1, 1500), (300, 320)):
        say(f"[case] lowest queries {new} {length}")
        R = ref.Ragged([new], [length], 16, 4, 64, seed=71)
        k, v = randn(rng, length, 4, 64, dtype=torch.float64), randn(rng, length, 4, 64, dtype=torch.float64)
        k[:, :, 3:5] = 0.0
        k[:, 1, 32:] = 0.0
        k[:, 1, 40] = torch.randint(0, 2, (length,)).double() * 2.0 ** -124  # scores 0 and about 2
        R.put(0, k, v)
        k, v = R.get(0, length)
        q = randn(rng, new, 256, 64)
        q[:, :, 3], q[:, :, 4] = low, -low
        q[:, 64:128, 40] = -low
        cache, batch = handles(R)
        out, lse = lbm.lb_kv_attend(cache, batch, dev(q), 0.125, want_lse=True)
        want, wl, _, reach = ref.attend(q.double(), k, v, 0.125, length - new, 0)
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
        b, bl = bounds(want, wl, *ref.attend(q.double(), k, v, 0.125, length - new, 0)[2:], torch.float32, 64, length)
        close(out, want, b, "out")
        close(lse, wl, bl, "lse")


@pytest.mark.parametrize("rank,rows,d_out", [(16, 3, 32), (32, 3, 32), (64, 20, 264), (128, 300, 40), (16, 300, 40)])
def test_lora_products_past_the_largest_bf16(rank, rows, d_out):
    """h = 2^128 - 2^118 is a finite 32-bit number that would round to an infinity in bf16: the result is 255.75 in each
    channel, 256 in bf16, and its negative."""
    say(f"[case] lora largest {rank} {rows}")
    x = torch.zeros(rows, 64, dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = 2.0 ** 127 * (2 - 2.0 ** -7), 1.5 * 2.0 ** 119
    a = torch.zeros(2, rank, 64, dtype=torch.bfloat16)
    a[0, 3, :2], a[1, rank - 1, :2] = 1.0, -1.0
    b = torch.full((2, d_out, rank), 2.0 ** -120, dtype=torch.bfloat16)
    y = torch.zeros(rows, d_out, dtype=torch.bfloat16)
    ids = torch.arange(rows, dtype=torch.int32) % 2
    out = lbm.lb_lora_add(*(dev(t) for t in (y, x, a, b, ids))).cpu().double()
    assert torch.equal(out, torch.where(ids[:, None] == 0, 256.0, -256.0).double().expand_as(out))


# ------------------------------------------------------------------ batches that do not fit


FAULTS = {  # of two sequences of 2 new tokens, 20 and 30 in all, one of 4 rows
    "none": {}, "page below": dict(page=-1), "page past": dict(page=6), "page far past": dict(page=2 ** 31 - 1), "page far below": dict(page=-2 ** 31),
    "length past the table": dict(length=33), "length far past": dict(length=10 ** 9), "length below 0": dict(length=-1),
    "length below the new tokens": dict(length=1), "length 0": dict(length=0), "starts past the rows": dict(starts=[0, 2, 9]),
    "one sequence has all rows": dict(starts=[0, 4, 4]), "angles": dict(positions=29), "few angles": dict(positions=19), "max_new": dict(max_new=1),
}


@pytest.mark.parametrize("fault", list(FAULTS))
@pytest.mark.parametrize("D,t", [(64, "f32"), (128, "bf16")])
def test_append_and_attend_where_a_batch_does_not_fit(fault, D, t):
    """Every byte of the pool after an append, and what attention gives after it, for the sequence that does not fit and
    for the one that does."""
    f = FAULTS[fault]
    say(f"[case] faults {fault} {D}")
    rng = np.random.default_rng(80)
    R = ref.Ragged([2, 2], [20, 30], 16, 1, D, seed=6)
    assert R.n_pages == 6
    for s in range(2):
        R.put(s, randn(rng, R.length[s], 1, D, dtype=torch.float64), randn(rng, R.length[s], 1, D, dtype=torch.float64))
    k, v, q = (randn(rng, 4, 1, D, dtype=DT[t]) for _ in range(3))
    if "page" in f:
        R.table[0, 1] = f["page"]
    if "length" in f:
        R.lengths[0] = f["length"]
    if "starts" in f:
        R.starts[:] = torch.tensor(f["starts"], dtype=torch.int32)
    max_new = f.get("max_new", 4 if "starts" in f else 2)
    cache, batch = batch_of(R, max_new)
    positions = f.get("positions", 40)
    cos, sin = lbm.lb_rope_table(positions, 16)
    rope = lbm.Rope(dev(cos), dev(sin))
    # what the header says of it: (sequence, row, position) of the tokens there are, and the keys and values that go in
    length = [min(max(int(x), 0), R.table.shape[1] * 16) for x in R.lengths]
    rows = []
    for s in range(2):
        a, z = (min(max(int(x), 0), 4) for x in R.starts[s:s + 2])
        rows += [(s, a + i, length[s] - (z - a) + i) for i in range(min(z - a, max_new))]
    q_out = torch.full((4, 1, D), 7.0, dtype=DT[t], device="cuda:0")
    lbm.lb_kv_append(cache, batch, dev(q), dev(k), dev(v), rope=rope, q_out=q_out)
    pool = ref.Ragged([2, 2], [20, 30], 16, 1, D, seed=6)
    pool.pages = R.pages.clone()
    turned = set()
    for s, row, p in rows:
        if not 0 <= p < positions:
            continue
        turned.add(row)
        page = int(R.table[s, p // 16])
        if not 0 <= page < R.n_pages:
            continue
        pool.table = torch.full((1, p // 16 + 1), page, dtype=torch.int32)
        kr = ref.rotate(k[row:row + 1].double(), cos[p:p + 1], sin[p:p + 1], False)
        # put() writes from token 0 on: the one token goes in by way of a pool whose others are its own
        tokens = [ref.Ragged.get(pool, 0, p + 1, pool.pages)[i] for i in range(2)]
        before = pool.pages.clone()
        pool.put(0, torch.cat([tokens[0][:p], kr]).nan_to_num(0), torch.cat([tokens[1][:p], v[row:row + 1].double()]).nan_to_num(0))
        after = pool.pages
        pool.pages = before
        slot, P = p % 16, 16
        at = torch.cat([slot * (D // 2) + torch.arange(D // 2), P * D // 2 + ((slot // 4) * (D // 2) + torch.arange(D // 2)) * 4 + slot % 4,
                        P * D + slot * (D // 32) + torch.arange(D // 32),
                        P * D + P * D // 32 + ((slot // 4) * (D // 32) + torch.arange(D // 32)) * 4 + slot % 4])
        pool.pages[page][:, at] = after[page][:, at]
    assert torch.equal(cache.pages.cpu(), pool.pages)
    assert all(bool((q_out[i] == 7.0).all()) == (i not in turned) for i in range(4))
    bits = 0
    if "page" in f:
        bits = lbm.LB_KV_BAD_PAGE
    elif f and fault not in ("one sequence has all rows",):
        bits = lbm.LB_KV_BAD_LENGTH
    # (a length past the table is cut to the table, whose last entry here may be no page)
    assert cache.status() & ~lbm.LB_KV_BAD_PAGE == bits & ~lbm.LB_KV_BAD_PAGE and cache.status() & bits == bits
    cache.flags.zero_()
    out, lse = torch.full((4, 1, D), 7.0, dtype=DT[t], device="cuda:0"), torch.full((4, 1), 7.0, device="cuda:0")
    lbm.lb_kv_attend(cache, batch, dev(q), 0.3, out=out, lse=lse)
    R.pages = pool.pages
    for s, row, p in rows:
        seen = [x for x in range(min(p, length[s] - 1) + 1) if 0 <= int(R.table[s, x // 16]) < R.n_pages]
        if not seen:
            assert bool((out[row] == 0).all()) and bool((lse[row] == -float("inf")).all())
            continue
        if any(x >= R.length[s] and (s, x) not in {(a, c) for a, _, c in rows} for x in seen):
            continue  # of the pool's garbage, whose scales may be none that an append writes
        pool.table = R.table[s:s + 1].clamp(0, R.n_pages - 1)
        kk, vv = (x[seen] for x in ref.Ragged.get(pool, 0, max(seen) + 1, R.pages))
        want, wl, mass, reach = ref.attend(q[row:row + 1].double(), kk, vv, 0.3, len(seen) - 1, 0)
        b, bl = bounds(want, wl, mass, reach, DT[t], D, len(seen))
        close(out[row:row + 1], want, b, f"row {row}")
        close(lse[row:row + 1], wl, bl, f"lse of row {row}")
    have = {row for _, row, _ in rows}
    assert all(bool((out[i] == 7.0).all()) and bool((lse[i] == 7.0).all()) for i in range(4) if i not in have)


@pytest.mark.parametrize("C", [41, 700, 30000])
def test_logits_of_minus_infinity_beside_nan(C):
    """A class without probability keeps -infinity where the rest of its row is NaN."""
    x = torch.zeros(3, C)
    x[0, 3], x[0, 7], x[1, 7], x[2, 3] = float("nan"), -float("inf"), -float("inf"), float("nan")
    got, score, lse = lbm.lb_logits_adjust(dev(x), target=dev(torch.tensor([7, 7, 0], dtype=torch.int32)))
    say(f"[case] logits -inf beside nan {C}")
    assert got[0, 7] == -float("inf") and got[1, 7] == -float("inf") and score[0] == -float("inf") and score[1] == -float("inf")
    assert int(torch.isnan(got[0]).sum()) == C - 1 and bool(torch.isnan(got[2]).all()) and bool(torch.isnan(score[2]))
    assert torch.isnan(lse).tolist() == [True, False, True] and bool(torch.isfinite(got[1, :7]).all())


def test_logits_with_the_longest_lists():
    """4096 ids on the longest part of a row: as with the lists' last biases and counts put in by hand."""
    say("[case] logits longest lists")
    rng = np.random.default_rng(90)
    C = 131072
    for R in (1, 600):  # parts of a row, and a row in one
        x = dev(randn(rng, R, C))
        past, ids = (torch.from_numpy(rng.integers(0, C, (1, 2048)).astype(np.int32)) for _ in range(2))
        values = randn(rng, 1, 2048)
        on = lbm.LogitRules(history=dev(past.expand(R, -1).contiguous()), presence=0.5, frequency=0.25, bias_ids=dev(ids), bias_values=dev(values))
        got, _, lse = lbm.lb_logits_adjust(x, on)
        z = x.double()
        counts = torch.bincount(past[0].long(), minlength=C).double()
        bias = torch.zeros(C, dtype=torch.float64)
        for w, b in zip(ids[0].tolist(), values[0].tolist()):
            bias[w] = b
        z += dev(bias - 0.5 * (counts > 0) - 0.25 * counts)
        want = torch.logsumexp(z, 1)
        # four roundings of the rules on values below 16, and sums of 2 C / 256 + 64 positive terms
        bound = 6 * 2.0 ** -24 * 64 + (2 * C / 256 + 64) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -22 * float(want.max())
        close(lse, want.cpu(), bound, "lse")
        close(got[0], (z - want[:, None])[0].cpu(), 2 * bound, "logprobs")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_attend_infinite_queries(t):
    """Scores of plus infinity make a row NaN, and so does a NaN; with minus infinity throughout a row is as one that
    sees nothing.  No other row has any of it."""
    inf = float("inf")
    for new, length in ((1, 50), (1, 1500), (310, 320)):
        say(f"[case] infinite queries {t} {new} {length}")
        rng = np.random.default_rng(74)
        R = ref.Ragged([new, 1], [length, 20], 16, 4, 64, seed=75)
        k, v = randn(rng, length, 4, 64, dtype=torch.float64), randn(rng, length, 4, 64, dtype=torch.float64)
        k[:, :, 2] = 1.0
        R.put(0, k, v)
        R.put(1, k[:20], v[:20])
        q = randn(rng, new + 1, 256, 64, dtype=DT[t])
        q[0, 0, 2], q[0, 64, 2], q[0, 128, 2] = inf, -inf, float("nan")  # heads 0, 64, 128: KV heads 0, 1, 2
        cache, batch = handles(R)
        out, lse = lbm.lb_kv_attend(cache, batch, dev(q), 0.125, want_lse=True)
        assert bool(torch.isnan(out[0, 0]).all()) and bool(torch.isnan(out[0, 128]).all())
        assert not bool(torch.isfinite(lse[0, [0, 64, 128]]).any())
        assert bool((out[0, 64] == 0).all()) and lse[0, 64] == -inf
        out[0, [0, 64, 128]] = 0.0
        lse[0, [0, 64, 128]] = 0.0
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("long", [40, 1500])
def test_attend_loose_batches_captured_and_replayed(long):
    """A graph captured under a bound serves other sequences of the same tensors: each replay is the eager call."""
    say(f"[case] loose graph {long}")
    rng = np.random.default_rng(46)
    S = 30
    R = filled(ref.Ragged([1] * S, [20] * (S - 2) + [long, long], 16, 2, 64, seed=47, pad_rows=50), rng)
    cache, batch = batch_of(R, 64)
    q = dev(randn(rng, R.n_rows, 4, 64))
    ws = torch.empty(max(16, lbm.lb_kv_attend_workspace(cache, batch, 4)), dtype=torch.uint8, device="cuda:0")
    out, lse = torch.zeros(R.n_rows, 4, 64, device="cuda:0"), torch.zeros(R.n_rows, 4, device="cuda:0")
    step = lambda: lbm.lb_kv_attend(cache, batch, q, 0.2, out=out, lse=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for new in ([1] * S, [0] * (S - 1) + [39], [2] * 20 + [0] * 9 + [19], [20] + [0] * 10 + [1] * 18 + [30], [0] * S):
        batch.starts.copy_(dev(torch.tensor(np.cumsum([0] + new).astype(np.int32))))
        results = []
        for run in (g.replay, step):
            out.fill_(7.0), lse.fill_(7.0)
            run()
            torch.cuda.synchronize()
            results.append((out.clone(), lse.clone()))
        for a, b in zip(*results):
            assert torch.equal(a, b) and bool((a[sum(new):] == 7.0).all())
        R.new = new
        check_some(R, q, *results[0], 0.2, 0, [s for s in range(S) if new[s]])
    assert cache.status() == 0


# ------------------------------------------------------------------ what lies before a window

WINDOWED = [  # new, length, page, q heads, kv heads, D, window, type: each of the kernels, and parts of the keys
    ([1, 1], [300, 77], 16, 4, 2, 64, 50, "f32"),
    ([1], [5000], 16, 4, 1, 128, 2100, "bf16"),
    ([3, 1], [200, 450], 32, 2, 1, 256, 33, "f16"),
    ([1] * 530, [100 + i % 300 for i in range(530)], 16, 4, 4, 64, 20, "bf16"),
    ([650], [900], 16, 128, 8, 64, 70, "bf16"),
    ([310, 300], [630, 433], 16, 128, 4, 128, 90, "f32"),
    ([305], [506], 32, 256, 2, 256, 100, "bf16"),
]


def windowed(case):
    """The case's tensors, and the first position of each sequence that some new token sees."""
    new, length, P, Hq, H, D, window, t = WINDOWED[case]
    rng = np.random.default_rng(600 + case)
    R = filled(ref.Ragged(new, length, P, H, D, seed=case), rng, shared=len(new) > 100)
    first = [max(0, ln - n - window + 1) for n, ln in zip(new, length)]
    return R, dev(randn(rng, R.n_rows, Hq, D, dtype=DT[t])), D ** -0.5, window, first


@pytest.mark.parametrize("case", range(len(WINDOWED)))
def test_attend_pages_before_the_window_may_be_gone(case):
    """A page of which no query sees a token need not be one, and is no fault of the data."""
    say(f"[case] window gone {case}")
    R, q, scale, window, first = windowed(case)
    cache, batch = handles(R)
    want = lbm.lb_kv_attend(cache, batch, q, scale, window=window, want_lse=True)
    assert cache.status() == 0
    for s, f in enumerate(first):
        R.table[s, :f // R.P] = -1 if s % 2 else R.n_pages + 7
    cache, batch = handles(R)
    got = lbm.lb_kv_attend(cache, batch, q, scale, window=window, want_lse=True)
    assert cache.status() == 0
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # a page that is seen in its last token alone is needed
    s = len(first) - 1
    if first[s]:
        R.table[s, first[s] // R.P] = -1
        cache, batch = handles(R)
        lbm.lb_kv_attend(cache, batch, q, scale, window=window)
        assert cache.status() == lbm.LB_KV_BAD_PAGE


@pytest.mark.parametrize("case", range(len(WINDOWED)))
def test_attend_tokens_before_the_window_have_no_effect(case):
    """Whatever bytes they hold, scales that stand for no number among them."""
    say(f"[case] window bytes {case}")
    R, q, scale, window, first = windowed(case)
    cache, batch = handles(R)
    want = lbm.lb_kv_attend(cache, batch, q, scale, window=window, want_lse=True)
    P, D = R.P, R.D
    for byte in (253, 254, 255):
        for s, f in enumerate(first):
            for x in range(max(0, f - 40), f):
                mem, slot = R.pages[int(R.table[s, x // P])], x % P
                mem[:, slot * (D // 2):(slot + 1) * (D // 2)] = 0x77
                mem[:, P * D // 2 + ((slot // 4) * (D // 2) + torch.arange(D // 2)) * 4 + slot % 4] = 0x77
                mem[:, P * D + slot * (D // 32):P * D + (slot + 1) * (D // 32)] = byte
                mem[:, P * D + P * D // 32 + ((slot // 4) * (D // 32) + torch.arange(D // 32)) * 4 + slot % 4] = byte
        cache, batch = handles(R)
        got = lbm.lb_kv_attend(cache, batch, q, scale, window=window, want_lse=True)
        for a, b in zip(want, got):
            assert torch.equal(a, b), byte
