"""What the fusion scorer's operators are measured on.

A caller of ``lb_decode_batch`` with an external scorer answers each fusion event with the
log-probabilities of word sequences.  The operators are those of such a scorer: keys and values
appended to a paged 4-bit cache with the position rotation on the way, attention over that cache,
low-rank adapters of many speakers beside a shared projection, and the rules that turn logits into
log-probabilities (over the words, or over the decoder's own 41 classes).

The cache holds blocks of 32 channels as e2m1 codes with a power of two as scale.  A page of P
tokens has, for each KV head, P*(D + D/16) bytes: key codes [P][D/2], value codes [P/4][D/2][4],
key scales [P][D/32], value scales [P/4][D/32][4]; a byte of codes holds an even channel in its low
half and the next one in its high half.

The shapes are those of the repository's workloads (1 to 1024 streams, up to 256 words a hypothesis,
125k words, the causal word LM's 256 channels in 4 heads) and generic ones of larger scorers.
"""

import math

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
REPETITION, PRESENCE, FREQUENCY = 1.3, 0.2, 0.1
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one live speaker's next word: the shapes of the repository's word LM, where only the call's own cost shows
        dict(name="append-live", op="append", seqs=1, new_lo=1, new_hi=1, ctx=40, q_heads=4, kv_heads=4, dim=64, page=16,
             rot=64, layout="half", stretch=1.0, dtype="fp32"),
        # the first words of ragged prompts behind a shared instruction, a quarter of each head rotated, long positions
        dict(name="append-prompt", op="append", seqs=12, new_lo=37, new_hi=4001, ctx=9000, q_heads=32, kv_heads=8, dim=128,
             page=64, rot=32, layout="interleaved", stretch=4.0, dtype="bf16"),
        # one speaker's next word over the words so far
        dict(name="attend-live", op="attend", seqs=1, new_lo=1, new_hi=1, len_lo=200, len_hi=200, q_heads=4, kv_heads=4,
             dim=64, page=16, window=0, dtype="fp32"),
        # a server's thousand live streams, one new word each
        dict(name="attend-streams", op="attend", seqs=1024, new_lo=1, new_hi=1, len_lo=3, len_hi=256, q_heads=4, kv_heads=4,
             dim=64, page=16, window=0, dtype="bf16"),
        # a few requests with a long history in front
        dict(name="attend-long", op="attend", seqs=4, new_lo=1, new_hi=1, len_lo=90_001, len_hi=131_072, q_heads=32,
             kv_heads=8, dim=128, page=64, window=0, dtype="bf16"),
        # ragged prompts, partly in the cache already
        dict(name="attend-prompt", op="attend", seqs=6, new_lo=65, new_hi=2048, len_lo=130, len_hi=4096, q_heads=32,
             kv_heads=8, dim=128, page=32, window=0, dtype="bf16"),
        # acoustic logits of a batch of utterances: a bonus on some classes, a temperature, to the decoder's log-probabilities
        dict(name="logits-classes", op="logits", rows=128_000, classes=41, history=0, biases=3, shared=True, masks=1,
             keep=1.0, scores=False, full=True, dtype="fp32"),
        # one next word: earlier words penalised, a speaker's own words favoured, what the grammar does not allow left out
        dict(name="logits-next", op="logits", rows=1, classes=125_002, history=48, biases=100, shared=False, masks=1,
             keep=0.3, scores=True, full=True, dtype="fp32"),
        # a fusion event: every word of the requested sequences scored, log-probabilities of the targets alone
        dict(name="logits-scoring", op="logits", rows=4096, classes=125_002, history=0, biases=64, shared=True, masks=2,
             keep=0.9, scores=True, full=False, dtype="bf16"),
        # a few live speakers, each with an adapter, beside the word LM's projection to queries, keys and values
        dict(name="lora-live", op="lora", rows=8, run=1, adapters=16, d_in=256, d_out=768, rank=16, dtype="fp32"),
        # many speakers in one step, each with an adapter of its own
        dict(name="lora-speakers", op="lora", rows=128, run=1, adapters=160, d_in=2048, d_out=8192, rank=64, dtype="fp16"),
        # prompts of some requests: runs of rows with one adapter, some requests without
        dict(name="lora-prompts", op="lora", rows=8192, run=300, adapters=24, d_in=4096, d_out=6144, rank=16, dtype="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend", "logits", "lora"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if op in ("append", "attend"):
        c["kv_heads"] = rng.choice([1, 2, 3, 4, 8])
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7])
        c["dim"] = rng.choice([64, 128, 128, 256])
        c["page"] = rng.choice([16, 32, 64, 128])
        c["seqs"] = log_int(1, 512)
        width = c["q_heads"] * c["dim"]
    if op == "append":
        c["new_hi"] = log_int(1, max(1, min(4000, 60_000_000 // (width * c["seqs"]))))
        c["new_lo"] = rng.randint(1, c["new_hi"])
        c["ctx"] = log_int(1, max(1, min(20_000, 1_000_000_000 // (c["seqs"] * c["kv_heads"] * c["dim"]))))
        c["rot"] = rng.choice([c["dim"], c["dim"] // 2, c["dim"] // 4, 16])
        c["layout"] = rng.choice(["half", "interleaved"])
        c["stretch"] = rng.choice([1.0, 2.0, 8.0])
    elif op == "attend":
        most = max(2, min(100_000, 250_000_000 // (c["seqs"] * c["kv_heads"] * c["dim"])))
        c["len_hi"] = log_int(1, most)
        c["len_lo"] = rng.randint(1, c["len_hi"])
        c["new_hi"] = 1
        if rng.random() < 0.5:  # several new tokens each: at most as many scores as the listed prompts have
            room = 400_000_000 // (c["seqs"] * c["q_heads"] * c["len_hi"])
            c["new_hi"] = log_int(1, max(1, min(c["len_lo"], room, 1500)))
        c["new_lo"] = rng.randint(1, c["new_hi"])
        c["window"] = rng.choice([0, 0, log_int(1, 5000)])
    elif op == "logits":
        c["classes"] = rng.choice([41, 41, log_int(2, 2000), log_int(2000, 130_000), 125_002])
        c["rows"] = log_int(1, max(1, min(100_000, 200_000_000 // c["classes"])))
        c["history"] = rng.choice([0, log_int(1, 300)])
        c["biases"] = rng.choice([0, log_int(1, min(200, c["classes"]))])
        c["shared"] = rng.random() < 0.5
        c["masks"] = rng.choice([0, 1, 5])
        c["keep"] = round(rng.uniform(0.05, 1.0), 2)
        c["full"] = rng.random() < 0.5
        c["scores"] = not c["full"] or rng.random() < 0.5
    else:
        c["d_in"], c["d_out"] = 8 * log_int(8, 700), 8 * log_int(8, 1000)
        c["rank"] = rng.choice([8, 16, 16, 24, 32, 64])
        c["rows"] = log_int(1, max(1, min(8000, 50_000_000 // max(c["d_in"], c["d_out"]))))
        c["run"] = log_int(1, 500)
        c["adapters"] = log_int(1, 128)
    return c


# ------------------------------------------------------------------ sizes of a case


def _spread(lo, hi, n):
    """n lengths from hi down to lo, evenly spread."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(c):
    """(new tokens, tokens in the cache with them) of each sequence, before the seed's order."""
    new = _spread(c["new_lo"], c["new_hi"], c["seqs"])
    if c["op"] == "append":
        return new, [c["ctx"] + n - (7 * i) % min(c["ctx"], 50) for i, n in enumerate(new)]
    return new, [max(a, b) for a, b in zip(new, _spread(c["len_lo"], c["len_hi"], c["seqs"]))]


def _visible(new, length, window):
    """Keys that the new tokens of a sequence see, over all of them, and the cached tokens that some of them see."""
    first = length - new
    if window == 0 or window >= length:
        return new * first + new * (new + 1) // 2, length
    pairs = sum(min(window, first + i + 1) for i in range(new))
    return pairs, min(length, new + window - 1)


def _adapter_runs(c):
    """An adapter (or -1) for each run of rows: neighbours differ, every ninth run has none."""
    runs = -(-c["rows"] // c["run"])
    return [-1 if i % 9 == 8 else (i * 7) % c["adapters"] for i in range(runs)]


def work(case):
    c = dict(case)
    size = 4 if c["dtype"] == "fp32" else 2
    if c["op"] in ("append", "attend"):
        new, length = _lengths(c)
        D, tokens = c["dim"], sum(new)
        held = D // 2 + D // 32  # bytes of one token's key or value of one head
        if c["op"] == "append":
            kv = tokens * c["kv_heads"]
            rows = tokens * (2 * c["q_heads"] + 4 * c["kv_heads"]) * D * size  # q read and written; k, v read, and written as held
            angles = tokens * c["rot"] * 4
            return {"bytes": rows + 4 * kv * held + angles, "flops": 3 * tokens * (c["q_heads"] + c["kv_heads"]) * c["rot"] + 8 * kv * D}
        seen = [_visible(n, ln, c["window"]) for n, ln in zip(new, length)]
        read = 2 * held * c["kv_heads"] * sum(s for _, s in seen)
        rows = tokens * c["q_heads"] * (2 * D * size + 4)
        return {"bytes": read + rows + 4 * sum(-(-ln // c["page"]) for ln in length),
                "flops": 4 * D * c["q_heads"] * sum(p for p, _ in seen)}
    if c["op"] == "logits":
        n = c["rows"] * c["classes"]
        extra = c["rows"] * 8 + (1 if c["shared"] else c["rows"]) * c["biases"] * 8 + c["rows"] * c["history"] * 4
        return {"bytes": n * (size + (4 if c["full"] else 0)) + extra + c["masks"] * -(-c["classes"] // 32) * 4, "flops": 8 * n}
    used = {a for a in _adapter_runs(c) if a >= 0}
    rows = c["rows"] * (c["d_in"] + 2 * c["d_out"]) * size
    with_one = sum(min(c["run"], c["rows"] - i * c["run"]) for i, a in enumerate(_adapter_runs(c)) if a >= 0)
    return {"bytes": rows + len(used) * c["rank"] * (c["d_in"] + c["d_out"]) * size + 4 * c["rows"],
            "flops": 2 * with_one * c["rank"] * (c["d_in"] + c["d_out"])}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def randint(hi, *shape):
        return torch.randint(hi, shape, generator=g, device="cuda")

    s = {"case": c}
    if c["op"] in ("append", "attend"):
        new, length = _lengths(c)
        order = torch.randperm(c["seqs"], generator=g, device="cuda").tolist()
        new, length = [new[i] for i in order], [length[i] for i in order]
        P, D, H = c["page"], c["dim"], c["kv_heads"]
        per = -(-max(length) // P)
        counts = torch.tensor([-(-ln // P) for ln in length], device="cuda")
        used = int(counts.sum())
        place = torch.randperm(used + 3, generator=g, device="cuda")[:used]
        first = torch.cumsum(counts, 0) - counts
        col = torch.arange(per, device="cuda")
        live = col[None] < counts[:, None]
        table = torch.where(live, place[(first[:, None] + col[None]).clamp_max(used - 1)], -1)
        s["pages"] = torch.randint(256, (used + 3, H, P * (D + D // 16)), generator=g, device="cuda", dtype=torch.uint8)
        s["table"] = table.to(torch.int32)
        s["lengths"] = torch.tensor(length, dtype=torch.int32, device="cuda")
        s["starts"] = torch.tensor([0] + new, dtype=torch.int32, device="cuda").cumsum(0).to(torch.int32)
        s["new"], s["most"] = sum(new), max(new)
        offset = 2 * randn(H, D).to(dt)  # keys have channels that are large for every token
        if c["op"] == "append":
            packed = randn(s["new"], (c["q_heads"] + 2 * H) * D).to(dt)  # as a projection to q, k and v leaves them
            q, k, v = packed.split([c["q_heads"] * D, H * D, H * D], dim=1)
            k += offset.view(1, -1)
            s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, D)) for t in (q, k, v))
            half = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
            angle = torch.arange(max(length), dtype=torch.float64, device="cuda")[:, None] / c["stretch"] * 10_000.0 ** (-2 * half / c["rot"])
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        else:
            s["q"] = randn(s["new"], c["q_heads"], D).to(dt)
            # what earlier steps appended; the ends of the last pages and the spare pages stay as they were
            blocks = s["pages"].view(used + 3, H, P * (D + D // 16))
            at = torch.arange(used * P, device="cuda")
            page, slot = place[at // P], at % P
            inside = (s["lengths"][:, None] - P * col[None])[live]  # tokens in each page, or more
            kept = slot < inside[at // P]
            page, slot = page[kept], slot[kept]
            for h in range(H):
                for which in (0, 1):
                    x = torch.randn(page.numel(), D, generator=g, device="cuda")
                    x = (x + 2 * torch.randn(1, D, generator=g, device="cuda")) if which == 0 else x
                    codes, scales = _pack(x.to(torch.bfloat16))
                    pair, group = torch.arange(D // 2, device="cuda")[None], torch.arange(D // 32, device="cuda")[None]
                    t = slot[:, None]
                    if which == 0:
                        code_at, scale_at = t * (D // 2) + pair, P * D + t * (D // 32) + group
                    else:
                        code_at = P * D // 2 + ((t // 4) * (D // 2) + pair) * 4 + t % 4
                        scale_at = P * D + P * D // 32 + ((t // 4) * (D // 32) + group) * 4 + t % 4
                    blocks[page[:, None], h, code_at] = codes
                    blocks[page[:, None], h, scale_at] = scales
        return s
    if c["op"] == "logits":
        R, C = c["rows"], c["classes"]
        s["logits"] = (3.0 * randn(R, C)).to(dt)
        s["temperature"] = 1.25 if c["full"] else 1.0
        rows = 1 if c["shared"] else R
        if c["history"]:
            h = (C * torch.rand(R, c["history"], generator=g, device="cuda").square()).to(torch.int32)
            kept = torch.arange(c["history"], device="cuda")[None] < randint(c["history"] + 1, R, 1)
            s["history"] = torch.where(kept, h, -1)
        if c["biases"]:
            ids = torch.rand(rows, min(C, 4096), generator=g, device="cuda").argsort(1)[:, :c["biases"]] * max(1, C // 4096)
            s["bias_ids"], s["bias_values"] = ids.to(torch.int32), 2.0 * randn(rows, c["biases"])
        if c["masks"]:
            words = -(-C // 32)
            bits = (torch.rand(c["masks"], words * 32, generator=g, device="cuda") < c["keep"]).view(-1, words, 32).long()
            packed = (bits << torch.arange(32, device="cuda")).sum(2)
            s["mask"] = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
            s["mask_row"] = randint(c["masks"], R).to(torch.int32)
        if c["scores"]:
            s["target"] = randint(C, R).to(torch.int32)
        return s
    s["x"] = randn(c["rows"], c["d_in"]).to(dt)
    s["y"] = randn(c["rows"], c["d_out"]).to(dt)
    s["a"] = (randn(c["adapters"], c["rank"], c["d_in"]) / math.sqrt(c["d_in"])).to(dt)
    s["b"] = (randn(c["adapters"], c["d_out"], c["rank"]) / math.sqrt(c["rank"])).to(dt)
    s["scale"] = 1.0 + torch.rand(c["adapters"], generator=g, device="cuda")
    names = torch.randperm(c["adapters"], generator=g, device="cuda").tolist()
    runs = [names[a] if a >= 0 else -1 for a in _adapter_runs(c)]
    s["adapter"] = torch.tensor(runs, dtype=torch.int32, device="cuda").repeat_interleave(c["run"])[:c["rows"]].contiguous()
    return s


# ------------------------------------------------------------------ the plain forms


def _pack(x):
    """Codes [n, D/2] and scale bytes [n, D/32] of x [n, D]."""
    x = x.double()
    n, D = x.shape
    blocks = x.view(n, D // 32, 32)
    m, p = torch.frexp(blocks.abs().amax(2))  # a = m 2^p, m in [0.5, 1)
    e = torch.where(m <= 0.75, p - 3, p - 2).clamp(-124, 125)
    e = torch.where(m == 0, torch.full_like(e, -124), e)
    y = torch.ldexp(blocks, -e[..., None].double()).view(n, D)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)).to(torch.uint8)
    code = code | (y < 0).to(torch.uint8) << 3
    return code[:, 0::2] | code[:, 1::2] << 4, (e + 127).to(torch.uint8)


def _unpack(codes, scales):
    """Values [..., D] of codes [..., D/2] and scale bytes [..., D/32], in 32 bits."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    scale = torch.exp2(scales.float() - 127)
    scale = torch.where(scales == 255, torch.full_like(scale, math.nan), scale)
    return level[both.int()] * scale.repeat_interleave(32, -1)


def _rotate(x, cos, sin, layout):
    """x [n, heads, D] in 64 bits, cos and sin [n, rot/2]."""
    rot = 2 * cos.shape[1]
    cos, sin, r = cos.double()[:, None], sin.double()[:, None], x[..., :rot].double()
    if layout == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:].double()], -1)


def _row_places(s):
    """The sequence and the position of each new token."""
    starts, lengths = s["starts"].long(), s["lengths"].long()
    row = torch.arange(s["new"], device=starts.device)
    seq = torch.searchsorted(starts, row, right=True) - 1
    return seq, lengths[seq] - starts[seq + 1] + row


def _append_plain(s):
    c = s["case"]
    _, pos = _row_places(s)
    cos, sin = s["cos"][pos], s["sin"][pos]
    q = _rotate(s["q"], cos, sin, c["layout"]).to(s["q"].dtype)
    k = _rotate(s["k"], cos, sin, c["layout"])
    held = [_unpack(*_pack(x.reshape(-1, c["dim"]))).view(s["k"].shape).to(s["k"].dtype) for x in (k, s["v"])]
    return {"q": q, "k": held[0], "v": held[1]}


def _attend_plain(s):
    c = s["case"]
    P, D, H = c["page"], c["dim"], c["kv_heads"]
    S, per = s["table"].shape
    G, N = c["q_heads"] // H, s["most"]
    blocks = s["pages"][s["table"].long().clamp_min(0)]  # [S, per, H, bytes]
    kc, vc, ks, vs = blocks.split([P * D // 2, P * D // 2, P * D // 32, P * D // 32], -1)
    k = _unpack(kc.unflatten(-1, (P, D // 2)), ks.unflatten(-1, (P, D // 32)))
    v = _unpack(vc.unflatten(-1, (P // 4, D // 2, 4)).transpose(-1, -2).flatten(-3, -2),
                vs.unflatten(-1, (P // 4, D // 32, 4)).transpose(-1, -2).flatten(-3, -2))
    k, v = (x.transpose(1, 2).reshape(S, H, per * P, D) for x in (k, v))
    lengths, starts = s["lengths"].long(), s["starts"].long()
    t = torch.arange(per * P, device="cuda")
    inside = (t[None] < lengths[:, None])[:, None, :, None]
    k, v = torch.where(inside, k, 0.0), torch.where(inside, v, 0.0)
    new = starts[1:] - starts[:-1]
    i = torch.arange(N, device="cuda")
    row = (starts[:-1, None] + i[None]).clamp_max(s["new"] - 1)
    q = s["q"].float()[row].view(S, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * N, D)
    score = torch.matmul(q, k.transpose(-1, -2)).view(S, H, G, N, per * P) / math.sqrt(D)
    pos = (lengths - new)[:, None] + i[None]
    seen = t[None, None] <= pos[..., None]
    if c["window"]:
        seen = seen & (t[None, None] > pos[..., None] - c["window"])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul((p / total).view(S, H, G * N, per * P), v).view(S, H, G, N, D)
    lse = (top + torch.log(total))[..., 0]
    kept = i[None] < new[:, None]
    o = o.permute(0, 3, 1, 2, 4).reshape(S, N, H * G, D)[kept]
    return {"out": o.to(s["q"].dtype), "lse": lse.permute(0, 3, 1, 2).reshape(S, N, H * G)[kept]}


def _logits_plain(s):
    z = s["logits"].float()
    R, C = z.shape
    if "history" in s:
        h = s["history"].long()
        count = torch.zeros(R, C + 1, device=z.device).scatter_add_(1, torch.where(h < 0, C, h), torch.ones(h.shape, device=z.device))[:, :C]
        z = torch.where(count > 0, torch.where(z > 0, z / REPETITION, z * REPETITION) - PRESENCE, z) - FREQUENCY * count
    if "bias_ids" in s:
        bias = torch.zeros(s["bias_ids"].shape[0], C, device=z.device).scatter_(1, s["bias_ids"].long(), s["bias_values"])
        z = z + bias
    z = z / s["temperature"]
    if "mask" in s:
        bit = torch.arange(C, device=z.device)
        allowed = (s["mask"].long()[:, bit >> 5] >> (bit & 31) & 1).bool()
        z = torch.where(allowed[s["mask_row"].long()] if s["mask"].shape[0] > 1 else allowed, z, -math.inf)
    top = z.amax(1, keepdim=True).clamp_min(-1e30)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    found = {"lse": lse[:, 0]}
    if "target" in s:
        found["score"] = torch.where(lse[:, 0] == -math.inf, -math.inf, z.gather(1, s["target"].long()[:, None])[:, 0] - lse[:, 0])
    if s["case"]["full"]:
        found["logp"] = torch.where(z == -math.inf, z, z - lse)
    return found


def _lora_plain(s):
    x, a, b = s["x"].float(), s["a"].float(), s["b"].float()
    which = s["adapter"].long()
    n, r = a.shape[:2]
    h = (x @ a.reshape(n * r, -1).t()).view(-1, n, r)  # every row with every adapter: two large products
    h = h * (which[:, None] == torch.arange(n, device=x.device))[..., None]
    delta = h.reshape(-1, n * r) @ b.transpose(1, 2).reshape(n * r, -1)
    scale = torch.where(which >= 0, s["scale"][which.clamp_min(0)], 0.0)
    return {"y": (s["y"].float() + scale[:, None] * delta).to(s["y"].dtype)}


# ------------------------------------------------------------------ the framework's calls


def _cache(lb, s):
    c = s["case"]
    cache = lb.KVCache(s["pages"], c["page"], c["kv_heads"], c["dim"])
    return cache, lb.KVBatch(s["starts"], s["lengths"], s["table"], s["new"], s["most"])


def _run_own(s):
    import paper_2603_14002_amd as lb

    c = s["case"]
    if c["op"] == "append":
        cache, batch = _cache(lb, s)
        layout = lb.LB_ROPE_HALF if c["layout"] == "half" else lb.LB_ROPE_INTERLEAVED
        q = lb.lb_kv_append(cache, batch, s["q"], s["k"], s["v"], rope=lb.Rope(s["cos"], s["sin"], layout))
        k, v = lb.lb_kv_read(cache, batch, s["k"].dtype)
        return {"q": q, "k": k, "v": v}
    if c["op"] == "attend":
        cache, batch = _cache(lb, s)
        out, lse = lb.lb_kv_attend(cache, batch, s["q"], 1.0 / math.sqrt(c["dim"]), window=c["window"], want_lse=True)
        return {"out": out, "lse": lse}
    if c["op"] == "logits":
        rules = lb.LogitRules(temperature=s["temperature"], history=s.get("history"), repetition=REPETITION, presence=PRESENCE,
                              frequency=FREQUENCY, bias_ids=s.get("bias_ids"), bias_values=s.get("bias_values"), mask=s.get("mask"), mask_row=s.get("mask_row"))
        logp, score, lse = lb.lb_logits_adjust(s["logits"], rules, target=s.get("target"), want_logprobs=c["full"])
        return {"lse": lse, **({"score": score} if c["scores"] else {}), **({"logp": logp} if c["full"] else {})}
    return {"y": lb.lb_lora_add(s["y"], s["x"], s["a"], s["b"], s["adapter"], s["scale"], out=torch.empty_like(s["y"]))}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append_plain, "attend": _attend_plain, "logits": _logits_plain, "lora": _lora_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_held(x):
    """What the cache holds of x [..., D] (64 bits): in each block of 32, the nearest level under the smallest scale that covers it."""
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    b = x.unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -124.0)
    guess = torch.floor(torch.log2(most.clamp_min(1e-37))) - 4
    for k in range(5, -1, -1):  # the smallest of these that covers the largest value
        e = torch.where(most <= 6 * torch.exp2(guess + k), guess + k, e)
    scale = torch.exp2(torch.where(most > 0, e, torch.full_like(e, -124.0)).clamp(-124, 125))
    y = (b / scale).abs()
    up = torch.searchsorted(level, y).clamp(1, 7)
    over, under = level[up] - y, y - level[up - 1]
    pick = torch.where((over < under) | ((over == under) & (up % 2 == 0)), up, up - 1)
    return (torch.where(b < 0, -1.0, 1.0) * level[pick] * scale).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "append":
        _, pos = _row_places(s)
        turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]
        rot = c["rot"]

        def rotated(x):
            r = x[..., :rot].double()
            pair = r.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["layout"] == "half" else r.unflatten(-1, (rot // 2, 2))
            u, w = pair[..., 0], pair[..., 1]
            pair = torch.stack([u * turn.real - w * turn.imag, w * turn.real + u * turn.imag], -1)
            r = pair.transpose(-1, -2).flatten(-2) if c["layout"] == "half" else pair.flatten(-2)
            return torch.cat([r, x[..., rot:].double()], -1)

        return {"q": rotated(s["q"]), "k": _exact_held(rotated(s["k"])), "v": _exact_held(s["v"].double())}
    if c["op"] == "attend":
        P, D, H = c["page"], c["dim"], c["kv_heads"]
        G = c["q_heads"] // H
        level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device="cuda")
        starts, lengths, outs, lses = s["starts"].tolist(), s["lengths"].tolist(), [], []
        for i, n in enumerate(lengths):
            a, z = starts[i], starts[i + 1]
            raw = s["pages"][s["table"][i, :-(-n // P)].long()]

            def values(lo, tokens_inside):
                codes = raw[..., lo:lo + P * D // 2]
                scales = raw[..., P * D + lo // 16:P * D + lo // 16 + P * D // 32]
                if tokens_inside:
                    codes, scales = (x.unflatten(-1, (P // 4, -1, 4)).transpose(-1, -2) for x in (codes, scales))
                codes, scales = codes.reshape(-1, H, P, D // 2), scales.reshape(-1, H, P, D // 32)
                x = level[torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()]
                x = x * (2.0 ** (scales.double() - 127)).repeat_interleave(32, -1)
                return x.transpose(0, 1).reshape(H, -1, D)[:, :n]

            k, v = values(0, False), values(P * D // 2, True)
            q = s["q"][a:z].double().view(z - a, H, G, D).permute(1, 2, 0, 3)
            t, p = torch.arange(n, device="cuda"), torch.arange(n - (z - a), n, device="cuda")[:, None]
            seen = (t <= p) & ((t > p - c["window"]) if c["window"] else (t >= 0))
            score = torch.where(seen, torch.matmul(q, k.mT.unsqueeze(1)) / D ** 0.5, -math.inf)
            lse = torch.logsumexp(score, -1)
            o = torch.matmul(torch.exp(score - lse[..., None]), v.unsqueeze(1))
            outs.append(o.permute(2, 0, 1, 3).reshape(z - a, H * G, D))
            lses.append(lse.permute(2, 0, 1).reshape(z - a, H * G))
        return {"out": torch.cat(outs), "lse": torch.cat(lses)}
    if c["op"] == "logits":
        found = {"lse": [], "score": [], "logp": []}
        R, C = s["logits"].shape
        step = max(1, 40_000_000 // C)
        for r in range(0, R, step):
            z = s["logits"][r:r + step].double()
            n = z.shape[0]
            at = torch.arange(n, device="cuda")[:, None]
            if "history" in s:
                h = s["history"][r:r + n].long()
                count = torch.zeros(n, C + 1, dtype=torch.float64, device="cuda")
                count.index_put_((at.expand_as(h), torch.where(h < 0, C, h)), torch.ones((), dtype=torch.float64, device="cuda"), accumulate=True)
                count = count[:, :C]
                z = torch.where(count > 0, torch.where(z > 0, z / REPETITION, z * REPETITION) - PRESENCE - FREQUENCY * count, z)
            if "bias_ids" in s:
                ids, values = ((x if c["shared"] else x[r:r + n]) for x in (s["bias_ids"].long(), s["bias_values"].double()))
                z = z.index_put((at.expand(n, ids.shape[1]), ids.expand(n, -1)), values.expand(n, -1), accumulate=True)
            z = z / s["temperature"]
            if "mask" in s:
                bits = (s["mask"][:, :, None] >> torch.arange(32, device="cuda")) & 1
                z = torch.where(bits.flatten(1)[:, :C][s["mask_row"][r:r + n].long()] == 1, z, -math.inf)
            lse = torch.logsumexp(z, 1)
            logp = torch.where(lse[:, None] == -math.inf, -math.inf, torch.log_softmax(z, 1))
            found["lse"].append(lse)
            if c["scores"]:
                found["score"].append(logp[at[:, 0], s["target"][r:r + n].long()])
            if c["full"]:
                found["logp"].append(logp)
        return {k: torch.cat(v) for k, v in found.items() if v}
    y = s["y"].double()
    for i, a in enumerate(s["adapter"].unique().tolist()):
        if a >= 0:
            rows = s["adapter"] == a
            y[rows] += s["scale"][a].double() * ((s["x"][rows].double() @ s["a"][a].double().t()) @ s["b"][a].double().t())
    return {"y": y}
