"""Plain 64-bit forms of the fusion scorer's operators, on the CPU, and the bookkeeping of
ragged batches that their tests share."""

import math

import numpy as np
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step


def encode(x):
    """Codes (0..15) and scale bytes of x [..., D] in 64 bits: by comparing with every border."""
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    e = torch.full_like(most, -124.0)
    for k in range(-124, 125):  # the smallest e of -124..125 that covers the largest value, else 125
        e = torch.where(most > 6.0 * 2.0 ** k, float(k + 1), e)
    y = torch.where(bad, 0.0, (b / torch.exp2(e)).abs())
    code = torch.zeros_like(y)
    for i in range(1, 8):
        border = (LEVELS[i - 1] + LEVELS[i]) / 2
        code += (y > border) | ((y == border) & (i % 2 == 0))
    code += 8.0 * (torch.signbit(b) & ~bad)
    scale = torch.where(bad, 255.0, e + 127.0)
    return code.flatten(-2).to(torch.uint8), scale[..., 0].to(torch.uint8)


def decode(code, scale):
    level = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    s = torch.where(scale == 255, math.nan, 2.0 ** (scale.double() - 127))
    return level[code.long()] * s.repeat_interleave(32, -1)


def rotate(x, cos, sin, interleaved):
    """x [n, heads, D], cos and sin [n, rot/2], in 64 bits."""
    x, rot = x.double().clone(), 2 * cos.shape[-1]
    c, s = cos.double()[:, None], sin.double()[:, None]
    one = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    two = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    a, b = x[..., one].clone(), x[..., two].clone()
    x[..., one], x[..., two] = a * c - b * s, b * c + a * s
    return x


class Ragged:
    """Sequences with `new` new tokens each of `length` tokens, their pages anywhere in a pool of garbage."""

    def __init__(self, new, length, P, H, D, seed=0, spare=2, pad_rows=0):
        rng = np.random.default_rng(seed)
        self.new, self.length, self.P, self.H, self.D = list(new), list(length), P, H, D
        counts = [-(-n // P) for n in length]
        self.n_pages = sum(counts) + spare
        place = rng.permutation(self.n_pages)[:sum(counts)]
        width = max([1] + counts)
        self.table = torch.full((len(length), width), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(counts):
            self.table[i, :c] = torch.from_numpy(place[at:at + c].astype(np.int32))
            at += c
        self.starts = torch.tensor(np.cumsum([0] + self.new).astype(np.int32))
        self.lengths = torch.tensor(self.length, dtype=torch.int32)
        self.n_rows = sum(self.new) + pad_rows
        # garbage: any byte, NaN scales among them
        self.pages = torch.from_numpy(rng.integers(0, 256, (self.n_pages, H, P * (D + D // 16)), dtype=np.uint8))

    def rows(self):
        """(sequence, position) of every row that is not padding."""
        return [(s, self.length[s] - n + i) for s, n in enumerate(self.new) for i in range(n)]

    def put(self, s, k, v):
        """Writes tokens 0.. of sequence s from k and v [tokens, H, D] (64 bits), byte by byte as the layout says."""
        P, H, D = self.P, self.H, self.D
        kc, ks = encode(k)
        vc, vs = encode(v)
        for t in range(k.shape[0]):
            page, slot = int(self.table[s, t // P]), t % P
            mem = self.pages[page]
            mem[:, slot * (D // 2):(slot + 1) * (D // 2)] = kc[t, :, 0::2] | kc[t, :, 1::2] << 4
            at = P * D // 2 + ((slot // 4) * (D // 2) + torch.arange(D // 2)) * 4 + slot % 4
            mem[:, at] = vc[t, :, 0::2] | vc[t, :, 1::2] << 4
            mem[:, P * D + slot * (D // 32):P * D + (slot + 1) * (D // 32)] = ks[t]
            at = P * D + P * D // 32 + ((slot // 4) * (D // 32) + torch.arange(D // 32)) * 4 + slot % 4
            mem[:, at] = vs[t]

    def get(self, s, n, pages=None):
        """Keys and values of tokens 0..n-1 of sequence s, [n, H, D] in 64 bits."""
        P, H, D = self.P, self.H, self.D
        pages = self.pages if pages is None else pages
        out = []
        for value in (False, True):
            codes, scales = torch.zeros(n, H, D, dtype=torch.uint8), torch.zeros(n, H, D // 32, dtype=torch.uint8)
            for t in range(n):
                mem, slot = pages[int(self.table[s, t // P])], t % P
                if value:
                    byte = mem[:, P * D // 2 + ((slot // 4) * (D // 2) + torch.arange(D // 2)) * 4 + slot % 4]
                    scales[t] = mem[:, P * D + P * D // 32 + ((slot // 4) * (D // 32) + torch.arange(D // 32)) * 4 + slot % 4]
                else:
                    byte = mem[:, slot * (D // 2):(slot + 1) * (D // 2)]
                    scales[t] = mem[:, P * D + slot * (D // 32):P * D + (slot + 1) * (D // 32)]
                codes[t, :, 0::2], codes[t, :, 1::2] = byte & 15, byte >> 4
            out.append(decode(codes, scales))
        return out


def attend(q, k, v, scale, first, window):
    """One sequence: q [m, Hq, D] of the positions first.., k, v [n, H, D], all 64 bits.  Returns out, lse, and per
    query and channel sum p|v| and per query the largest sum |q k| scale, for error bounds."""
    m, Hq, D = q.shape
    n, H = k.shape[0], k.shape[1]
    out, lse = torch.zeros(m, Hq, D, dtype=torch.float64), torch.full((m, Hq), -math.inf, dtype=torch.float64)
    mass, reach = torch.zeros(m, Hq, D, dtype=torch.float64), torch.zeros(m, Hq, dtype=torch.float64)
    for i in range(m):
        p = first + i
        lo = max(0, p - window + 1) if window else 0
        if p < 0 or lo > min(p, n - 1):
            continue
        for g in range(H):
            heads = slice(g * (Hq // H), (g + 1) * (Hq // H))
            kk, vv = k[lo:p + 1, g], v[lo:p + 1, g]
            s = (q[i, heads] @ kk.t()) * scale
            lse[i, heads] = torch.logsumexp(s, 1)
            w = torch.exp(s - lse[i, heads, None])
            out[i, heads] = w @ vv
            mass[i, heads] = w @ vv.abs()
            reach[i, heads] = ((q[i, heads].abs() @ kk.abs().t()) * abs(scale)).amax(1)
    return out, lse, mass, reach


def logits_rules(x, history=None, repetition=1.0, presence=0.0, frequency=0.0, bias_ids=None, bias_values=None, mask=None,
                 mask_row=None, temperature=1.0):
    """Rows of logits after the rules, 64 bits, one class at a time."""
    z = x.double().clone()
    R, C = z.shape
    for r in range(R):
        if history is not None:
            ids = [int(w) for w in history[r] if 0 <= int(w) < C]
            for w in set(ids):
                v = float(z[r, w])
                v = v / repetition if v > 0 else v * repetition
                z[r, w] = v - presence - frequency * ids.count(w)
        if bias_ids is not None:
            row = r if bias_ids.shape[0] > 1 else 0
            last = {int(w): float(b) for w, b in zip(bias_ids[row], bias_values[row]) if 0 <= int(w) < C}
            for w, b in last.items():
                z[r, w] += b
        z[r] /= temperature
        if mask is not None:
            k = int(mask_row[r]) if mask_row is not None else r if mask.shape[0] > 1 else 0
            if 0 <= k < mask.shape[0]:
                bits = torch.from_numpy(np.unpackbits(mask[k].numpy().view(np.uint8), bitorder="little")[:C].astype(bool))
                z[r] = torch.where(bits, z[r], -math.inf)
    return z


def log_softmax(z):
    """(log-probabilities, lse); a row with nothing left: -infinity throughout."""
    lse = torch.logsumexp(z, 1)
    return torch.where(z == -math.inf, z, z - lse[:, None]), lse
