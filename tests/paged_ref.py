"""The paged cache's operators in plain Python and 64 bits, for the tests: page bookkeeping one request after the
other, the append one run of tokens after the other, attention one sequence after the other."""
import math

import numpy as np
import torch

PAGE, D = 64, 64
E_MIN, E_MAX = -48, 47


def pages_of(n):
    return -(-n // PAGE)


class Pool:
    """Free pages (a list, the last goes out first), a table and lengths, as lists."""

    def __init__(self, stack, table, seq_len):
        self.stack, self.table, self.len = list(stack), [list(r) for r in table], list(seq_len)

    def assign(self, new, rows, total_pages):
        width = len(self.table[0])
        slots, pos, row0, granted = [-1] * rows, [-1] * rows, [0], []
        total, asked, free0 = 0, 0, len(self.stack)
        for b, n in enumerate(new):
            first = min(total, rows)
            total += max(n, 0)
            row0.append(min(total, rows))
            valid = n >= 0 and self.len[b] >= 0 and self.len[b] + n <= PAGE * width and total <= rows
            if not valid:
                granted.append(0)
                continue
            held = pages_of(self.len[b])
            need = pages_of(self.len[b] + n) - held
            asked += need
            if need and asked > free0:
                granted.append(0)
                continue
            granted.append(1)
            for i in range(need):
                self.table[b][held + i] = self.stack.pop()
            for j in range(n):
                p = self.len[b] + j
                page = self.table[b][p // PAGE]
                pos[first + j] = p
                slots[first + j] = page * PAGE + p % PAGE if 0 <= page < total_pages else -1
            self.len[b] += n
        return slots, pos, row0, granted

    def release(self, keep):
        width, freed = len(self.table[0]), []
        for b, k in enumerate(keep):
            if self.len[b] < 0 or self.len[b] > PAGE * width:
                continue
            k = min(max(k, 0), self.len[b])
            for p in range(pages_of(k), pages_of(self.len[b])):
                freed.append(self.table[b][p])
                self.table[b][p] = -1
            self.len[b] = k
        self.stack += freed[::-1]


def e4m3(x):
    """The e4m3 values nearest to x (fp64), ties to even, saturated at 448."""
    x = np.asarray(x, np.float64)
    size = np.abs(x)
    step = 2.0 ** (np.floor(np.log2(np.maximum(size, 2.0 ** -6))) - 3)
    return np.copysign(np.minimum(np.round(size / step) * step, 448.0), x)


def decode(codes):
    """The e4m3 values of uint8 codes."""
    c = np.arange(256)
    e, m, s = (c >> 3) & 15, c & 7, np.where(c >= 128, -1.0, 1.0)
    lut = s * np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    lut[[127, 255]] = np.nan
    return lut[codes]


def exponent(amax):
    if amax == 0:
        return E_MIN
    m, e = math.frexp(amax)                    # amax = m 2^e, 1/2 <= m < 1
    return min(max(e - 9 + (m > 0.875), E_MIN), E_MAX)


def rope32(x, cs, pos, half):
    """x [rows][heads][64] fp32 rotated in fp32, products and sums rounded on their own."""
    c, s = cs[pos][:, None, :, 0], cs[pos][:, None, :, 1]
    out = np.empty_like(x)
    a, b = (x[..., :32], x[..., 32:]) if half else (x[..., 0::2], x[..., 1::2])
    with np.errstate(over="ignore", invalid="ignore"):
        p, q = a * c - b * s, a * s + b * c
    if half:
        out[..., :32], out[..., 32:] = p, q
    else:
        out[..., 0::2], out[..., 1::2] = p, q
    return out


class CacheRef:
    """Code values and exponents of a cache, by page and token: k, v [L][H][pages][64][64], e [L][H][pages][2]."""

    def __init__(self, cache):
        k, v, s = cache.values()
        self.k = k.double().cpu().numpy()
        self.v = v.reshape(k.shape).double().cpu().numpy()
        self.e = np.round(np.log2(s.double().cpu().numpy())).astype(int)

    def append(self, k, v, slots, pos, cs, half, layer0=0, positions=None):
        """k, v: fp32 [nlayers][rows][H][64]."""
        nl, rows = k.shape[:2]
        pages = self.k.shape[2]
        live = [0 <= s < pages * PAGE and (cs is None or 0 <= p < len(cs)) for s, p in zip(slots, pos)]
        kr = k if cs is None else np.stack([rope32(k[l], cs, np.where(live, pos, 0), half) for l in range(nl)])
        r = 0
        while r < rows:
            if not live[r]:
                r += 1
                continue
            n = 1
            while r + n < rows and live[r + n] and slots[r + n] == slots[r] + n and slots[r + n] % PAGE:
                n += 1
            page, at = slots[r] // PAGE, slots[r] % PAGE
            for l in range(nl):
                for h in range(k.shape[2]):
                    kk, vv = kr[l, r:r + n, h].astype(np.float64), v[l, r:r + n, h].astype(np.float64)
                    bad = ~(np.isfinite(kk).all(1) & np.isfinite(vv).all(1))
                    for x, codes, i in ((kk, self.k, 0), (vv, self.v, 1)):
                        x = np.where(bad[:, None], 0.0, x)
                        e = exponent(np.abs(x).max())
                        old = self.e[layer0 + l, h, page, i]
                        here = codes[layer0 + l, h, page]
                        if at:
                            e = max(e, old)
                            if e > old:
                                here[:] = e4m3(here * 2.0 ** float(old - e))
                        self.e[layer0 + l, h, page, i] = e
                        q = e4m3(x * 2.0 ** float(-e))
                        if i == 0:
                            q[bad] = np.nan
                        here[at:at + n] = q
            r += n


def attend(k, v, q, pos, row0, table, seq_len, causal, scale, cs64=None, half=False):
    """k, v [L][Hkv][pages][64][64] values, q [L][rows][H][64] (fp64 tensors on one device); the rest lists. cs64:
    (cos, sin) as complex fp64 [positions][32], or None. Returns (out, (spread, floor), size), with, for softmax
    weights w, spread = sum_j w_j |v_j|, floor = max(w) sum_j |v_j| and size = max_j sum_d |q_d k_jd| * scale, which the
    tests' bounds go by; rows of no sequence and rows at a negative position are NaN in
    out."""
    L, rows, H = q.shape[:3]
    Hkv = k.shape[1]
    G = H // Hkv
    out = torch.full_like(q, float("nan"))
    spread, floor, size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((L, rows, H, 1), dtype=q.dtype, device=q.device)
    for b in range(len(seq_len)):
        lo, hi, n = row0[b], row0[b + 1], seq_len[b]
        if hi <= lo:
            continue
        refused = torch.tensor([x < 0 for x in pos[lo:hi]], device=q.device)
        if n == 0:
            out[:, lo:hi] = 0
            out[:, lo:hi][:, refused] = float("nan")
            continue
        ids = table[b][:pages_of(n)]
        kb = k[:, :, ids].reshape(L, Hkv, -1, D)[:, :, :n]
        vb = v[:, :, ids].reshape(L, Hkv, -1, D)[:, :, :n]
        qb = q[:, lo:hi]
        p = torch.tensor(pos[lo:hi], device=q.device).clamp(min=0)
        if cs64 is not None:
            z = cs64[p][:, None]
            if half:
                w = torch.complex(qb[..., :32].contiguous(), qb[..., 32:].contiguous()) * z
                qb = torch.cat([w.real, w.imag], -1)
            else:
                w = torch.view_as_complex(qb.reshape(L, hi - lo, H, 32, 2).contiguous()) * z
                qb = torch.view_as_real(w).reshape(qb.shape)
        qb = qb.reshape(L, hi - lo, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(L, Hkv, -1, D)
        seen = torch.ones((hi - lo, n), dtype=torch.bool, device=q.device)
        if causal:
            seen = torch.arange(n, device=q.device) <= p[:, None]
        seen = seen.repeat(G, 1)
        kt = kb.transpose(2, 3).contiguous()
        s = (torch.matmul(qb, kt) * scale).masked_fill(~seen, float("-inf"))
        t = (torch.matmul(qb.abs(), kt.abs()) * scale).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        w = torch.softmax(s, -1)
        back = lambda x: x.reshape(L, Hkv, G, hi - lo, -1).permute(0, 3, 1, 2, 4).reshape(L, hi - lo, H, -1)
        # (a weight of zero times a value that is no number is none either: values are finite here)
        out[:, lo:hi] = back(torch.matmul(w, vb))
        out[:, lo:hi][:, refused] = float("nan")
        flat = torch.matmul(seen.to(q.dtype).expand(w.shape).contiguous(), vb.abs()) * w.amax(-1, keepdim=True)
        spread[:, lo:hi] = back(torch.matmul(w, vb.abs()))
        floor[:, lo:hi] = back(flat)
        size[:, lo:hi] = back(t)
    return out, (spread, floor), size


def bound(out, spread, size, length, prec, dtype):
    """How far a result may be from the 64-bit one, elementwise.

    A score's error: RoPE rounds each product and sum (3 steps of 2^-24), q' is held to 2^-11 (prec 0) or in two fp16
    parts to 2^-22 (and, over its row's power of two, 2^-25 absolutely, which the same term covers: entries below
    2^-3 of the largest matter less), and the sum over 64 products, the scaling and the subtraction of the maximum
    round at most 70 times: eps_s * size, size >= |score|. A weight's relative error is the score's, the exp2's
    (2^-22), and its rounding to fp16 (2^-11; prec 2: two parts, 2^-22). The largest weight is held as 2^7 at least, and
    fp16 has steps of 2^-24, so that a weight or its second part may also be off by 2^-25 where it is small:
    2^-32 of the largest, times |v| for every token: 2^-32 floor. Numerator and denominator have the relative errors
    once each; both sum `length` terms in fp32. Last the output's own rounding."""
    spread, floor = spread
    eps_s = {0: 2.0 ** -11, 1: 2.0 ** -22, 2: 2.0 ** -22}[prec] + 76 * 2.0 ** -24
    eps_p = 2.0 ** -22 if prec == 2 else 2.0 ** -11
    rel = 2 * torch.expm1(eps_s * size) + eps_p + 2.0 ** -21 + 2 * (length + 64) * 2.0 ** -24
    half = torch.finfo(dtype).eps / 2
    return ((rel * spread + 2.0 ** -32 * floor) * (1 + half) + half * out.abs() + 1e-30
            + (2.0 ** -25 if dtype == torch.float16 else 0.0))
