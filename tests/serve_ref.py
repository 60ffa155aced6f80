"""The operators around the paged 4-bit cache in plain Python, for the tests: codes by comparison with the grid, pages
byte by byte, norms and attention in 64 bits, verification one token after the other."""
import math

import numpy as np
import torch

import paged_ref

PAGE, D = 64, 64
E_MIN, E_MAX = -48, 47
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SIGNS = np.array([[1.0 - 2.0 * (bin(i & j).count("1") % 2) for j in range(D)] for i in range(D)])


def hadamard32(x):
    """x [..., 64] fp32 times the signs' matrix over 8, by sums and differences of entries 1, 2, .. 32 apart."""
    x = np.array(x, np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        for n in (1, 2, 4, 8, 16, 32):
            y = x.reshape(*x.shape[:-1], D // 2 // n, 2, n)
            x = np.stack([y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]], -2).reshape(x.shape)
        return x * np.float32(0.125)


def exponent(amax):
    """The least E with amax <= 6 * 2^E, within [E_MIN, E_MAX]."""
    if amax == 0:
        return E_MIN
    m, e = math.frexp(amax)                    # amax = m 2^e, 1/2 <= m < 1
    return min(max(e - 3 + (m > 0.75), E_MIN), E_MAX)


def e2m1(x):
    """Codes of x (fp64): the nearest of the grid, ties to the even code, saturated."""
    x = np.asarray(x, np.float64)
    size = np.minimum(np.abs(x), 8.0)[..., None]              # (past the grid; far beyond it differences would round)
    far = np.abs(size - GRID)
    near = far.min(-1, keepdims=True)
    tied = far == near                         # (two of the grid at most)
    first = tied.argmax(-1)
    both = tied.sum(-1) > 1
    code = first + (both & (first % 2 == 1))
    return (code + 8 * np.signbit(x)).astype(np.uint8)


def value_of(codes):
    return np.concatenate([GRID, -GRID])[codes]


def at_key(t, d):
    return 32 * t + d // 2


def at_value(t, d):
    i, g, r = t // 16, t // 4 % 4, t % 4
    return i // 2 * 1024 + d // 4 * 64 + g * 16 + i % 2 * 8 + r * 2 + d % 4 // 2


def at_key_scale(t):
    return t % 16 * 4 + t // 16


def at_value_scale(t):
    return 64 + t // 4 % 4 * 16 + t // 16 * 4 + t % 4


KEY = np.array([[at_key(t, d) for d in range(D)] for t in range(PAGE)])
VALUE = np.array([[at_value(t, d) for d in range(D)] for t in range(PAGE)])
KEY_SCALE, VALUE_SCALE = np.array([at_key_scale(t) for t in range(PAGE)]), np.array([at_value_scale(t) for t in range(PAGE)])


class CacheRef:
    """The bytes of a Cache4."""

    def __init__(self, cache):
        self.k, self.v, self.s = (t.cpu().numpy().copy() for t in (cache.k_codes, cache.v_codes, cache.scales))

    def put(self, l, h, slot, kc, ke, vc, ve):
        page, t = slot // PAGE, slot % PAGE
        for plane, where, codes in ((self.k, KEY, kc), (self.v, VALUE, vc)):
            for d in range(D):
                byte = where[t, d]
                held = plane[l, h, page, byte]
                plane[l, h, page, byte] = (held & 0xF0) | codes[d] if d % 2 == 0 else (held & 0x0F) | codes[d] << 4
        self.s[l, h, page, KEY_SCALE[t]], self.s[l, h, page, VALUE_SCALE[t]] = ke, ve

    def append(self, k, v, slots, pos, cs, half, layer0=0):
        """k, v: fp32 [nlayers][rows][H][64]."""
        pages = self.k.shape[2]
        for l in range(k.shape[0]):
            live = [0 <= s < pages * PAGE and (cs is None or 0 <= p < len(cs)) for s, p in zip(slots, pos)]
            kr = k[l] if cs is None else paged_ref.rope32(k[l], cs, np.where(live, pos, 0), half)
            kr, vr = hadamard32(kr), hadamard32(v[l])
            for r, slot in enumerate(slots):
                if not live[r]:
                    continue
                for h in range(k.shape[2]):
                    x, y = kr[r, h].astype(np.float64), vr[r, h].astype(np.float64)
                    if not (np.isfinite(x).all() and np.isfinite(y).all()):
                        self.put(layer0 + l, h, slot, self.bad_codes(x), 255, np.zeros(D, np.uint8), 127)
                        continue
                    ke, ve = exponent(np.abs(x).max()), exponent(np.abs(y).max())
                    self.put(layer0 + l, h, slot, e2m1(x * 2.0 ** -ke), ke + 127, e2m1(y * 2.0 ** -ve), ve + 127)

    @staticmethod
    def bad_codes(x):
        return np.zeros(D, np.uint8)           # (not compared: the scale says that the key is no number)

    def values(self):
        """(keys, values) as fp64 [L][H][pages][64][64] in the Hadamard basis."""
        out = []
        for plane, where, at in ((self.k, KEY, KEY_SCALE), (self.v, VALUE, VALUE_SCALE)):
            nibble = (plane[..., where] >> (4 * (np.arange(D) % 2))) & 15
            e = self.s[..., at].astype(np.float64)
            x = value_of(nibble) * 2.0 ** (e - 127.0)[..., None]
            x[e == 255] = np.nan
            out.append(x)
        return out


def rotated(x, pos, cs64, half):
    """x [L, rows, heads, 64] fp64 at positions pos [rows]; cs64: (cos, sin) as complex [positions][32], or None."""
    if cs64 is None:
        return x
    z = cs64[pos][:, None]
    if half:
        w = torch.complex(x[..., :32].contiguous(), x[..., 32:].contiguous()) * z
        return torch.cat([w.real, w.imag], -1)
    w = torch.view_as_complex(x.reshape(*x.shape[:-1], 32, 2).contiguous()) * z
    return torch.view_as_real(w).reshape(x.shape)


def attend(k, v, q, pos, row0, table, seq_len, causal, scale, cs64=None, half=False):
    """k, v [L][Hkv][pages][64][64] in the Hadamard basis, q [L][rows][H][64] (fp64 tensors on one device). Returns out
    and what bound() goes by: spread = sum_j w_j sum_d |v_jd| / 8 (in the Hadamard basis, for all dimensions), size =
    max_j sum_d |q_d k_jd| * scale and reach = sum_d |q'_d| / 8 * max_j sum_d |k_jd| * scale."""
    had = torch.tensor(SIGNS / 8.0, device=q.device)
    q = rotated(q, torch.tensor(pos, device=q.device).clamp(min=0), cs64, half)
    out, (spread, _), size = paged_ref.attend(k, v, q @ had, pos, row0, table, seq_len, causal, scale)
    G = q.shape[2] // k.shape[1]
    most = torch.zeros_like(size)
    for b, n in enumerate(seq_len):
        if n > 0 and row0[b + 1] > row0[b]:
            rows = k[:, :, table[b][:paged_ref.pages_of(n)]].abs().sum(-1).flatten(2)[..., :n]
            most[:, row0[b]:row0[b + 1]] = rows.amax(-1).repeat_interleave(G, 1)[:, None, :, None]
    reach = q.abs().sum(-1, keepdim=True) / 8 * most * scale
    return out @ had, spread.sum(-1, keepdim=True) / 8, size, reach


def bound(out, spread, size, reach, length, eps, dtype):
    """How far a result may be from the 64-bit one, elementwise. eps: what the rounding of a query's entry and of a weight
    leaves, relative to them.

    RoPE rounds three times for each entry and the butterflies six, relative to the sum of the entries' sizes that go
    in: 10 * 2^-24 (entries' sizes grow by sqrt 2 in a rotation) of reach in a score, and eps[0] of its own size (an entry's
    rounding is relative to itself down to 2^-38 of its row's largest, the rest of which 2^-24 covers); the sum over 64 products
    and parts, the scales and the difference from the reference round at most 200 times 2^-24 of it. A weight has the
    score's error, the exp2's (2^-22) and its own rounding's; numerator and denominator both. Where weights are held in
    fp16 its steps are 2^-32 of the largest w_j scale_j, each times a code of at most 6: for `length` tokens less than
    the 2^-24 length of the sums, as spread is more than w_j scale_j for codes that are not nearly all zero. Both sum
    `length` terms in fp32, a few parts each, and joins of waves and splits scale them a few times. Errors of the
    numerator are relative to sum_j w_j |v_j| by dimension of the Hadamard basis, and the way back sums them over the
    dimensions: `spread`; its own butterflies round seven times more. Last the output's own rounding."""
    score = eps[0] * size + 2.0 ** -24 * (200 * size + 15 * reach)
    rel = 2 * torch.expm1(score) + 2 * eps[1] + 2.0 ** -21 + (2 * 3 * length + 100) * 2.0 ** -24
    half = torch.finfo(dtype).eps / 2
    return rel * spread * (1 + half) + half * out.abs() + 1e-30 + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def norm_rope(x, weight, eps, angles, half):
    """x [L, rows, heads, 64], weight [L, 64] fp64, angles: complex [rows][32] or None."""
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight[:, None, None]
    if angles is None:
        return y
    return rotated(y, torch.arange(x.shape[1], device=x.device), angles, half)


def counted(p):
    return p if math.isfinite(p) and p > 0 else 0.0


def verify(target, draft, tokens, row0, uniform, uniform_next, seq_len):
    """target, draft: fp64 arrays [rows][vocab] (draft None: certain); the rest lists. Returns accepted, keep and, for each
    sequence, the tokens that may come next: [(token, its weights' sum before it, up to it, the border)] by exact sums."""
    from fractions import Fraction
    accepted, keep, drawn = [], [], []
    rows, vocab = target.shape
    for b in range(len(row0) - 1):
        lo, hi = row0[b], row0[b + 1]
        if lo < 0 or hi <= lo or hi > rows:
            accepted.append(0)
            keep.append(seq_len[b])
            drawn.append(-1)
            continue
        n = 0
        while lo + n + 1 < hi:
            t, d = lo + n, int(tokens[lo + n + 1])
            if not 0 <= d < vocab:
                break
            q = 1.0 if draft is None else counted(float(draft[t, d]))
            u = float(uniform[t])
            if math.isnan(u) or not Fraction(u) * Fraction(q) < Fraction(counted(float(target[t, d]))):
                break
            n += 1
        rejected = lo + n + 1 < hi
        p = np.where(np.isfinite(target[lo + n]) & (target[lo + n] > 0), target[lo + n], 0.0)
        w = p
        if rejected:
            if draft is None:
                q = np.zeros(vocab)
                if 0 <= int(tokens[lo + n + 1]) < vocab:
                    q[int(tokens[lo + n + 1])] = 1.0
            else:
                q = np.where(np.isfinite(draft[lo + n]) & (draft[lo + n] > 0), draft[lo + n], 0.0)
            w = np.maximum(p - q, 0.0)
            if not w.any():
                w = p
        accepted.append(n)
        keep.append(seq_len[b] - (hi - lo - 1) + n)
        r = float(uniform_next[b])
        if not w.any():
            drawn.append(-1)
        elif math.isnan(r):
            drawn.append(int(np.flatnonzero(w)[-1]))
        else:
            upto, total, border = Fraction(0), sum(map(Fraction, w[w > 0])), None
            border = Fraction(r) * total
            for x in np.flatnonzero(w):
                upto += Fraction(w[x])
                if upto > border:
                    break
            drawn.append(int(x))
    return accepted, keep, drawn
