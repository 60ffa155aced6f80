"""Performance cases of the serving step around a paged 4-bit KV cache: queries and keys normed and rotated before it,
keys and values quantized into it and read back, attention over it, and the verification of drafted tokens after it.

A case is a dict of plain values; its "op" says what one pass does:
  norm     norm every head of q and k and rotate it by its row's positions
  store    quantize new keys and values into the pages, then read the same tokens back
  attend   attention of the new rows over the pages
  step     norm, quantize and attend, with q, k and v as slices of one projection's output
  verify   accept or reject drafted tokens and draw every sequence's next one
A sequence of a cache case has up to `cached` tokens before the pass and up to `new` in it (exactly those unless
`ragged`). The tokens attended to are both. `dtype` is the type of q, k, v and the outputs, or of the probabilities.

Sizes are those of the repository's workloads (20 heads x 33 layers, 40 heads, 1024 and 8192 tokens, 64 ragged
sequences, 33 symbols) and generic ones of grouped heads, chunked prefill and large vocabularies around them.

With `own` false, run() is the operators' plain form in torch; with `own` true it makes the library's calls.
"""
import math

import torch

own = False

D = 64
PAGE = 64
E_MIN, E_MAX = -48, 47
EPS = 1e-6
DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

_CACHE = {"layers": 1, "heads": 20, "kv_heads": 20, "batch": 1, "cached": 0, "new": 1, "ragged": False,
          "causal": True, "dtype": "fp16", "rope": "pairs", "axes": 1}
_VERIFY = {"vocab": 33, "batch": 8, "drafts": 3, "ragged": False, "dtype": "fp32", "draft": True}


def _case(op, name=None, **kw):
    c = dict(_VERIFY if op == "verify" else _CACHE, op=op, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The queries and keys of 64 new tokens in one layer, grouped heads.
        _case("norm", "norm_tokens_layer", heads=40, kv_heads=8, batch=64, cached=1000, ragged=True, dtype="bf16"),
        # The prompts of 16 requests with image patches in them: positions of three axes.
        _case("norm", "norm_prompts_layer", heads=40, kv_heads=8, batch=16, new=1024, dtype="bf16", rope="half", axes=3),
        # One new token of each of 16 sequences in one layer, read back: the smallest store.
        _case("store", "store_tokens_layer", heads=40, kv_heads=8, batch=16, cached=300, ragged=True, dtype="bf16"),
        # A ragged batch of 64 prompts in one layer, as a request's pages are written and moved out again.
        _case("store", "store_prompts_layer", heads=40, kv_heads=8, batch=64, new=1024, ragged=True, dtype="bf16"),
        # One sequence's next token in one layer, 1024 tokens before it.
        _case("attend", "attend_token_layer", cached=1024),
        # The same in all 33 layers: the shape of the repository's headline step.
        _case("attend", "attend_token_model", layers=33, cached=1024),
        # One layer of 16 sequences of 8192 cached tokens, 40 heads: the longest contexts, bound by memory.
        _case("attend", "attend_long_layer", heads=40, kv_heads=40, batch=16, cached=8191),
        # Chunks of prompts on top of what is cached, grouped heads, bf16.
        _case("attend", "attend_chunk_layer", heads=40, kv_heads=8, batch=4, cached=4000, new=512, ragged=True,
              dtype="bf16"),
        # fp32 in and out, the other RoPE pairing, odd lengths, a few drafted tokens per sequence.
        _case("attend", "attend_fp32_layer", heads=12, kv_heads=4, batch=5, cached=777, new=9, ragged=True,
              dtype="fp32", rope="half"),
        # A decode step of 64 ragged sequences in one layer, grouped heads: norm, store, attend.
        _case("step", "step_batch_layer", heads=40, kv_heads=8, batch=64, cached=2000, ragged=True, dtype="bf16"),
        # Three drafted symbols of each of 8 sequences over an alphabet of 33: latency.
        _case("verify", "verify_symbols", vocab=33, batch=8, drafts=3),
        # Up to six drafted tokens of each of 32 sequences over a large vocabulary.
        _case("verify", "verify_tokens", vocab=131072, batch=32, drafts=6, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "store", "attend", "attend", "step", "verify"])
    if op == "verify":
        vocab = _log(rng, 20, 200_000)
        drafts = _log(rng, 1, 12)
        batch = _log(rng, 1, max(1, min(256, 25_000_000 // (vocab * (drafts + 1)))))
        return _case(op, vocab=vocab, batch=batch, drafts=drafts, ragged=rng.random() < 0.6,
                     dtype=rng.choice(["fp32", "fp32", "fp16", "bf16"]), draft=rng.random() < 0.8)
    kv = rng.choice([1, 2, 4, 5, 8, 12, 20, 33])
    kw = {"kv_heads": kv, "heads": kv * (1 if kv > 8 else rng.choice([1, 2, 3, 5, 7, 8])),
          "dtype": rng.choice(["fp16", "fp16", "bf16", "bf16", "fp32"]),
          "rope": rng.choice(["pairs", "pairs", "half", "none"]), "ragged": rng.random() < 0.7}
    kw["new"] = 1 if rng.random() < 0.4 else _log(rng, 1, 1024)
    kw["cached"] = rng.choice([0, _log(rng, 1, 8000)])
    length = kw["new"] + kw["cached"]
    # (layer, sequence, head) tuples that the tokens and the pairs of tokens leave room for
    room = min(2_000_000 // (kv * length), 300_000_000 // (kw["heads"] * kw["new"] * length),
               600_000 // (kw["heads"] * kw["new"]))
    kw["batch"] = _log(rng, 1, max(1, min(128, room)))
    kw["layers"] = 1 if rng.random() < 0.7 else max(1, min(36, room // kw["batch"]))
    if op in ("norm", "step") and kw["rope"] != "none":
        kw["axes"] = rng.choice([1, 1, 2, 3])
    if op in ("attend", "step"):
        kw["causal"] = kw["new"] == 1 or rng.random() < 0.7
    return _case(op, **kw)


# ------------------------------------------------------------------ inputs
def _sizes(case):
    """(cached, new) tokens of every sequence: a property of the case, so that every seed has the same work."""
    B = case["batch"]
    if not case["ragged"]:
        return [(case["cached"], case["new"])] * B
    g = torch.Generator().manual_seed(B * 10007 + case["cached"] * 31 + case["new"])
    cached = torch.randint(case["cached"] // 16, case["cached"] + 1, (B,), generator=g)
    new = torch.randint((case["new"] + 15) // 16, case["new"] + 1, (B,), generator=g)
    cached[B - 1], new[0] = case["cached"], case["new"]
    return list(zip(cached.tolist(), new.tolist()))


def _drafts(case):
    """The drafted tokens of every sequence."""
    B, n = case["batch"], case["drafts"]
    if not case["ragged"]:
        return [n] * B
    g = torch.Generator().manual_seed(B * 7919 + n)
    drafts = torch.randint(0, n + 1, (B,), generator=g)
    drafts[0] = n
    return drafts.tolist()


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _sections(case):
    """The pairs that each axis turns."""
    n = case["axes"]
    return [32 - (n - 1) * (32 // (n + 1))] + [32 // (n + 1)] * (n - 1) if n > 1 else [32]


def _order():
    """Where a page keeps token t, dimension d: the bytes of its key and value code, and of the token's two scales."""
    t, d = torch.arange(PAGE, device=DEV)[:, None], torch.arange(D, device=DEV)[None]
    k = t * 32 + d // 2
    v = t // 32 * 1024 + d // 4 * 64 + t // 4 % 4 * 16 + t // 16 % 2 * 8 + t % 4 * 2 + d % 4 // 2
    t = t[:, 0]
    return k, v, t % 16 * 4 + t // 16, 64 + t // 4 % 4 * 16 + t // 16 * 4 + t % 4


def _hadamard(x):
    """x [..., 64] times the Hadamard matrix over 8: sums and differences of entries 1, 2, .. 32 apart, in this order."""
    for step in (1, 2, 4, 8, 16, 32):
        a, b = x.unflatten(-1, (D // 2 // step, 2, step)).unbind(-2)
        x = torch.stack([a + b, a - b], -2).flatten(-3)
    return x * 0.125


def _exponents(x):
    """For vectors x [..., 64] the least E with max|x| <= 6 * 2^E, within [E_MIN, E_MAX]."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)                                                # amax = m 2^e with m in [1/2, 1)
    e = torch.where(amax > 0, e - 3 + (m > 0.75).int(), torch.full_like(e, E_MIN))
    return e.clamp(E_MIN, E_MAX)


def _codes(x, e):
    """e2m1 codes of x / 2^e, to nearest, ties to the even code, saturated."""
    y = torch.ldexp(x, -e[..., None])
    size = y.abs()
    code = torch.zeros_like(size, dtype=torch.uint8)
    for edge, tie_up in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (size >= edge) if tie_up else (size > edge)
    return code | (torch.signbit(y).to(torch.uint8) << 3)


def _quantized(x):
    x = _hadamard(x)
    e = _exponents(x)
    return _codes(x, e), (e + 127).to(torch.uint8)


def _values(codes, scales, at_code, at_scale):
    """What pages hold, fp32 [..., 64 tokens, 64]: codes [..., 2048] and scales [..., 128]."""
    nibble = (codes[..., at_code] >> (torch.arange(D, device=DEV, dtype=torch.uint8) % 2 * 4)) & 15
    lut = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=DEV)
    return torch.ldexp(lut[nibble.long()], scales[..., at_scale].int()[..., None] - 127)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 29)
    return _prepare_verify(case, g) if case["op"] == "verify" else _prepare_cache(case, seed, g)


def _prepare_verify(case, g):
    B, V, dtype = case["batch"], case["vocab"], DTYPES[case["dtype"]]
    drafts = torch.tensor(_drafts(case), device=DEV)
    row0 = torch.cumsum(torch.cat([drafts.new_zeros(1), drafts + 1]), 0).to(torch.int32)
    rows = int(sum(_drafts(case))) + B
    logits = 3.0 * torch.randn((rows, V), generator=g, device=DEV)
    s = {"case": case, "rows": rows, "row0": row0, "target": torch.softmax(logits, -1).to(dtype)}
    # what a smaller model makes of the same contexts, and the tokens that it drew (each row's is the one before its own)
    guess = torch.softmax(logits + 0.8 * torch.randn((rows, V), generator=g, device=DEV), -1).to(dtype)
    s["draft"] = guess if case["draft"] else None
    drawn = torch.multinomial(guess.float(), 1, generator=g)[:, 0] if case["draft"] else s["target"].float().argmax(-1)
    s["tokens"] = torch.cat([torch.randint(0, V, (1,), generator=g, device=DEV), drawn[:-1]])
    s["uniform"] = torch.rand(rows, generator=g, device=DEV)
    s["uniform_next"] = torch.rand(B, generator=g, device=DEV)
    s["seq_len"] = (torch.randint(20, 2000, (B,), generator=g, device=DEV) + drafts + 1).to(torch.int32)
    s["max_drafts"] = max(_drafts(case))
    if own:
        from paper_2603_26110_amd import serve
        need = serve.verify_workspace_bytes(V, B)
        s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=DEV) if need else None
    return s


def _prepare_cache(case, seed, g):
    L, H, Hkv, B = case["layers"], case["heads"], case["kv_heads"], case["batch"]
    dtype, op = DTYPES[case["dtype"]], case["op"]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed * 7 + 1)).tolist()
    sizes = [_sizes(case)[i] for i in order]
    cached = torch.tensor([c for c, _ in sizes], dtype=torch.int32, device=DEV)
    new = torch.tensor([n for _, n in sizes], dtype=torch.int32, device=DEV)
    rows = sum(n for _, n in sizes)
    longest = max(c + n for c, n in sizes)
    s = {"case": case, "rows": rows, "max_new": max(n for _, n in sizes), "max_len": longest}
    b = torch.repeat_interleave(torch.arange(B, device=DEV), new.long())
    row0 = torch.cumsum(torch.cat([new.new_zeros(1), new]), 0).to(torch.int32)
    s["pos"] = (torch.arange(rows, device=DEV) - row0[b] + cached[b]).to(torch.int32)
    s["row0"], s["seq_len"] = row0, cached + new
    # the new rows, as one projection leaves them: queries, keys and values of a token side by side
    loud = torch.argsort(torch.rand((L, 1, Hkv, D), generator=g, device=DEV), -1)[..., :4]
    gain = torch.ones((L, 1, Hkv, D), device=DEV).scatter_(-1, loud, 20.0)  # (four channels of a key head are loud)
    qkv = torch.randn((L, rows, H + 2 * Hkv, D), generator=g, device=DEV)
    qkv[:, :, H:H + Hkv] *= gain
    s["qkv"] = qkv.to(dtype)
    del qkv
    parts = (s["qkv"][:, :, :H], s["qkv"][:, :, H:H + Hkv], s["qkv"][:, :, H + Hkv:])
    s["q"], s["k"], s["v"] = [t.contiguous() for t in parts] if op in ("store", "attend") else parts
    # cos and sin of position p, pair m: p * 10000^(-2m/64), from double precision
    ang = torch.arange(longest, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (
        -2.0 * torch.arange(D // 2, dtype=torch.float64, device=DEV) / D)
    s["cs"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous() if case["rope"] != "none" else None
    normed = op in ("norm", "step")
    if normed:
        # the first axis counts on, the others stay within a picture's width
        s["axes"] = torch.stack([s["pos"] if a == 0 else s["pos"] // 24 ** (a - 1) % 24 for a in range(case["axes"])])
        s["axes"] = s["axes"].clamp(max=longest - 1).to(torch.int32).contiguous()
        s["q_weight"], s["k_weight"] = 0.5 + torch.rand((2, L, D), generator=g, device=DEV)
    if op != "norm":
        used = [_pages(c + n) for c, n in sizes]
        pages = sum(used) + max(4, sum(used) // 8)
        perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        owner = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(used, device=DEV))
        first = torch.cumsum(torch.tensor([0] + used, device=DEV), 0)
        table = torch.full((B, _pages(longest)), -1, dtype=torch.int32, device=DEV)
        table[owner, torch.arange(sum(used), device=DEV) - first[owner]] = perm[:sum(used)]
        s["table"], s["pages"] = table, pages
        s["slots"] = table[b, s["pos"].long() // PAGE].long() * PAGE + s["pos"].long() % PAGE
        # what the pages hold: keys as they are after RoPE, heavy-tailed values
        at = _order()
        planes, scales = [], torch.empty((L, Hkv, pages, 2 * PAGE), dtype=torch.uint8, device=DEV)
        for which in (0, 1):
            x = torch.randn((L, Hkv, pages, PAGE, D), generator=g, device=DEV)
            if which:
                x /= torch.randn((4, L, Hkv, pages, PAGE, 1), generator=g, device=DEV).square().mean(0).sqrt()
            else:
                x *= gain[:, 0, :, None, None]
            code, scale = _quantized(x)
            del x
            plane = torch.empty((L, Hkv, pages, PAGE * D // 2), dtype=torch.uint8, device=DEV)
            plane[..., at[which][:, ::2]] = code[..., ::2] | (code[..., 1::2] << 4)
            scales[..., at[2 + which]] = scale
            planes.append(plane)
        s["k_codes"], s["v_codes"], s["scales"] = *planes, scales
    if own:
        from paper_2603_26110_amd import paged, serve
        flags = paged.ROPE_HALF if case["rope"] == "half" else 0
        s["params"] = paged.Params(L, H, Hkv, rope_cs=s["cs"], io_dtype=dtype, flags=flags, softmax_scale=0.125)
        # (where q and k come rotated, what follows has no table)
        s["after"] = paged.Params(L, H, Hkv, io_dtype=dtype, softmax_scale=0.125) if normed else s["params"]
        if op != "norm":
            s["cache"] = serve.Cache4(L, Hkv, pages, buffers=(s["k_codes"], s["v_codes"], s["scales"]))
            need = serve.workspace_bytes(s["params"], L, B, s["max_new"], s["max_len"])
            s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=DEV) if need else None
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2603_26110_amd import serve
    op = s["case"]["op"]
    if op == "verify":
        return serve.verify(s["target"], s["draft"], s["tokens"], s["row0"], s["uniform"], s["uniform_next"],
                            seq_len=s["seq_len"], workspace=s["workspace"])
    q, k, out = s["q"], s["k"], []
    if op in ("norm", "step"):
        q, k = serve.norm_rope(s["params"], q, k, s["axes"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                               sections=_sections(s["case"]))
    if op == "norm":
        return [q, k]
    if op in ("store", "step"):
        serve.append(s["after"], s["cache"], k, s["v"], s["slots"], s["pos"])
    if op == "store":
        return serve.read(s["after"], s["cache"], s["slots"])
    return serve.attend(s["after"], s["cache"], q, s["pos"], s["row0"], s["table"], s["seq_len"], s["max_new"],
                        s["max_len"], causal=s["case"]["causal"], workspace=s["workspace"])


def _plain(s):
    op = s["case"]["op"]
    if op == "verify":
        return _verify_plain(s)
    if op == "norm":
        return _norm_plain(s)
    if op == "store":
        _append_plain(s, _rotated(s["k"].float(), s["cs"], s["pos"], s["case"]["rope"]))
        return _read_plain(s)
    if op == "attend":
        return _attend_plain(s, _rotated(s["q"].float(), s["cs"], s["pos"], s["case"]["rope"]))
    q, k = _norm_plain(s)
    _append_plain(s, k.float())
    return _attend_plain(s, q.float())


def _turned(x, c, n, rope):
    """Pairs of x [L, rows, heads, 64] turned by cos and sin [rows, 1, 32]."""
    if rope == "half":
        a, b = x[..., :32], x[..., 32:]
        return torch.cat([a * c - b * n, a * n + b * c], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2)


def _rotated(x, cs, pos, rope):
    return x if rope == "none" else _turned(x, cs[pos.long(), :, 0][:, None], cs[pos.long(), :, 1][:, None], rope)


def _norm_plain(s):
    case, out = s["case"], []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight[:, None, None]
        if case["rope"] != "none":
            pair = torch.arange(32, device=DEV)
            axis = torch.repeat_interleave(torch.arange(case["axes"], device=DEV), torch.tensor(_sections(case), device=DEV))
            angle = s["cs"][s["axes"].long()[axis].T, pair][:, None]        # [rows, 1, 32, 2]
            y = _turned(y, angle[..., 0], angle[..., 1], case["rope"])
        out.append(y.to(x.dtype))
    return out


def _append_plain(s, k):
    at = _order()
    page, token = s["slots"] // PAGE, s["slots"] % PAGE
    for x, plane, which in ((k, s["k_codes"], 0), (s["v"].float(), s["v_codes"], 1)):
        code, scale = _quantized(x.transpose(1, 2))                         # [L, Hkv, rows, 64]
        plane[:, :, page[:, None], at[which][token][:, ::2]] = code[..., ::2] | (code[..., 1::2] << 4)
        s["scales"][:, :, page, at[2 + which][token]] = scale


def _read_plain(s):
    at, out = _order(), []
    page, token = s["slots"] // PAGE, s["slots"] % PAGE
    lut = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=DEV)
    for plane, which in ((s["k_codes"], 0), (s["v_codes"], 1)):
        nibble = (plane[:, :, page[:, None], at[which][token]] >> (torch.arange(D, device=DEV, dtype=torch.uint8) % 2 * 4)) & 15
        x = torch.ldexp(lut[nibble.long()], s["scales"][:, :, page, at[2 + which][token]].int()[..., None] - 127)
        out.append(_hadamard(x).transpose(1, 2).to(DTYPES[s["case"]["dtype"]]).contiguous())
    return out


def _attend_plain(s, q):
    case, table = s["case"], s["table"].long().clamp(min=0)
    L, H, Hkv, B = case["layers"], case["heads"], case["kv_heads"], case["batch"]
    N, n, T, G = s["rows"], s["max_new"], s["max_len"], case["heads"] // case["kv_heads"]
    at = _order()
    j = torch.arange(T, device=DEV)
    # keys and values as the pages hold them, in the Hadamard basis, where queries meet them
    k, v = [_values(plane[:, :, table], s["scales"][:, :, table], at[which], at[2 + which]).flatten(-3, -2)[..., :T, :]
            for plane, which in ((s["k_codes"], 0), (s["v_codes"], 1))]     # [L, Hkv, B, T, 64]
    q = _hadamard(q)
    # rows padded to the most that a sequence has
    new = s["row0"].diff().long()
    i = torch.arange(n, device=DEV)
    inside = i < new[:, None]                                               # [B, n]
    row = (s["row0"][:-1].long()[:, None] + i).clamp(max=N - 1)
    qp = q[:, row].view(L, B, n, Hkv, G, D).permute(0, 3, 1, 4, 2, 5).reshape(L, Hkv, B, G * n, D)
    logits = torch.matmul(qp, k.transpose(-1, -2).contiguous()) * 0.125
    del k, qp
    seen = (j < s["seq_len"][:, None])[:, None].expand(B, n, T)
    if case["causal"]:
        seen = seen & (j <= s["pos"][row][..., None])
    logits = logits.view(L, Hkv, B, G, n, T).masked_fill_(~seen[:, None], float("-inf"))
    logits -= logits.amax(-1, keepdim=True).clamp(min=-3e38)
    weights = logits.exp_()
    total = weights.sum(-1, keepdim=True)
    # (what lies behind a sequence has a weight of zero)
    out = torch.matmul(weights.view(L, Hkv, B, G * n, T), v.contiguous()).view(L, Hkv, B, G, n, D) / total
    out = _hadamard(out).permute(0, 2, 4, 1, 3, 5).reshape(L, B, n, H, D)[:, inside]
    return out.to(DTYPES[case["dtype"]])


def _verify_plain(s):
    """In 64 bits: the products and differences of the given probabilities are exact there, and sums that a border is
    looked for in do not move it."""
    row0, drafts = s["row0"].long(), s["row0"].diff().long() - 1
    n = max(s["max_drafts"], 1)
    i = torch.arange(n, device=DEV)
    there = i < drafts[:, None]                                             # [B, n]
    row = torch.where(there, row0[:-1, None] + i, 0)
    token = s["tokens"][torch.where(there, row + 1, 0)]
    p = s["target"][row, token].double()
    q = s["draft"][row, token].double() if s["draft"] is not None else torch.ones_like(p)
    good = there & (s["uniform"][row].double() * q < p)
    accepted = torch.cumprod(good.int(), 1).sum(1)
    at = row0[:-1] + accepted                                               # the row whose token is drawn anew
    p = s["target"][at].double()
    rejected = (accepted < drafts)[:, None]
    drafted = s["tokens"][torch.where(rejected[:, 0], at + 1, 0)]
    q = s["draft"][at].double() if s["draft"] is not None else torch.zeros_like(p).scatter_(1, drafted[:, None], 1.0)
    rest = torch.where(rejected, (p - q).clamp(min=0.0), p)
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, p)
    upto = torch.cumsum(rest, -1)
    # the first token up to which there is more than the given share
    token = (upto <= s["uniform_next"].double()[:, None] * upto[:, -1:]).sum(-1)
    return [accepted.int(), token, (s["seq_len"] - drafts + accepted).int()]


# ------------------------------------------------------------------ work
def work(case):
    """Bytes and operations that a pass cannot do without."""
    io = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "verify":
        # a row of the target for each sequence, and one of the draft where a token is rejected: of the
        # drafted tokens 0.72 are kept, by the distance that prepare() puts between the two
        kept = sum(0.72 ** n for n in _drafts(case))
        rows = case["batch"] + (case["batch"] - kept if case["draft"] else 0.0)
        return {"bytes": rows * case["vocab"] * io + (sum(_drafts(case)) + case["batch"]) * 24,
                "flops": 3 * rows * case["vocab"]}
    sizes = _sizes(case)
    L, H, Hkv, op = case["layers"], case["heads"], case["kv_heads"], case["op"]
    rows = sum(n for _, n in sizes)
    rope = 0 if case["rope"] == "none" else rows * D * 4
    b = f = 0
    if op in ("norm", "step"):
        b += L * (H + Hkv) * rows * 2 * D * io + rope * case["axes"]
        f += L * (H + Hkv) * rows * 8 * D
    if op in ("store", "step"):
        b += L * Hkv * rows * (2 * D * io + D + 2) + rope + rows * 12
        f += L * Hkv * rows * 24 * D
    if op == "store":
        b += L * Hkv * rows * (2 * D * io + D + 2) + rows * 8
        f += L * Hkv * rows * 16 * D
    if op in ("attend", "step"):
        held = sum(c + n for c, n in sizes)
        pairs = sum(n * c + (n * (n + 1) // 2 if case["causal"] else n * n) for c, n in sizes)
        b += L * Hkv * held * (D + 2) + L * H * rows * D * 2 * io + rope + rows * 4
        f += L * H * pairs * 4 * D
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ the definition, in 64 bits
def _hadamard64(x):
    """x [..., 64] times the matrix of the signs (-1)^(bits that i and j share), over 8."""
    i = torch.arange(D, device=DEV)
    shared = i[:, None] & i
    parity = sum((shared >> b) & 1 for b in range(6)) % 2
    return x @ ((1.0 - 2.0 * parity).double() / 8.0)


def _turned64(x, theta, rope):
    """theta: the angles, fp64 [rows, 32]."""
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), theta)[:, None]
    if rope == "half":
        w = torch.complex(x[..., :32].contiguous(), x[..., 32:].contiguous()) * z
        return torch.cat([w.real, w.imag], -1)
    w = torch.view_as_complex(x.reshape(*x.shape[:-1], 32, 2).contiguous()) * z
    return torch.view_as_real(w).reshape(x.shape)


def _freq64():
    return 10000.0 ** (-torch.arange(32, dtype=torch.float64, device=DEV) / 32.0)


def _held64(x):
    """The values that a vector is held as: (multiples of a power of two in the e2m1 grid), in the Hadamard basis."""
    x = _hadamard64(x)
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 6.0)).clamp(E_MIN, E_MAX)
    y = x / torch.exp2(e)
    size = y.abs()
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=1.0))) - 1)
    return (torch.round(size / step) * step).clamp(max=6.0) * torch.sign(y) * torch.exp2(e)


def _pages64(s, which):
    """Values of a plane by page and token, fp64 [L, Hkv, pages, 64, 64], read nibble by nibble."""
    planes, scales = (s["k_codes"], s["v_codes"])[which], s["scales"]
    table = torch.tensor([m * sign for sign in (1.0, -1.0) for m in E2M1], dtype=torch.float64, device=DEV)
    out = torch.empty((*planes.shape[:3], PAGE, D), dtype=torch.float64, device=DEV)
    for t in range(PAGE):
        i, g, r = t // 16, t // 4 % 4, t % 4
        if which == 0:
            held = planes[..., 32 * t:32 * t + 32]
            e = scales[..., 4 * (t % 16) + i]
        else:
            held = planes[..., 1024 * (i // 2):1024 * (i // 2) + 1024].unflatten(-1, (16, 4, 2, 4, 2))[..., g, i % 2, r, :].flatten(-2)
            e = scales[..., 64 + 16 * g + 4 * i + r]
        both = torch.stack([held % 16, held // 16], -1).flatten(-2).long()
        out[..., t, :] = table[both] * torch.exp2(e.double() - 127.0)[..., None]
    return out


def exact(case, seed):
    if case["op"] == "verify":
        return None                                                         # whole numbers, which run() gives in full
    s = prepare(case, seed)
    L, H, Hkv, B, G = case["layers"], case["heads"], case["kv_heads"], case["batch"], case["heads"] // case["kv_heads"]
    op, rope = case["op"], case["rope"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    if op in ("norm", "step"):
        axis = [a for a, n in enumerate(_sections(case)) for _ in range(n)]
        theta = torch.stack([s["axes"][a].double() for a in axis], -1) * _freq64()
        done = []
        for x, weight in ((q, s["q_weight"]), (k, s["k_weight"])):
            x = x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * weight.double()[:, None, None]
            done.append(x if rope == "none" else _turned64(x, theta, rope))
        if op == "norm":
            return done
        # (the step hands them on in their own type)
        q, k = [x.to(s["q"].dtype).double() for x in done]
    elif rope != "none":
        theta = s["pos"].double()[:, None] * _freq64()
        q, k = _turned64(q, theta, rope), _turned64(k, theta, rope)
    if op == "store":
        return [_hadamard64(_held64(k)), _hadamard64(_held64(v))]
    kp, vp = _pages64(s, 0), _pages64(s, 1)
    if op == "step":
        page, token = s["slots"] // PAGE, s["slots"] % PAGE
        kp[:, :, page, token] = _held64(k).transpose(1, 2)
        vp[:, :, page, token] = _held64(v).transpose(1, 2)
    q = _hadamard64(q)
    res = torch.empty((L, s["rows"], H, D), dtype=torch.float64, device=DEV)
    row0, lens = s["row0"].tolist(), s["seq_len"].tolist()
    for b in range(B):
        n, T = row0[b + 1] - row0[b], lens[b]
        ids = s["table"][b, :_pages(T)].long()
        for l in range(L):
            kb = kp[l][:, ids].reshape(Hkv, -1, D)[:, :T]
            vb = vp[l][:, ids].reshape(Hkv, -1, D)[:, :T]
            qb = q[l, row0[b]:row0[b + 1]].transpose(0, 1).reshape(Hkv, G * n, D)
            a = (qb @ kb.transpose(1, 2).contiguous() / 8.0).view(Hkv, G, n, T)
            if case["causal"]:
                later = torch.arange(T, device=DEV) > s["pos"][row0[b]:row0[b + 1], None]
                a = a.masked_fill(later, float("-inf"))
            w = torch.softmax(a, -1).view(Hkv, G * n, T)
            o = (w @ vb).view(Hkv, G, n, D)
            res[l, row0[b]:row0[b + 1]] = o.permute(2, 0, 1, 3).reshape(n, H, D)
    return _hadamard64(res)
