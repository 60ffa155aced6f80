"""The 4-bit cache's operators where scores and scales leave the ordinary, and every launch that their rules choose."""
import math

import numpy as np
import pytest
import torch

import paged_ref
import serve_ref as ref
import paper_2603_26110_amd as tq
from paper_2603_26110_amd import paged, serve
from test_gpu_serve import (BF16, DEV, F16, F32, angles, check_attend, check_norm, check_verify, gen, i32, i64, layout,
                            random_cache, rows_of)

pytestmark = pytest.mark.gpu

# Every launch of attention: (layers, kv heads, group, lengths, new rows). Up to 64 rows a unit (new * group): tiles of 1, 4 and 16
# rows, each with four waves a block, eight, one (2048 units of eight pages at most), splits of eight waves, and
# splits of four (65 to 128 units of 64 pages and more); then more rows: blocks of 64 without and with splits, and of 128.
TILES = {"1": (1, 1), "4": (1, 3), "16": (3, 2)}
FEW = {f"{name}_{tile}": (L, H, G, lens, [new] * len(lens))
       for tile, (G, new) in TILES.items()
       for name, (L, H, lens) in {"four_waves": (1, 2, [300, 70, 5]), "eight_waves": (2, 2, [1025, 400]), "one_wave": (8, 33, [100 + i for i in range(8)]),
                                  "splits": (1, 2, [4500]), "four_wave_splits": (1, 8, [4200 + i for i in range(9)])}.items()}
MANY = {"many_64": (1, 2, 1, [300, 90], [70, 66]), "many_splits": (1, 1, 1, [7000], [100]), "many_128": (4, 12, 1, [130] * 16, [100] * 16)}
ALL = {**FEW, **MANY}


def weight_eps(case, kind):
    """What the kernel that runs leaves of a weight, by the result's type."""
    few = max(case[4]) * case[2] <= 64
    return {F16: 2.0 ** -11 if few else 2.0 ** -16, BF16: 2.0 ** -11 if few else 2.0 ** -8, F32: 2.0 ** -22}[kind]


def test_the_cases_are_those_launches():
    # (the rules say where there are splits by the workspace that they need)
    for name, (L, H, G, lens, news) in ALL.items():
        need = serve.workspace_bytes(paged.Params(L, H * G, H), L, len(lens), max(news), max(lens))
        assert (need > 0) == ("splits" in name), name
        units = L * H * len(lens) * math.ceil(news[0] * G / (16 if news[0] * G > 4 else news[0] * G))
        if name.startswith("one_wave"):
            assert units >= 2048 and max(lens) <= 512
        if name.startswith("four_wave_splits"):
            assert 65 <= units <= 128 and min(lens) > 64 * 63
        if name.startswith("splits"):
            assert units <= 64


@pytest.mark.parametrize("dtype,rope,fp32_out", [(F16, "pairs", False), (BF16, "half", False), (F32, "none", False)])
@pytest.mark.parametrize("name", list(FEW))
def test_attend_every_launch(name, dtype, rope, fp32_out, monkeypatch):
    # with what the kernel for up to 64 rows leaves of a query and a weight, and bounds below what the weighted values add up to
    bound = ref.bound

    def tight(out, spread, size, reach, length, eps, kind):
        most = bound(out, spread, size, reach, length, (2.0 ** -22, weight_eps(FEW[name], kind)), kind)
        assert bool((most < spread).all())
        return most
    monkeypatch.setattr(ref, "bound", tight)
    out = check_attend(*FEW[name], dtype, rope, fp32_out=fp32_out, seed=len(name))
    assert bool(out.isfinite().all())


# ------------------------------------------------------------------ large scores
def put(cache, params, table, lens, k, v):
    slots = [table[b][t // 64] * 64 + t % 64 for b, n in enumerate(lens) for t in range(n)]
    serve.append(params, cache, k, v, i64(slots))


@pytest.mark.parametrize("kind", [F16, BF16, F32])
@pytest.mark.parametrize("power", [10, 15, 16, 20, 24, 28, 40])
@pytest.mark.parametrize("name", list(ALL))
def test_equal_scores_weigh_the_same_at_any_size(name, power, kind):
    # keys and queries of one channel: scores are +-2^power of which the sum over 64 products is exact, and the same for
    # all tokens but every fifth, whose key is half as long (its weight is zero from 2^10 on: exp(-512)). A row's result is
    # the mean of the values that the others have, whose scales lie 2^24 apart. With a negative query the shorter keys
    # have the larger scores.
    case = ALL[name]
    L, H, G, lens, news = case
    table, pos, row0, pages = layout(lens, news, 3)
    cache, params = serve.Cache4(L, H, pages), paged.Params(L, H * G, H, None, F32 if kind is F32 else kind, 0, 2.0 ** (power - 20))
    n, rows = sum(lens), row0[-1]
    g = np.random.default_rng(power)
    short = torch.tensor(([False] * 4 + [True]) * n, device=DEV)[:n]
    k, v = torch.zeros((L, n, H, 64), device=DEV), torch.zeros((L, n, H, 64), device=DEV)
    k[..., 9] = torch.where(short, 2.0 ** 9, 2.0 ** 10)[None, :, None]
    size = torch.tensor(2.0 ** g.integers(-12, 13, (L, n, H)), dtype=F32, device=DEV)
    v.scatter_(-1, torch.tensor(g.integers(0, 64, (L, n, H, 1)), device=DEV), size[..., None])
    put(cache, params, table, lens, k.to(params.io_dtype), v.to(params.io_dtype))
    q = torch.zeros((L, rows, H * G, 64), device=DEV)
    sign = torch.where(torch.arange(rows, device=DEV) % 3 == 1, -1.0, 1.0)
    q[..., 9] = 2.0 ** 10 * sign[None, :, None]
    max_new, max_len = max(news), max(lens)
    room = torch.zeros(max(serve.workspace_bytes(params, L, len(lens), max_new, max_len), 1), dtype=torch.uint8, device=DEV)
    out = serve.attend(params, cache, q.to(params.io_dtype), i32(pos), i32(row0), i32(table), i32(lens), max_new, max_len, workspace=room)
    # Scores, exponents and weights are exact but for the exp2 (2^-22), the weight's rounding, and below 2^16 (of log2 e times the
    # score) one rounding of score and scale's exponent: half a step, 2^-24 relative. As in ref.bound with no error of a query's.
    # Sums of L1 norms: a value of one channel has entries of 1/8 of it in the other basis: spread is its size.
    score = 2.0 ** (power + 0.53)
    slack = math.log(2) * 2.0 ** -24 * score if score < 2.0 ** 16 else 0.0
    first = 0
    for b, length in enumerate(lens):
        vb, sb = v[:, first:first + length].double(), short[first:first + length]
        for r in {*range(row0[b], row0[b + 1], max(1, news[b] // 10)), row0[b + 1] - 1}:
            counts = (sb if sign[r] < 0 else ~sb).clone()
            counts[pos[r] + 1:] = False
            if not bool(counts.any()):             # (a short sequence in which nobody is longer)
                counts[:pos[r] + 1] = True
            want = vb[:, counts].mean(1).repeat_interleave(G, 1)
            spread = vb[:, counts].mean(1).sum(-1, keepdim=True).repeat_interleave(G, 1)
            zero = torch.zeros_like(spread)
            most = ref.bound(want, spread, zero, zero, length, (0.0, weight_eps(case, kind)), kind) + 2 * math.expm1(slack) * spread
            off = (out[:, r].double() - want).abs()
            assert bool((off <= most).all()), (b, r, float((off / most).max()))
        first += length


@pytest.mark.parametrize("io,fp32_out", [(BF16, False), (BF16, True), (F32, False)])
@pytest.mark.parametrize("name", ["four_waves_1", "eight_waves_4", "splits_16", "four_wave_splits_1", "one_wave_4", "many_64", "many_128"])
def test_one_key_decides(name, io, fp32_out):
    # keys of all sizes and scores of up to 2^46: where the largest score is far above the others, by more than what a query's
    # rounding, the sums in binary32 and the scales' range may hide, the result is that token's value (no fp16: up to 6 * 2^47)
    case = ALL[name]
    L, H, G, lens, news = case
    table, pos, row0, pages = layout(lens, news, 5)
    cache = random_cache(L, H, pages, 6, 79, 175)
    params = paged.Params(L, H * G, H, None, io, tq.OUT_FP32 if fp32_out else 0)
    q = rows_of((L, row0[-1], H * G, 64), 7, io)
    out = serve.attend(params, cache, q, i32(pos), i32(row0), i32(table), i32(lens), max(news), max(lens))
    kind = out.dtype
    k, v = (torch.from_numpy(x).to(DEV) for x in ref.CacheRef(cache).values())
    had = torch.tensor(ref.SIGNS / 8, device=DEV)
    few = max(news) * G <= 64
    part = 2.0 ** -22 if few or kind is not BF16 else 2.0 ** -11           # what is left of a query's entry
    asked = told = 0
    for b, n in enumerate(lens):
        kb, vb = (x[:, :, table[b][:paged_ref.pages_of(n)]].flatten(2, 3)[:, :, :n] for x in (k, v))
        for r in range(row0[b], row0[b + 1], max(1, news[b] // 4)):
            p = pos[r] + 1
            qr = (q[:, r].double() @ had).unflatten(1, (H, G))             # [L][H][G][64]
            s = (qr[:, :, :, None] * kb[:, :, None, :p]).sum(-1) * 0.125 / math.log(2)
            size = (qr.abs()[:, :, :, None] * kb.abs()[:, :, None, :p]).sum(-1).amax(-1) * 0.125 / math.log(2)
            if p > 1:
                top, at = s.topk(2, -1)
                # (both scores off by the query's rounding and 200 roundings of binary32; then 2^-60 of values 2^95 apart)
                sure = top[..., 0] - top[..., 1] > 2 * (part + 200 * 2.0 ** -24) * size + 95 + 60
                at = at[..., 0]
            else:
                sure, at = torch.ones_like(size, dtype=torch.bool), torch.zeros_like(size, dtype=torch.long)
            held = torch.gather(vb, 2, at[..., None].expand(*at.shape, 64))
            want, spread = held @ had, held.abs().sum(-1, keepdim=True) / 8
            zero = torch.zeros_like(spread)
            most = ref.bound(want, spread, zero, zero, n, (0.0, weight_eps(case, kind)), kind)
            assert bool((most.isfinite() & (most <= spread + 1)).all())    # (zeros would not pass, but for the least values)
            off = (out[:, r].unflatten(1, (H, G)).double() - want).abs()
            assert bool((off <= most)[sure].all()), (b, r, float((off / most)[sure].max()))
            asked, told = asked + sure.numel(), told + int(sure.sum())
    assert told >= asked / 2, (told, asked)


# ------------------------------------------------------------------ keys far apart
@pytest.mark.parametrize("dtype,fp32_out", [(F16, False), (BF16, False), (BF16, True), (F32, False)])
@pytest.mark.parametrize("gap", [30, 36, 37, 60])
@pytest.mark.parametrize("L,H,B,new", [(1, 1, 2, 170), (4, 12, 16, 170), (1, 1, 2, 2)])
def test_small_keys_beside_large_ones(L, H, B, new, gap, dtype, fp32_out):
    # the last tokens of the second page (of few-row calls: the last of all) have keys 2^gap times as large as the others, in
    # blocks of 64 rows, of 128 and of few: rows that do not see them keep all digits, on this page and the one before
    n = 170
    lens, news = [n] * B, [new] * B
    table, pos, row0, pages = layout(lens, news, 3)
    cache = random_cache(L, H, pages, 4, 120, 124)
    large = [126, 127] if new > 2 else [169]
    for b in range(B):
        for t in large:
            cache.scales[:, :, table[b][t // 64], int(ref.KEY_SCALE[t % 64])] = 122 + gap
    params = paged.Params(L, H, H, None, dtype, tq.OUT_FP32 if fp32_out else 0)
    q = rows_of((L, row0[-1], H, 64), 7, dtype, 2.0 ** -4)
    out = serve.attend(params, cache, q, i32(pos), i32(row0), i32(table), i32(lens), new, n)
    kind = out.dtype
    k, v = (torch.from_numpy(x).to(DEV) for x in ref.CacheRef(cache).values())
    had = torch.tensor(ref.SIGNS / 8, device=DEV)
    qeps = 2.0 ** -11 if kind is BF16 and new > 64 else 2.0 ** -22
    for b in range(B):
        kb, vb = (x[:, :, table[b]].flatten(2, 3)[:, :, :n] for x in (k, v))
        rows = [r for r in range(row0[b], row0[b + 1]) if pos[r] < large[0]]
        qb = q[:, rows].transpose(1, 2).double()                           # [L][H][rows][64]
        seen = torch.arange(n, device=DEV) <= i32([pos[r] for r in rows])[:, None]
        qh = qb @ had
        s = (torch.matmul(qh, kb.transpose(2, 3).contiguous()) * 0.125).masked_fill(~seen, -math.inf)
        size = (torch.matmul(qh.abs(), kb.abs().transpose(2, 3).contiguous()) * 0.125).masked_fill(~seen, 0).amax(-1, keepdim=True)
        reach = qb.abs().sum(-1, keepdim=True) / 8 * kb.abs().sum(-1)[:, :, None].masked_fill(~seen, 0).amax(-1, keepdim=True) * 0.125
        w = torch.softmax(s, -1)
        want, spread = torch.matmul(w, vb) @ had, torch.matmul(w, vb.abs()).sum(-1, keepdim=True) / 8
        most = ref.bound(want, spread, size, reach, n, (qeps, weight_eps((L, H, 1, lens, news), kind)), kind)
        off = (out[:, rows].transpose(1, 2).double() - want).abs()
        assert len(rows) == (126 if new > 2 else 1) and bool((most <= spread).all())
        assert bool((off <= most).all()), (b, float((off / most).max()))


# ------------------------------------------------------------------ verify
@pytest.mark.parametrize("vocab,B,pad,dtype", [(32_768, 170, 0, F32), (32_768, 170, 0, F16), (32_771, 200, 5, F16), (47_929, 153, 0, BF16)])
def test_verify_with_more_units_a_block(vocab, B, pad, dtype):
    # blocks take more than four units of 2048 entries from 2560 units on; rows that are aligned to 16 bytes, and not
    assert B * math.ceil(vocab / 2048) >= 2560
    g = np.random.default_rng(B)
    n = g.integers(0, 3, B)
    row0 = np.concatenate([[0], np.cumsum(n + 1)]).tolist()
    rows = row0[-1]
    wide = torch.zeros((2, rows, vocab + pad), dtype=dtype, device=DEV)
    # (a few entries of every row, the last among them: the exact sums that the draws are compared with go over these)
    at = torch.randint(0, vocab, (rows, 60), generator=gen(B), device=DEV)
    at[:, 0] = vocab - 1
    for x, seed in zip(wide, (1, 2)):
        x.scatter_(1, at, torch.rand((rows, 60), generator=gen(seed), device=DEV).to(dtype) / 32)
    target, draft = wide[0, :, :vocab], wide[1, :, :vocab]
    drawn = at[torch.arange(rows, device=DEV), torch.randint(0, 60, (rows,), generator=gen(5), device=DEV)].tolist()
    tokens = [0] + drawn[:-1]                                # (a draft has a probability in the row before it)
    for share in (0.2, 1.0):
        check_verify(target, draft, tokens, row0, (g.random(rows) * share).tolist(), g.random(B).tolist(), g.integers(20, 99, B).tolist())


# ------------------------------------------------------------------ norm_rope
@pytest.mark.parametrize("rope", ["none", "pairs", "half"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_over_the_range_of_its_squares(dtype, rope):
    # eps 0, heads whose largest entry is from 2^-60 to 2^60: their squares are binary32's (the lowest steps, 2^-149, are
    # 64 * 2^-150 of a sum of 2^-120, within its rounding), in rows of one call
    powers = [-60, -59, -40, 0, 40, 59, 60]
    x = rows_of((1, len(powers), 3, 64), 4, F32)
    x = (x / x.abs().amax(-1, keepdim=True)).double()
    x[..., 5] = 1.0
    x = (x * 2.0 ** torch.tensor(powers, dtype=torch.float64, device=DEV)[:, None, None]).to(dtype)
    cs = None if rope == "none" else tq.rope_table(9)
    params = paged.Params(1, 3, 3, cs, dtype, tq.ROPE_HALF if rope == "half" else 0)
    pos = i32([3] * len(powers))
    z = None if cs is None else angles(9)[pos.long()]
    for got in serve.norm_rope(params, x, x, pos, eps=0.0):
        check_norm(got, x, None, 0.0, z, rope == "half")


# ------------------------------------------------------------------ quality
def test_the_4_bit_cache_keeps_its_quality():
    # On these inputs exact attention over what the definition's codes hold (computed on the CPU in 64 bits) has a mean
    # cosine of 0.9219 and a relative error of 0.3819; the kernels' roundings are below 10^-3 of a result, and a code that
    # a rounding of RoPE turns over changes one of 64 entries of one of 256 tokens. The worst head is above the worst of the
    # 3-bit variants.
    from paper_2603_26110_amd import quality
    inp = quality.inputs(heads=4, tokens=256, calib=64, seed=7)
    r = quality.metrics(quality.decode_paged(inp, 4), inp["ref"])
    assert r["cos_mean"] > 0.9219 - 0.003 and r["rel_l2"] < 0.3819 + 0.005, r
    assert r["cos_min"] > min(x["cos_min"] for x in quality.run(heads=4, tokens=256, calib=1024, seed=7))
