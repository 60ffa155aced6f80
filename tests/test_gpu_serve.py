"""The operators around the paged 4-bit cache on the GPU against plain implementations (tests/serve_ref.py)."""
import numpy as np
import pytest
import torch

import paged_ref
import serve_ref as ref
import paper_2603_26110_amd as tq
from paper_2603_26110_amd import paged, serve

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
# By the result's type: a query's entry in fp16, one part (2^-11) or two (2^-22); a weight in fp16 or bf16, one part (2^-11, 2^-8) or
# more (fp32 results: 2^-22 at least)
EPS = {F16: (2.0 ** -22, 2.0 ** -11), BF16: (2.0 ** -11, 2.0 ** -8), F32: (2.0 ** -22, 2.0 ** -22)}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def random_cache(L, H, pages, seed, lo=115, hi=130):
    """A cache whose pages hold codes of all kinds and scales of bytes lo .. hi - 1."""
    g, c = gen(seed), serve.Cache4(L, H, pages)
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device=DEV))
    c.scales.copy_(torch.randint(lo, hi, c.scales.shape, generator=g, device=DEV))
    return c


def angles(n):
    """(cos, sin) of positions 0 .. n-1 in 64 bits, as complex numbers [n][32]."""
    m = torch.arange(32, dtype=torch.float64, device=DEV)
    t = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-m / 32)
    return torch.polar(torch.ones_like(t), t)


def rows_of(shape, seed, dtype, sizes=1.0, pad=0):
    """Random rows [L][rows][heads][64], as a slice of wider rows where pad > 0."""
    L, rows, H, _ = shape
    x = torch.randn((L, rows, H + pad, 64), generator=gen(seed), device=DEV) * sizes
    return x.to(dtype)[:, :, :H]


# ------------------------------------------------------------------ append and read
def same_bytes(cache, want):
    s = cache.scales.cpu().numpy()
    assert np.array_equal(s, want.s)
    for name, a, b, where, at in (("k", cache.k_codes, want.k, ref.KEY, ref.KEY_SCALE),
                                  ("v", cache.v_codes, want.v, ref.VALUE, ref.VALUE_SCALE)):
        a = a.cpu().numpy()
        fine = (s[..., at] != 255)[..., None]                # (codes of a key that is no number do not count)
        for x in (a, b):
            x[..., where[:, ::2]] = np.where(fine, x[..., where[:, ::2]], 0)
        assert np.array_equal(a, b), name


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rope", ["none", "pairs", "half"])
@pytest.mark.parametrize("L,H,rows,layer0,nl,pad", [(1, 1, 1, 0, 1, 0), (2, 3, 33, 1, 1, 0), (3, 2, 70, 0, 3, 3), (1, 5, 131, 0, 1, 1)])
def test_append_writes_the_nearest_codes(dtype, rope, L, H, rows, layer0, nl, pad):
    pages, positions = 4, 50
    cache = random_cache(L, H, pages, rows)
    want = ref.CacheRef(cache)
    g = np.random.default_rng(rows + L)
    slots = g.permutation(pages * 64)[:rows]                 # any order, every byte of a page by some row
    slots[g.random(rows) < 0.1] = -1
    if rows > 4:
        slots[:3] = [pages * 64, -2 ** 40, 2 ** 40]
    pos = g.integers(-2 if rows > 4 else 0, positions + (2 if rows > 4 else 0), rows)
    k, v = rows_of((nl, rows, H, 64), 1, dtype, 3.0, pad), rows_of((nl, rows, H, 64), 2, dtype, 0.02, pad)
    if rows > 8:
        k[0, 5, 0] *= 0
        v[0, 5, 0] *= 0
        k[0, 6, 0, 17], v[nl - 1, 7, H - 1, 63] = float("nan"), float("inf")
        k[0, 8, 0] = 60000.0                                 # (one entry after the butterflies: 480 000)
    cs = None if rope == "none" else tq.rope_table(positions)
    params = paged.Params(L, H, H, cs, dtype, tq.ROPE_HALF if rope == "half" else 0)
    serve.append(params, cache, k, v, i64(slots.tolist()), None if cs is None else i32(pos.tolist()), layer0=layer0)
    want.append(k.float().cpu().numpy(), v.float().cpu().numpy(), slots.tolist(), pos.tolist(),
                None if cs is None else cs.cpu().numpy(), rope == "half", layer0)
    same_bytes(cache, want)


def test_append_at_the_ends_of_the_range():
    # fp32 far above and below the scales, borders of exponents and codes, and sums that leave binary32
    rows = []
    for e in (-149, -126, -60, -51, -50, -49, -48, 0, 46, 47, 48, 49, 50, 60, 100, 121):
        for m in (1.0, 1.5, 1.5000001, 1.9999999):
            rows.append([m * 2.0 ** e] + [0.0] * 63)
    rows += [[2.0 ** 120] * 64, [3e38] * 64, [3e38, -3e38] * 32, [1e-45] * 64, [0.0] * 64, [-0.0] * 64]
    x = torch.tensor(rows, dtype=torch.float64).to(F32).to(DEV)[None, :, None]
    n = x.shape[1]
    for k, v in ((x, x.flip(1)), (x.flip(1), x)):
        cache = random_cache(1, 1, 2, 3)
        want = ref.CacheRef(cache)
        slots = list(range(n, 0, -1))
        serve.append(paged.Params(1, 1, 1, io_dtype=F32), cache, k.contiguous(), v.contiguous(), i64(slots))
        want.append(k.cpu().numpy(), v.cpu().numpy(), slots, [0] * n, None, False)
        same_bytes(cache, want)


@pytest.mark.parametrize("dtype,fp32_out", [(F16, False), (BF16, False), (F32, False), (BF16, True)])
@pytest.mark.parametrize("L,H,rows,layer0,nl", [(1, 1, 1, 0, None), (3, 2, 77, 1, 2), (2, 9, 40, 0, 1), (2, 3, 64, 1, None)])
def test_read_gives_what_the_cache_holds(dtype, fp32_out, L, H, rows, layer0, nl):
    pages = 3
    cache = random_cache(L, H, pages, rows)
    cache.scales[:, 0, 1, ref.KEY_SCALE[9]] = 255
    cache.v_codes[:, 0, 1, torch.from_numpy(ref.VALUE[9]).to(DEV)] = 0
    k, v = ref.CacheRef(cache).values()
    g = np.random.default_rng(rows)
    slots = g.integers(0, pages * 64, rows)                  # (the same one several times is fine here)
    if rows > 5:
        slots[:5] = [64 + 9, -1, pages * 64, 2 ** 33, 0]
    params = paged.Params(L, H, H, io_dtype=dtype, flags=tq.OUT_FP32 if fp32_out else 0)
    out = serve.read(params, cache, i64(slots.tolist()), layer0=layer0, nlayers=nl)
    nl = L - layer0 if nl is None else nl
    there = (slots >= 0) & (slots < pages * 64)
    s = np.where(there, slots, 0)
    for got, held in zip(out, (k, v)):
        want = ref.hadamard32(held[layer0:layer0 + nl, :, s // 64, s % 64]).transpose(0, 2, 1, 3).copy()
        want[:, ~there] = np.nan
        assert got.dtype == (F32 if fp32_out else dtype) and got.shape == (nl, rows, H, 64)
        assert np.array_equal(got.float().cpu().numpy(), torch.from_numpy(want).to(got.dtype).float().numpy(), equal_nan=True)
    again = tuple(torch.zeros_like(t) for t in out)
    assert serve.read(params, cache, i64(slots.tolist()), layer0=layer0, nlayers=nl, out=again)[0] is again[0]
    for a, b in zip(again, out):
        assert torch.equal(a.nan_to_num(7), b.nan_to_num(7))


def test_what_is_written_comes_back_close():
    # a vector's error is at most half a step of the largest binade in each of 64 entries of the Hadamard basis: steps
    # are up to 2 * 2^E where the largest entry is above 3 * 2^E, a third of it at most; the basis keeps the length
    x = rows_of((1, 64, 2, 64), 5, F32, 2.0)
    cache, params, slots = serve.Cache4(1, 2, 1), paged.Params(1, 2, 2, io_dtype=F32), i64(list(range(64)))
    serve.append(params, cache, x, x, slots)
    for y in serve.read(params, cache, slots):
        top = (x.double() @ torch.tensor(ref.SIGNS / 8, device=DEV)).abs().amax(-1)
        assert bool(((y - x).double().norm(dim=-1) <= 8 * top / 3 * 1.0001).all())
        assert float((y - x).norm() / x.norm()) < 0.2


# ------------------------------------------------------------------ attend
def layout(lens, news, seed, spare=3):
    """Pages of sequences of lens tokens, the last news of them new: (table, pos, row0, pages)."""
    g = np.random.default_rng(seed)
    used = [paged_ref.pages_of(n) for n in lens]
    pages = sum(used) + spare
    ids = g.permutation(pages).tolist()
    table, at = [], 0
    for u in used:
        table.append(ids[at:at + u] + [-1] * (max(max(used), 1) - u))
        at += u
    pos = [n - m + i for n, m in zip(lens, news) for i in range(m)]
    return table, pos, np.concatenate([[0], np.cumsum(news)]).tolist(), pages


def check_attend(L, H, G, lens, news, dtype, rope="none", causal=True, fp32_out=False, max_len=None, max_new=None, lo=115, hi=130,
                 scale=0.125, qsize=1.0, layer0=0, nl=None, seed=0, spoil=None):
    table, pos, row0, pages = layout(lens, news, seed + len(lens))
    nl = L if nl is None else nl
    cache = random_cache(L, H, pages, seed + 1, lo, hi)
    rows = row0[-1]
    q = rows_of((nl, rows, H * G, 64), seed + 2, dtype, qsize, pad=2)
    top = max(pos + [0]) + 1
    cs = None if rope == "none" else tq.rope_table(top)
    params = paged.Params(L, H * G, H, cs, dtype, (tq.ROPE_HALF if rope == "half" else 0) | (tq.OUT_FP32 if fp32_out else 0), scale)
    k, v = (torch.from_numpy(x[layer0:layer0 + nl]).to(DEV) for x in ref.CacheRef(cache).values())
    if spoil is not None:                                    # what no row may look at
        spoil(cache, table, lens)
    max_new, max_len = max_new or max(news + [1]), max_len or max(lens + [1])
    args = (params, cache, q, i32(pos), i32(row0), i32(table), i32(lens), max_new, max_len)
    need = serve.workspace_bytes(params, nl, len(lens), max_new, max_len)
    room = torch.zeros(need, dtype=torch.uint8, device=DEV) if need else None
    out = serve.attend(*args, causal=causal, layer0=layer0, workspace=room)
    want, spread, size, reach = ref.attend(k, v, q.double(), pos, row0, table, lens, causal, scale,
                                           None if cs is None else angles(top), rope == "half")
    kind = F32 if fp32_out else dtype
    assert out.dtype == kind and out.shape == q.shape
    off, most = (out.double() - want).abs(), ref.bound(want, spread, size, reach, max(lens), EPS[kind], kind)
    assert bool((off <= most).all()), (float((off - most).max()), float((off / most).max()))
    again = serve.attend(*args, causal=causal, layer0=layer0, workspace=room)
    assert torch.equal(out, again)                           # (the counters are zero again, and the order is fixed)
    if room is not None:
        assert not bool(room[:16384].any())
    return out


FEW = [  # layers, kv heads, group, lengths, new: eight waves, one, four; splits; tiles of 16 rows; odd groups
    (1, 1, 1, [1], [1]), (1, 2, 1, [64], [1]), (1, 2, 3, [65, 3], [1, 1]), (1, 3, 5, [200, 1, 63], [3, 1, 2]),
    (2, 4, 1, [1025], [1]), (1, 1, 8, [4500], [1]), (1, 1, 16, [3000, 4000], [4, 1]), (1, 2, 7, [700, 90, 130], [9, 5, 2]),
    (4, 8, 2, [100, 128, 1, 60, 90, 127, 5, 64], [1] * 8), (8, 33, 1, [40] * 8, [1] * 8), (8, 33, 1, [400 + i for i in range(8)], [1] * 8)]


@pytest.mark.parametrize("dtype,rope,fp32_out", [(F16, "pairs", False), (BF16, "half", False), (F32, "none", False),
                                                 (F16, "none", False), (F32, "pairs", False), (BF16, "pairs", True), (F16, "half", True)])
@pytest.mark.parametrize("case", FEW, ids=range(len(FEW)))
def test_attend_few_rows(case, dtype, rope, fp32_out):
    check_attend(*case, dtype, rope, fp32_out=fp32_out, seed=len(case[3]))


MANY = [  # 128-row blocks, 64-row blocks with two groups, splits; ragged; one row past a tile
    (1, 1, 1, [65], [65]), (1, 2, 5, [300, 40, 100], [30, 13, 20]), (1, 1, 8, [5000], [9]), (1, 1, 1, [7000], [100]),
    (1, 2, 2, [129, 257, 64], [129, 64, 1]), (6, 33, 1, [130] * 4, [130] * 4), (1, 3, 3, [600, 1, 300], [43, 1, 300])]


@pytest.mark.parametrize("dtype,rope,fp32_out,causal", [(F16, "pairs", False, True), (BF16, "half", False, True), (F32, "none", False, False),
                                                        (BF16, "none", False, False), (F32, "half", False, True), (F16, "pairs", True, True)])
@pytest.mark.parametrize("case", MANY, ids=range(len(MANY)))
def test_attend_many_rows(case, dtype, rope, fp32_out, causal):
    check_attend(*case, dtype, rope, causal=causal, fp32_out=fp32_out, seed=len(case[3]))


def test_attend_some_layers_and_loose_bounds():
    check_attend(3, 2, 2, [70, 300], [1, 4], F16, "pairs", layer0=1, nl=2, max_len=5000, max_new=10)
    check_attend(3, 2, 2, [70, 300], [1, 4], BF16, "half", layer0=2, nl=1, max_len=9000, max_new=200)


@pytest.mark.parametrize("news", [[1, 3], [100, 3]])
def test_attend_whatever_lies_behind_the_sequence(news):
    def spoil(cache, table, lens):
        for row, n in zip(table, lens):
            for t in range(n, 64 * paged_ref.pages_of(n)):
                at = [int(ref.KEY_SCALE[t % 64]), int(ref.VALUE_SCALE[t % 64])]
                cache.scales[:, :, row[t // 64], at] = 255 if t % 2 else 254
        used = {p for row in table for p in row}
        for p in range(cache.pages):
            if p not in used:
                cache.scales[:, :, p] = 255
    check_attend(1, 2, 1, [101, 64 + 3], news, F16, spoil=spoil, max_new=max(news))
    check_attend(1, 2, 1, [101, 64 + 3], news, BF16, spoil=spoil, causal=False, max_new=max(news))


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_attend_scales_of_all_sizes(new, dtype):
    # tokens side by side whose scales are anywhere in the range: values of 2^-48 and 2^47, scores up to 2^46 (one key
    # decides), and a range where many keys count
    check_attend(1, 2, 2, [300], [new], F32 if dtype is F32 else BF16, lo=79, hi=175, seed=5)
    check_attend(1, 2, 2, [300], [new], dtype, lo=100, hi=124, qsize=0.02, seed=6)
    check_attend(1, 2, 1, [200], [new], dtype, lo=124, hi=132, qsize=20.0, seed=7)     # scores in the thousands


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("gap", [30, 36, 37, 60])
def test_attend_small_keys_before_large_ones(new, gap):
    # the page's last tokens have keys 2^gap times as large as the others: rows that do not see them keep all digits
    n = 100
    table, pos, row0, pages = layout([n], [new], 3)
    cache = random_cache(1, 1, pages, 4, 120, 124)
    for t in (62, 63, 90, 99):
        cache.scales[0, 0, table[0][t // 64], int(ref.KEY_SCALE[t % 64])] = 122 + gap
    params = paged.Params(1, 1, 1, io_dtype=F32)
    q = rows_of((1, new, 1, 64), 7, F32, 2.0 ** -4)
    out = serve.attend(params, cache, q, i32(pos), i32(row0), i32(table), i32([n]), new, n)
    k, v = (torch.from_numpy(x).to(DEV) for x in ref.CacheRef(cache).values())
    for p in range(n - new, n):
        r = p - (n - new)
        w, spread, size, reach = ref.attend(k, v, q[:, r:r + 1].double(), [p], [0, 1], table, [p + 1], True, 0.125)
        off = (out[:, r:r + 1].double() - w).abs()
        assert bool((off <= ref.bound(w, spread, size, reach, n, EPS[F32], F32)).all()), p


@pytest.mark.parametrize("new,G", [(1, 3), (80, 1)])
def test_attend_a_small_value_beside_a_large_one(new, G):
    # the large value's key is never looked at (a score of -2^14 or so against 2^14): the small values keep their digits
    n, H = 128, 1
    table, pos, row0, pages = layout([n], [new], 3)
    cache = serve.Cache4(1, H, pages)
    params = paged.Params(1, G, H, io_dtype=F32)
    k, v = torch.zeros((1, n, H, 64), device=DEV), torch.zeros((1, n, H, 64), device=DEV)
    k[..., 0], v[..., 3] = 64.0, 1.5 * 2.0 ** -20
    k[0, 7, 0, 0], v[0, 7, 0, 3] = -64.0, 1.5 * 2.0 ** 40
    slots = [table[0][t // 64] * 64 + t % 64 for t in range(n)]
    serve.append(params, cache, k, v, i64(slots))
    q = torch.zeros((1, new, G, 64), device=DEV)
    q[..., 0] = 2048.0
    out = serve.attend(params, cache, q, i32(pos), i32(row0), i32(table), i32([n]), new, n, causal=False)
    want = torch.zeros_like(out)
    want[..., 3] = 1.5 * 2.0 ** -20
    # (every value is 1.5 * 2^-23 times a sign in the Hadamard basis, so that sums are exact but for the weights')
    assert bool(((out - want).abs() <= 1.5 * 2.0 ** -20 * 2.0 ** -17).all())


@pytest.mark.parametrize("many", [False, True])
def test_attend_rows_that_are_not_valid(many):
    new, H, G = (80, 2, 1) if many else (3, 2, 2)
    lens = [100, 90, 0, 200, 130, 100]
    news = [new, new, new, new, new, 0]
    table, pos, row0, pages = layout(lens, [n if m else 0 for n, m in zip(news, news)], 4)
    pos = [p if p >= 0 else 5 for p in pos]
    cache = random_cache(1, H, pages, 9)
    params = paged.Params(1, H * G, H, tq.rope_table(300), F16)
    rows = row0[-1] + 4                                      # (and four rows that no sequence has)
    q = rows_of((1, rows, H * G, 64), 1, F16)
    lens[3] = 260                                            # past max_len
    pos[row0[1]], pos[row0[1] + 1] = -1, 300
    pos += [3] * 4
    bad = [list(r) for r in table]
    bad[4][1] = pages                                        # the second page of a sequence: rows that see it
    pos[row0[4]] = 40                                        # ... this one does not
    q[0, row0[0] + 1, 0, 5] = float("inf")
    out = torch.full(q.shape, 7.0, dtype=F16, device=DEV)
    serve.attend(params, cache, q, i32(pos), i32(row0), i32(bad), i32(lens), new, 200, out=out)
    nan = out.isnan().all(-1)[0]
    want = torch.zeros_like(nan)
    want[row0[0] + 1, 0] = True
    want[row0[1]] = want[row0[1] + 1] = True
    want[row0[3]:row0[4]] = True
    want[row0[4] + 1:row0[5]] = i32(pos[row0[4] + 1:row0[5]])[:, None] >= 64
    assert torch.equal(nan, want) and bool((out[0, row0[-1]:] == 7).all())
    assert bool((out[0, row0[2]:row0[3]] == 0).all())        # nothing to see
    assert not bool(out.isnan().any(-1)[0][~want].any())
    good = [r for r in [*range(row0[2]), *range(row0[4], row0[5])] if not bool(want[r].any())]
    k, v = (torch.from_numpy(x).to(DEV) for x in ref.CacheRef(cache).values())
    lens[3] = 0
    ref_q = q.double().nan_to_num(0, 0, 0)
    w, spread, size, reach = ref.attend(k, v, ref_q, [max(p, 0) % 300 for p in pos], row0, table, lens, True, 0.125, angles(300))
    most = ref.bound(w, spread, size, reach, 200, EPS[F16], F16)
    assert bool(((out.double() - w).abs() <= most)[0, good].all())


@pytest.mark.parametrize("new", [2, 90])
def test_attend_keys_that_are_no_numbers(new):
    n = 100
    table, pos, row0, pages = layout([n, n], [new, new], 8)
    cache, params = serve.Cache4(1, 1, pages), paged.Params(1, 1, 1, io_dtype=F32)
    k = rows_of((1, 2 * n, 1, 64), 1, F32)
    v = rows_of((1, 2 * n, 1, 64), 2, F32)
    v[0, n - 1, 0, 3] = float("nan")                         # the first sequence's last token
    k[0, 2 * n - 2, 0, 60] = float("-inf")                   # the second's last but one
    slots = [table[b][t // 64] * 64 + t % 64 for b in range(2) for t in range(n)]
    serve.append(params, cache, k, v, i64(slots))
    q = rows_of((1, 2 * new, 1, 64), 3, F32)
    out = serve.attend(params, cache, q, i32(pos), i32(row0), i32(table), i32([n, n]), new, n)
    nan = out.isnan().all(-1)[0, :, 0].tolist()
    assert nan == [p >= (n - 1 if r < new else n - 2) for r, p in enumerate(pos)]
    assert torch.equal(out.isnan().any(-1), out.isnan().all(-1))


def test_attend_rows_that_are_no_sequence_s():
    cache = random_cache(1, 1, 3, 2)
    params = paged.Params(1, 1, 1)
    q = rows_of((1, 6, 1, 64), 1, F16)
    out = torch.full(q.shape, 3.0, dtype=F16, device=DEV)
    # before the first, decreasing, past the rows
    serve.attend(params, cache, q, i32([5] * 6), i32([2, 3, 1, 7]), i32([[0], [1], [2]]), i32([9, 9, 9]), 6, 64, out=out)
    assert bool((out[0, [0, 1, 3, 4, 5]] == 3).all()) and not bool((out[0, 2] == 3).any())


# ------------------------------------------------------------------ norm_rope
def check_norm(got, x, weight, eps, cs64, half):
    """Sums of 64 squares, the root and the quotient round less than 80 times 2^-24; a rotation three more, of entries
    whose sizes it adds; then the result's own rounding."""
    w = torch.ones((x.shape[0], 64), dtype=torch.float64, device=DEV) if weight is None else weight.double()
    want = ref.norm_rope(x.double(), w, eps, cs64, half)
    plain = ref.norm_rope(x.double(), w, eps, None, half).abs()
    pair = plain if cs64 is None else plain + (plain.roll(32, -1) if half else plain.unflatten(-1, (32, 2)).flip(-1).flatten(-2))
    step = torch.finfo(got.dtype).eps / 2
    most = 84 * 2.0 ** -24 * pair * (1 + step) + step * want.abs() + (2.0 ** -25 if got.dtype is F16 else 1e-38)
    off = (got.double() - want).abs()
    assert bool((off <= most).all()), float((off / most).max())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rope", ["none", "pairs", "half"])
@pytest.mark.parametrize("L,rows,H,Hkv,pad,weighted", [(1, 1, 1, 1, 0, True), (2, 5, 6, 2, 3, True), (1, 70, 40, 8, 1, False), (3, 17, 33, 33, 0, True)])
def test_norm_rope(dtype, rope, L, rows, H, Hkv, pad, weighted):
    q, k = rows_of((L, rows, H, 64), 1, dtype, 3.0, pad), rows_of((L, rows, Hkv, 64), 2, dtype, 0.01, pad)
    positions = 40
    cs = None if rope == "none" else tq.rope_table(positions)
    params = paged.Params(L, H, Hkv, cs, dtype, tq.ROPE_HALF if rope == "half" else 0)
    pos = torch.randint(0, positions, (rows,), generator=gen(3), device=DEV).int()
    qw, kw = (0.5 + torch.rand((2, L, 64), generator=gen(4), device=DEV)) if weighted else (None, None)
    eps = 1e-5
    qo, ko = serve.norm_rope(params, q, k, pos, qw, kw, eps=eps)
    z = None if cs is None else angles(positions)[pos.long()]
    check_norm(qo, q, qw, np.float32(eps).item(), z, rope == "half")
    check_norm(ko, k, kw, np.float32(eps).item(), z, rope == "half")
    # in place, in the projection's own rows
    a, b = q.clone() if pad == 0 else q, k
    out = serve.norm_rope(params, a, b, pos, qw, kw, eps=eps, out=(a, b))
    assert out[0] is a and torch.equal(a, qo) and torch.equal(b, ko)


@pytest.mark.parametrize("rope", ["pairs", "half"])
@pytest.mark.parametrize("sections", [[32], [16, 16], [8, 12, 12], [0, 31, 0, 1], [5, 0, 27]])
def test_norm_rope_of_several_axes(rope, sections):
    rows, n = 37, 500
    q, k = rows_of((2, rows, 4, 64), 1, F32), rows_of((2, rows, 2, 64), 2, F32)
    params = paged.Params(2, 4, 2, tq.rope_table(n), F32, tq.ROPE_HALF if rope == "half" else 0)
    pos = torch.randint(0, n, (len(sections), rows), generator=gen(3), device=DEV).int()
    qo, ko = serve.norm_rope(params, q, k, pos, eps=0.0, sections=sections)
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    z = torch.stack([angles(n)[pos[a].long(), m] for m, a in enumerate(axis)], -1)
    for got, x in ((qo, q), (ko, k)):
        check_norm(got, x, None, 0.0, z, rope == "half")
    # a bad position counts on axes that have pairs
    for a, s in enumerate(sections):
        bad = pos.clone()
        bad[a, 3], bad[a, 9] = -1, n
        got = serve.norm_rope(params, q, k, bad, eps=0.0, sections=sections)
        for x, y in zip(got, (qo, ko)):
            rest = [r for r in range(rows) if r not in (3, 9)]
            assert torch.equal(x[:, rest], y[:, rest])
            assert bool(x[:, [3, 9]].isnan().all()) if s else torch.equal(x, y)


def test_norm_rope_of_zeros_and_what_is_no_number():
    x = torch.zeros((1, 4, 1, 64), dtype=F32, device=DEV)
    x[0, 1, 0, 5], x[0, 2, 0, 7], x[0, 3] = float("nan"), float("inf"), 1e-30
    params = paged.Params(1, 1, 1, tq.rope_table(8), F32)
    qo, ko = serve.norm_rope(params, x, x.clone(), i32([0, 1, 2, 0]))
    assert bool((qo[0, 0] == 0).all()) and bool(qo[0, 1].isnan().all()) and bool(qo[0, 2, 0, [6, 7]].isnan().all())
    assert torch.allclose(qo[0, 3], torch.full_like(qo[0, 3], 1e-27), rtol=1e-5) and torch.equal(qo[0, 3], ko[0, 3])


# ------------------------------------------------------------------ verify
def check_verify(target, draft, tokens, row0, uniform, uniform_next, seq_len, room=True):
    B = len(row0) - 1
    need = serve.verify_workspace_bytes(target.shape[1], B)
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV) if need and room else None
    args = (target, draft, i64(tokens), i32(row0), torch.tensor(uniform, device=DEV, dtype=F32),
            torch.tensor(uniform_next, device=DEV, dtype=F32))
    got = [t.tolist() for t in serve.verify(*args, i32(seq_len), workspace=ws)]
    want = ref.verify(target.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy(), tokens, row0,
                      args[4].tolist(), args[5].tolist(), seq_len)
    assert got[0] == want[0] and got[2] == want[1] and got[1] == want[2], (got, want)
    a, t, none = serve.verify(*args, workspace=ws)
    assert none is None and a.tolist() == got[0] and t.tolist() == got[1]
    if ws is not None:
        assert not bool(ws[:16384].any())
    return got


def probabilities(rows, vocab, seed, dtype, sharp=2.0, pad=0):
    """Two models' rows; the second is the first's, disturbed."""
    x = sharp * torch.randn((rows, vocab), generator=gen(seed), device=DEV)
    y = x + 0.7 * torch.randn((rows, vocab), generator=gen(seed + 1), device=DEV)
    out = []
    for t in (x, y):
        wide = torch.full((rows, vocab + pad), float("nan"), device=DEV, dtype=dtype)
        wide[:, :vocab] = torch.softmax(t, -1)
        out.append(wide[:, :vocab])
    return out


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("vocab,B,drafts,pad", [(1, 3, 2, 0), (2, 5, 1, 1), (33, 8, 3, 0), (257, 4, 6, 2), (2047, 3, 2, 0), (2048, 3, 2, 0),
                                                (2049, 3, 2, 0), (4096, 2, 1, 8), (10_007, 5, 4, 1), (131_072, 3, 2, 0), (600_001, 1, 2, 0)])
def test_verify(dtype, certain, vocab, B, drafts, pad):
    g = np.random.default_rng(vocab + B)
    n = g.integers(0, drafts + 1, B)
    n[0] = drafts
    row0 = np.concatenate([[0], np.cumsum(n + 1)]).tolist()
    rows = row0[-1]
    target, draft = probabilities(rows, vocab, vocab, dtype, pad=pad)
    drawn = torch.multinomial((target if certain else draft).float().contiguous(), 1, generator=gen(7))[:, 0].tolist()
    tokens = [0] + drawn[:-1]
    for share in (0.0, 0.3, 1.0):                            # few random numbers reject, some do, all may
        u = g.random(rows, dtype=np.float32) * np.float32(share)
        check_verify(target, None if certain else draft, tokens, row0, u.tolist(), g.random(B, dtype=np.float32).tolist(),
                     g.integers(20, 99, B).tolist())


@pytest.mark.parametrize("vocab", [7, 5000])
def test_verify_at_the_borders(vocab):
    # one sequence a question: p_t(d) = 1/4, q_t(d) = 1/2
    third = vocab // 3
    p, q = torch.zeros((2, vocab), device=DEV), torch.zeros((2, vocab), device=DEV)
    p[:, 0], p[:, third], p[:, vocab - 1] = 0.25, 0.25, 0.5
    q[:, third], q[:, vocab - 1] = 0.5, 0.5
    big = 1 - 2.0 ** -24
    ask = [(third, 0.5, 0.3), (third, 0.5 - 2.0 ** -25, 0.0), (third, 0.5 - 2.0 ** -25, 0.25), (third, 0.0, 0.25 - 2.0 ** -26),
           (third, 0.0, 0.5), (third, 0.0, big), (third, 1.0, 0.0), (third, 1.0, big), (1, 0.0, 0.5), (1, 0.9, 0.5),
           (0, 0.99, 0.1), (-1, 0.0, 0.5), (vocab, 0.0, 0.5), (2 ** 40, 0.0, 0.5), (third, float("nan"), 0.5), (third, 0.0, float("nan"))]
    B = len(ask)
    tokens = [t for d, _, _ in ask for t in (5, d)]
    u = [x for _, r, _ in ask for x in (r, 0.5)]
    got = check_verify(p.repeat(B, 1), q.repeat(B, 1), tokens, list(range(0, 2 * B + 1, 2)), u, [n for _, _, n in ask], [9] * B)
    assert got[0] == [0, 1, 1, 1, 1, 1, 0, 0, 0, 0, 1, 0, 0, 0, 0, 1]
    assert got[1][1:6] == [0, third, 0, vocab - 1, vocab - 1] and got[1][7] == 0
    check_verify(p.repeat(B, 1), None, tokens, list(range(0, 2 * B + 1, 2)), u, [n for _, _, n in ask], [9] * B)


@pytest.mark.parametrize("vocab", [9, 7000])
def test_verify_of_probabilities_that_are_none(vocab):
    inf, nan = float("inf"), float("nan")
    rows = torch.rand((8, vocab), generator=gen(1), device=DEV)
    other = torch.rand((8, vocab), generator=gen(2), device=DEV)
    rows[0], rows[2, 1::2], rows[4] = 0.0, nan, -1.0          # no weight at all; some; none
    rows[6, 3], other[6, 4], other[6, 5] = inf, -2.0, nan
    other[2] = 0.0
    tokens = [0, 3, 0, 2, 0, 1, 0, 3]
    for u in (0.0, 0.999):
        got = check_verify(rows, other, tokens, [0, 2, 4, 6, 8], [u] * 8, [0.1, 0.5, 0.5, 0.9], [5] * 4)
        assert got[1][0] == -1 and got[1][2] == -1 and got[0][3] == 0
    # nothing is left of the target where it is below the draft: all of it counts
    p = torch.full((2, vocab), 0.25, device=DEV)
    got = check_verify(p, p * 2, [0, 3], [0, 2], [0.5, 0.5], [0.5], [5])
    assert got[0] == [0] and got[1] == [vocab // 2]


def test_verify_of_rows_that_are_not_valid():
    target, draft = probabilities(6, 50, 3, F32)
    out = check_verify(target, draft, [1, 2, 3, 4, 5, 6], [2, 2, 1, 4, 7, -1, 3], [0.1] * 6, [0.5] * 6, [10, 11, 12, 13, 14, 15])
    assert out[1][0] == out[1][1] == -1 and out[2][0] == 10 and out[1][3] == -1
    got = serve.verify(target[:0], None, i64([]), i32([0, 0]), target[:0, 0], target[:1, 0].contiguous(), i32([4]))
    assert [t.tolist() for t in got] == [[0], [-1], [4]]


def test_verify_draws_as_the_target_does():
    # 200 000 sequences of two drafts over 11 symbols: what comes out at each place has the target's frequencies. The
    # standard error of a frequency p is sqrt(p (1 - p) / n); six of them are passed with a chance of 2e-9 each
    B, vocab, g = 4096, 11, gen(11)
    p, q = probabilities(3, vocab, 21, F32)
    counts, total = torch.zeros(vocab, dtype=torch.float64, device=DEV), 0
    second, after = torch.zeros_like(counts), 0
    for _ in range(49):
        d = torch.stack([torch.multinomial(q[i], B, True, generator=g) for i in (0, 1)])
        tokens = torch.stack([torch.zeros_like(d[0]), d[0], d[1]], 1).flatten()
        a, t, _ = serve.verify(p.repeat(B, 1), q.repeat(B, 1), tokens, torch.arange(0, 3 * B + 1, 3, device=DEV).int(),
                               torch.rand(3 * B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV))
        first = torch.where(a > 0, d[0], t)
        counts += torch.bincount(first, minlength=vocab)
        total += B
        two = torch.where(a > 1, d[1], t)[a > 0]
        second += torch.bincount(two, minlength=vocab)
        after += two.numel()
    for c, n, want in ((counts, total, p[0]), (second, after, p[1])):
        want = want.double() / want.double().sum()
        assert bool(((c / n - want).abs() <= 6 * (want * (1 - want) / n).sqrt()).all())


# ------------------------------------------------------------------ together
def model(L, H, Hkv, dtype, cs, seed):
    qw, kw = 0.5 + torch.rand((2, L, 64), generator=gen(seed), device=DEV)
    return paged.Params(L, H, Hkv, cs, dtype), paged.Params(L, H, Hkv, io_dtype=dtype), qw, kw


def test_a_serving_loop_with_drafts():
    # prompts, then steps of drafted tokens: every step norms, appends, attends, verifies and gives back what was rejected; the cache
    # and the lengths at the end are those of appending the tokens that were kept, one call for all
    L, H, Hkv, B, vocab, D = 2, 4, 2, 5, 97, 3
    cs = tq.rope_table(400)
    before, params, qw, kw = model(L, H, Hkv, BF16, cs, 5)
    pool, cache = paged.PagePool(40), serve.Cache4(L, Hkv, 40)
    table = torch.full((B, 6), -1, dtype=torch.int32, device=DEV)
    seq_len, g = i32([0] * B), gen(3)
    embed = torch.randn((vocab, L, H + 2 * Hkv, 64), generator=g, device=DEV).to(BF16)   # a token's projection
    held = [torch.randint(0, vocab, (n,), generator=g, device=DEV).tolist() for n in (63, 1, 130, 64, 20)]
    room = torch.zeros(max(serve.workspace_bytes(params, L, B, 1 + D, 384), serve.verify_workspace_bytes(vocab, B), 1),
                       dtype=torch.uint8, device=DEV)

    def step(tokens):
        rows = sum(map(len, tokens))
        slots, pos, row0, granted = paged.assign(pool, table, seq_len, i32([len(t) for t in tokens]), rows)
        assert granted.tolist() == [1] * B
        qkv = embed[i64([x for t in tokens for x in t])].transpose(0, 1)
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        q, k = serve.norm_rope(before, q, k, pos, qw, kw)
        serve.append(params, cache, k, v, slots)
        return slots, pos, row0, serve.attend(params, cache, q, pos, row0, table, seq_len, max(map(len, tokens)), 384, workspace=room)

    step(held)
    for n in range(12):
        drafts = [torch.randint(0, vocab, (int(d),), generator=g, device=DEV).tolist() for d in np.random.default_rng(n).integers(0, D + 1, B)]
        last = torch.randint(0, vocab, (B,), generator=g, device=DEV).tolist()
        tokens = [[x] + d for x, d in zip(last, drafts)]
        slots, pos, row0, out = step(tokens)
        rows = row0[-1].item()
        target = torch.softmax(out[0].float().flatten(1)[:, :vocab] * 3, -1)      # (logits of a kind)
        target[:, :] = torch.softmax(torch.randn((rows, vocab), generator=g, device=DEV), -1) * 0.5 + target * 0.5
        u = torch.rand(rows, generator=g, device=DEV) * 0.02
        accepted, token, keep = serve.verify(target, None, i64([x for t in tokens for x in t]), row0, u,
                                             torch.rand(B, generator=g, device=DEV), seq_len, workspace=room)
        paged.release(pool, table, seq_len, keep)
        for b, a in enumerate(accepted.tolist()):
            held[b] += tokens[b][:1 + a]
        assert seq_len.tolist() == [len(t) for t in held]
    lens = [len(t) for t in held]
    fresh = serve.Cache4(L, Hkv, 40)
    at = [table[b, p // 64].item() * 64 + p % 64 for b in range(B) for p in range(lens[b])]
    qkv = embed[i64([x for t in held for x in t])].transpose(0, 1)
    pos = i32([p for n in lens for p in range(n)])
    _, k = serve.norm_rope(before, qkv[:, :, :H], qkv[:, :, H:H + Hkv], pos, qw, kw)
    serve.append(params, fresh, k, qkv[:, :, H + Hkv:], i64(at))
    for a, b in zip(serve.read(params, cache, i64(at)), serve.read(params, fresh, i64(at))):
        assert torch.equal(a, b)
    used = sum(paged_ref.pages_of(n) for n in lens)
    assert pool.state.tolist() == [40 - used, 0, 0, 0]


def test_the_quality_command_s_row_is_the_cache_s():
    # the output of quality.decode_paged is the exact attention over what the cache holds, and above every 3-bit variant's
    # worst case; the bound is that of the attention tests
    from paper_2603_26110_amd import quality
    inp = quality.inputs(heads=4, tokens=256, calib=64, seed=7)
    got = quality.decode_paged(inp, 4)
    cache, params = serve.Cache4(1, 4, 4), paged.Params(1, 4, 4, tq.rope_table(256))
    k, v, q = (torch.from_numpy(np.ascontiguousarray(inp[n][0])).to(DEV) for n in ("k", "v", "q"))
    serve.append(params, cache, k, v, i64(list(range(256))), i32(list(range(256))))
    kr, vr = (torch.from_numpy(x).to(DEV) for x in ref.CacheRef(cache).values())
    w, spread, size, reach = ref.attend(kr, vr, q[None].double(), [255], [0, 1], [[0, 1, 2, 3]], [256], True, 0.125, angles(256))
    most = ref.bound(w, spread, size, reach, 256, EPS[F32], F32)[0, 0].cpu().numpy()
    assert (np.abs(got - w[0, 0].cpu().numpy()) <= most).all()
    assert quality.metrics(got, inp["ref"])["rel_l2"] > quality.metrics(quality.decode_paged(inp), inp["ref"])["rel_l2"]


def test_a_captured_step():
    # norm, append, attend and verify in one graph, replayed with new inputs and eager work between
    L, H, Hkv, B, vocab = 1, 8, 2, 3, 5000
    cs = tq.rope_table(3000)
    before, params, qw, kw = model(L, H, Hkv, F16, cs, 5)
    lens, news = [2500, 65, 130], [3, 2, 4]
    table, pos, row0, pages = layout(lens, news, 4)
    start = random_cache(L, Hkv, pages, 8)
    rows = row0[-1]
    slots = [table[b][p // 64] * 64 + p % 64 for b in range(B) for p in range(lens[b] - news[b], lens[b])]
    pos, row0, table, lens, slots = i32(pos), i32(row0), i32(table), i32(lens), i64(slots)
    cache = serve.Cache4(L, Hkv, pages, buffers=tuple(t.clone() for t in (start.k_codes, start.v_codes, start.scales)))
    need = max(serve.workspace_bytes(params, L, B, 4, 2500), serve.verify_workspace_bytes(vocab, B))
    assert need > 16384
    room = torch.zeros(need, dtype=torch.uint8, device=DEV)
    qkv = torch.zeros((L, rows, H + 2 * Hkv, 64), dtype=F16, device=DEV)
    target, draft = torch.zeros((2, rows, vocab), device=DEV).unbind(0)
    u, un, tokens = torch.zeros(rows, device=DEV), torch.zeros(B, device=DEV), torch.zeros(rows, dtype=torch.int64, device=DEV)

    def step(cache, room):
        q, k = serve.norm_rope(before, qkv[:, :, :H], qkv[:, :, H:H + Hkv], pos, qw, kw)
        serve.append(params, cache, k, qkv[:, :, H + Hkv:], slots)
        out = serve.attend(params, cache, q, pos, row0, table, lens, 4, 2500, workspace=room)
        return (out, *serve.read(params, cache, slots), *serve.verify(target, draft, tokens, row0, u, un, lens, workspace=room))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, room)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(cache, room)
    other = torch.zeros_like(room)
    for n in range(4):
        g = gen(50 + n)
        qkv.copy_(torch.randn(qkv.shape, generator=g, device=DEV))
        p, d = probabilities(rows, vocab, 60 + n, F32)
        target.copy_(p)
        draft.copy_(d)
        tokens.copy_(torch.randint(0, vocab, (rows,), generator=g, device=DEV))
        u.copy_(torch.rand(rows, generator=g, device=DEV) * 0.3)
        un.copy_(torch.rand(B, generator=g, device=DEV))
        graph.replay()
        got = [t.clone() for t in held]
        eager = step(serve.Cache4(L, Hkv, pages, buffers=tuple(t.clone() for t in (cache.k_codes, cache.v_codes, cache.scales))),
                     other if n % 2 else room)
        for a, b in zip(got, eager):
            assert torch.equal(a, b), n


def test_calls_on_two_streams():
    # attention and verification at once, a workspace each
    L, H, Hkv, B, vocab = 1, 8, 1, 2, 20_000
    lens, news = [5000, 3000], [2, 1]
    table, pos, row0, pages = layout(lens, news, 4)
    cache, params = random_cache(L, Hkv, pages, 8), paged.Params(L, H, Hkv, io_dtype=BF16)
    q = rows_of((L, row0[-1], H, 64), 1, BF16)
    args = (params, cache, q, i32(pos), i32(row0), i32(table), i32(lens), 2, 5000)
    target, draft = probabilities(row0[-1], vocab, 5, F32)
    ask = (target, draft, i64([1, 2, 3]), i32(row0), torch.tensor([0.0, 0.5, 0.5], device=DEV), torch.tensor([0.3, 0.6], device=DEV))
    want, drawn = serve.attend(*args), serve.verify(*ask)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    rooms = [torch.zeros(serve.workspace_bytes(params, L, B, 2, 5000), dtype=torch.uint8, device=DEV),
             torch.zeros(serve.verify_workspace_bytes(vocab, B), dtype=torch.uint8, device=DEV)]
    assert all(r.numel() for r in rooms)
    torch.cuda.synchronize()
    got, tokens = [], []
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            got.append(serve.attend(*args, workspace=rooms[0]))
        with torch.cuda.stream(streams[1]):
            tokens.append(serve.verify(*ask, workspace=rooms[1]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
    assert all(torch.equal(a, b) for t in tokens for a, b in zip(t[:2], drawn[:2]))
    # one workspace for both, in order
    shared = torch.zeros(max(r.numel() for r in rooms), dtype=torch.uint8, device=DEV)
    for _ in range(3):
        assert torch.equal(serve.attend(*args, workspace=shared), want)
        assert serve.verify(*ask, workspace=shared)[1].tolist() == drawn[1].tolist()


def test_captured_without_a_workspace():
    # every call of a graph then has room of its own, cleared at each replay
    lens, news = [5000, 3000], [2, 1]
    table, pos, row0, pages = layout(lens, news, 4)
    cache, params = random_cache(1, 1, pages, 8), paged.Params(1, 8, 1, io_dtype=BF16)
    q = rows_of((1, row0[-1], 8, 64), 1, BF16)
    args = (params, cache, q, i32(pos), i32(row0), i32(table), i32(lens), 2, 5000)
    target, draft = probabilities(3, 20_000, 5, F32)
    ask = (target, draft, i64([1, 2, 3]), i32(row0), torch.tensor([0.0, 0.5, 0.5], device=DEV), torch.tensor([0.3, 0.6], device=DEV))
    want, drawn = serve.attend(*args), serve.verify(*ask)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve.attend(*args), serve.verify(*ask)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, got = serve.attend(*args), serve.verify(*ask)
    for _ in range(3):
        out.zero_()
        got[1].zero_()
        graph.replay()
        assert torch.equal(out, want) and torch.equal(got[0], drawn[0]) and torch.equal(got[1], drawn[1])
        assert torch.equal(serve.attend(*args), want)


def test_broadcast_rows_and_strided_probabilities():
    # queries, keys and values that several rows, heads or layers share; probabilities whose rows are further apart
    cache, params = serve.Cache4(2, 3, 2), paged.Params(2, 6, 3, tq.rope_table(80), F16)
    one = rows_of((1, 1, 1, 64), 3, F16)
    k, q = one.expand(2, 70, 3, 64), one.expand(2, 70, 6, 64)
    slots, pos = list(range(70)), list(range(70))
    serve.append(params, cache, k, k, i64(slots), i32(pos))
    whole = serve.Cache4(2, 3, 2)
    serve.append(params, whole, k.contiguous(), k.contiguous(), i64(slots), i32(pos))
    assert torch.equal(cache.k_codes, whole.k_codes) and torch.equal(cache.v_codes, whole.v_codes) and torch.equal(cache.scales, whole.scales)
    rest = (i32(pos), i32([0, 70]), i32([[0, 1]]), i32([70]), 70, 70)
    assert torch.equal(serve.attend(params, cache, q, *rest), serve.attend(params, cache, q.contiguous(), *rest))
    for a, b in zip(serve.norm_rope(params, q, k, i32(pos)), serve.norm_rope(params, q.contiguous(), k.contiguous(), i32(pos))):
        assert torch.equal(a, b)
    with pytest.raises(tq.TQError, match="stride of zero"):
        serve.norm_rope(params, q, k, i32(pos), out=(q, k))
    target, draft = probabilities(12, 3001, 5, BF16)
    ask = lambda p, d: serve.verify(p, d, i64([1, 2, 3, 4]), i32([0, 4]), torch.full((4,), 0.1, device=DEV), torch.full((1,), 0.7, device=DEV))
    for a, b in zip(ask(target[::3], draft[::3]), ask(target[::3].contiguous(), draft[::3].contiguous())):
        assert a is None or torch.equal(a, b)


def test_a_cache_of_another_kind_is_refused():
    c8, c4 = paged.Cache(1, 1, 2), serve.Cache4(1, 1, 2)
    params = paged.Params(1, 1, 1)
    x, z = rows_of((1, 1, 1, 64), 1, F16), i32([0])
    for call in (lambda: paged.append(params, c4, x, x, z.long()), lambda: serve.append(params, c8, x, x, z.long()),
                 lambda: paged.attend(params, c4, x, z, i32([0, 1]), i32([[0]]), i32([1]), 1, 1),
                 lambda: serve.attend(params, c8, x, z, i32([0, 1]), i32([[0]]), i32([1]), 1, 1),
                 lambda: serve.read(params, c8, z.long())):
        with pytest.raises(TypeError, match="Cache"):
            call()


def test_slots_past_32_bits_of_bytes():
    # a page whose codes lie past 2^32 bytes of their plane
    pages = 2 ** 21 + 3
    cache, params = serve.Cache4(1, 1, pages), paged.Params(1, 1, 1, io_dtype=F32)
    x = rows_of((1, 3, 1, 64), 1, F32)
    slots = [(pages - 1) * 64 + 5, (pages - 2) * 64, 7]
    serve.append(params, cache, x, x, i64(slots))
    small = serve.Cache4(1, 1, 1)
    serve.append(params, small, x, x, i64([0, 1, 2]))
    for a, b in zip(serve.read(params, cache, i64(slots)), serve.read(params, small, i64([0, 1, 2]))):
        assert torch.equal(a, b)
    q = rows_of((1, 1, 1, 64), 2, F32)
    out = [serve.attend(params, c, q, i32([0]), i32([0, 1]), i32([[p]]), i32([1]), 1, 64)
           for c, p in ((cache, pages - 2), (small, 0))]
    serve.append(params, small, x[:, 1:2], x[:, 1:2], i64([0]))
    want = serve.attend(params, small, q, i32([0]), i32([0, 1]), i32([[0]]), i32([1]), 1, 64)
    assert torch.equal(out[0], want)
