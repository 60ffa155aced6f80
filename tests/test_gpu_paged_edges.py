"""The paged cache at the edges of what it documents: queries and scores past the ordinary, value scales far apart, bad
pages, the types and pairings that the other tests do not reach."""

import math

import pytest
import torch

import paged_ref as ref
import paper_2603_26110_amd as tq
from paper_2603_26110_amd import paged
from test_gpu_paged import BF16, DEV, F16, F32, SHAPES, World, i32, random_cache, same_cache

pytestmark = pytest.mark.gpu

# (lens, new, heads, kv_heads): every kind of launch that attention has
FEW = {"four_waves": ([200, 65], [1, 2], 6, 2), "eight_waves": ([1025], [1], 4, 4), "splits": ([8192], [1], 4, 1),
       "one_wave": ([130] * 64, [1] * 64, 32, 32)}
MANY = {"two_groups": ([200, 90], [70, 66], 2, 1), "splits": ([9000], [70], 2, 1), "one_group": ([130] * 32, [129] * 32, 12, 12)}
ALL = {**{"few_" + k: v for k, v in FEW.items()}, **{"many_" + k: v for k, v in MANY.items()}}


# ---------------------------------------------------------------- queries
@pytest.mark.parametrize("dtype,rope,out_f32", [(BF16, "none", False), (F16, "none", False), (BF16, "half", False),
                                                (F16, "pairs", False), (F32, "none", False), (F16, "none", True)])
@pytest.mark.parametrize("kind", list(ALL))
def test_an_infinite_query_has_no_result(kind, dtype, rope, out_f32):
    # every key has one sign in the query's infinite channel, so that every score is -inf: the mask's value
    w = World(*ALL[kind], dtype=dtype, rope=rope, out_f32=out_f32, seed=31)
    k, _, _ = w.cache.values()
    codes = w.cache.k_codes.view(w.params.num_layers, w.params.kv_heads, w.pages, 64, 64)
    codes[..., 3] |= 0x80                                  # (negative; no code of this world's is NaN)
    codes[..., 3] = torch.where(codes[..., 3] == 0x80, 0x90, codes[..., 3].int()).to(torch.uint8)
    fine = w.call()
    w.check(fine)
    q = w.q.clone()
    rows = sorted({0, w.rows // 2, w.rows - 1})
    q[:, rows, :, 3] = float("inf")
    for causal in (True, False):
        got, other = w.call(causal, q=q), w.call(causal)
        assert bool(got[:, rows].isnan().all())
        rest = torch.ones(w.rows, dtype=torch.bool, device=DEV)
        rest[rows] = False
        assert torch.equal(got[:, rest], other[:, rest])
    empty = w.call(q=q, seq_len=i32([0] * len(w.lens)))   # (a row that sees nothing has no score either)
    assert bool((empty == 0).all())


@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("kind", list(ALL))
def test_an_fp16_query_without_rope_is_exact(kind, out_f32):
    # a channel of the largest size, in which the keys are zero, takes no bits from the others (down to fp16's lowest)
    w = World(*ALL[kind], dtype=F16, rope="none", out_f32=out_f32, seed=33, scale=8.0)
    w.cache.k_codes.view(w.params.num_layers, w.params.kv_heads, w.pages, 64, 64)[..., 7] = 0
    w.q *= 2.0 ** -6
    w.q[..., 20:40] *= 2.0 ** -9
    w.q[..., 7] = 65504.0
    w.check(w.call())


@pytest.mark.parametrize("dtype,rope,out_f32", [(F16, "pairs", False), (F16, "half", True), (BF16, "pairs", False),
                                                (BF16, "half", True), (F32, "pairs", False), (F32, "none", False)])
@pytest.mark.parametrize("kind", list(ALL))
def test_a_large_channel_takes_no_bits_from_the_others(kind, dtype, rope, out_f32):
    # (the keys are zero in it and in its partner; the other channels decide the scores)
    w = World(*ALL[kind], dtype=dtype, rope=rope, out_f32=out_f32, seed=34, scale=8.0)
    w.cache.k_codes.view(w.params.num_layers, w.params.kv_heads, w.pages, 64, 64)[..., [6, 7, 39]] = 0
    w.q *= 2.0 ** -6
    w.q[..., 7] = 65504.0
    w.check(w.call())


@pytest.mark.parametrize("kind", list(ALL))
def test_positions_past_the_sequence_see_all_of_it(kind):
    # without RoPE any position that is not negative is one: the largest, too
    w = World(*ALL[kind], rope="none", seed=35)
    want = w.call(False)
    for p in (max(w.lens) - 1, 2 ** 24, 2 ** 31 - 2, 2 ** 31 - 1):
        assert torch.equal(w.call(True, pos=i32([p] * w.rows)), want), p


@pytest.mark.parametrize("dtype,out_f32", [(F16, False), (BF16, False), (F32, False), (F16, True)])
@pytest.mark.parametrize("kind", list(ALL))
def test_scores_of_billions(kind, dtype, out_f32):
    """Scores whose binary32 steps are larger than the range of the weights: the largest takes all."""
    w = World(*ALL[kind], dtype=dtype, rope="none", out_f32=out_f32, seed=36, scale=1.0)
    w.q *= 15000.0
    w.cache.scales[..., 0] *= 2.0 ** 13
    k, v, s = w.cache.values()
    k = k.double() * s[..., 0].double()[..., None, None]
    v = v.reshape(k.shape).double() * s[..., 1].double()[..., None, None]
    got, G, clear, rows = w.call(False), w.params.num_heads // w.params.kv_heads, 0, 0
    number = torch.isfinite(w.q).all(-1)                 # (15000 times a normal number may pass 65504)
    assert torch.equal(torch.isfinite(got).all(-1), number) and torch.equal(got.isnan().any(-1), ~number)
    half = torch.finfo(got.dtype).eps / 2
    for b, n in enumerate(w.lens[:3]):
        ids, lo, hi = w.table[b][:ref.pages_of(n)], w.row0[b], w.row0[b + 1]
        kb, vb = (x[0][:, ids].reshape(w.params.kv_heads, -1, 64)[:, :n] for x in (k, v))
        for h in range(w.params.num_heads):
            q = w.q[0, lo:hi, h].double()
            score, size = q @ kb[h // G].T, q.abs() @ kb[h // G].abs().T
            two = score.topk(2, -1)
            # the sum of 64 products rounds 64 times at most, its scaling and the difference three times
            far = (two.values[:, 0] - two.values[:, 1] > 2 * 70 * 2.0 ** -24 * size.amax(-1) + 40) & number[0, lo:hi, h]
            clear, rows = clear + int(far.sum()), rows + hi - lo
            want = vb[h // G][two.indices[:, 0]]
            off = (got[0, lo:hi, h].double() - want).abs()[far]
            # (the weight that is left is one fp16 value, or two parts, over itself; the others are below 2^-57)
            assert bool((off <= (half + 2.0 ** -21) * want.abs()[far] + 2.0 ** -40).all())
    assert clear > 0.99 * rows


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,B,H", [(1, 1, 1), (1, 1, 300), (1, 70, 32), (70, 1, 1), (70, 20, 20), (129, 32, 12)])
def test_scores_whose_steps_are_eight(rows, B, H, dtype):
    """Half of the pages have scores of 2^26 (in powers of two), where binary32 counts in eights, the others 2^26 + 8."""
    n = 8 if B * H >= 2048 else 16
    cache = paged.Cache(1, H, n)
    params = paged.Params(1, H, H, None, dtype, softmax_scale=math.log(2.0))
    k, v, s = cache.values()
    k.zero_()
    for d, value in ((0, 256.0), (1, 2.0 ** -5)):
        k[:, :, (0 if d == 0 else n // 2):, :, d] = torch.full((), value, device=DEV).to(k.dtype)
    v[:, :, :n // 2] = torch.ones_like(v[:, :, :n // 2])
    v[:, :, n // 2:] = (torch.ones(v[:, :, n // 2:].shape, device=DEV) * 3).to(v.dtype)
    s[..., 0], s[..., 1] = 2.0 ** 5, 1.0
    q = torch.zeros((1, B * rows, H, 64), dtype=dtype, device=DEV)
    q[..., 0], q[..., 1] = 2.0 ** 13, 8.0
    got = paged.attend(params, cache, q, i32([64 * n - 1] * (B * rows)), i32(list(range(0, B * rows + 1, rows))),
                       i32([list(range(n))] * B), i32([64 * n] * B), rows, 64 * n)
    want = (1.0 * 2.0 ** -8 + 3.0) / (2.0 ** -8 + 1.0)
    assert float((got.double() - want).abs().max()) <= (2 * 2.0 ** -11 + 1088 * 2.0 ** -23 + torch.finfo(dtype).eps / 2) * want


# ------------------------------------------------ types, bounds, row offsets
OTHERS = [(F16, "none", False), (F16, "half", False), (F16, "half", True), (BF16, "none", False), (BF16, "pairs", False),
          (BF16, "none", True), (F32, "half", False), (F32, "pairs", False)]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("dtype,rope,out_f32", OTHERS)
def test_attend_of_the_other_types(shape, dtype, rope, out_f32):
    w = World(*SHAPES[shape], dtype=dtype, rope=rope, out_f32=out_f32, fused=shape % 2 == 0, layers=1 + shape % 2, seed=50 + shape)
    for causal in (True, False):
        w.check(w.call(causal), causal)


@pytest.mark.parametrize("kind", list(ALL))
@pytest.mark.parametrize("dtype,rope,out_f32", OTHERS)
def test_every_launch_of_the_other_types(kind, dtype, rope, out_f32):
    w = World(*ALL[kind], dtype=dtype, rope=rope, out_f32=out_f32, seed=37)
    for causal in (True, False):
        w.check(w.call(causal), causal)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_bounds_that_are_not_reached(dtype):
    # a serving loop gives its capacity: other kernels and splits, the same result within its bound
    w = World([300, 5, 64, 1025], [1, 4, 0, 2], 6, 2, dtype=dtype, seed=38)
    for max_new in (4, 40, 1000):
        for max_len in (1025, 4000, 100_000, 2 ** 30):
            for causal in (True, False):
                w.check(w.call(causal, max_new=max_new, max_len=max_len), causal)


@pytest.mark.parametrize("new", [1, 40, 200])
def test_rows_that_row0_puts_outside_are_not_written(new):
    lens, news = [400, 300, 200, 250, 220], [new, min(new, 300), min(new, 200), min(new, 3), min(new, 220)]
    w = World(lens, news, 4, 2, seed=39)
    fine = w.call()
    w.check(fine)

    def rows(row0, untouched):
        out = torch.full_like(fine, 7.0)
        w.call(row0=i32(row0), out=out)
        for b in range(5):
            at = slice(w.row0[b], w.row0[b + 1])
            if b in untouched:
                assert bool((out[:, at] == 7).all()), b
            else:
                assert torch.equal(out[:, at], fine[:, at]), b
    rows(w.row0, ())
    # a first row before the rows, a last one behind them: those sequences are skipped, the others are not
    rows([-1] + w.row0[1:5] + [w.rows + 1], (0, 4))
    rows([-2 ** 31] + w.row0[1:5] + [2 ** 31 - 1], (0, 4))
    # everything behind the rows, or before them
    rows([w.rows + 5] * 6, range(5))
    rows([-7] * 6, range(5))


# ----------------------------------------------------------- value scales
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,new", [(160, 1), (165, 65), (770, 65)])
def test_value_scales_far_apart_after_many_tokens(B, new, dtype):
    """A first page with scores of zero, pages whose scores are 2^14.9 times the weight and whose values are the largest
    that there are, then pages of the smallest scale. Every sequence owns the same pages, and its rows see all."""
    n, low, high = 160, 16, 128                           # pages: scores of zero; high scores and values; the rest small
    cache, params = paged.Cache(1, 1, n), paged.Params(1, 1, 1, None, dtype, softmax_scale=math.log(2.0))
    k, v, s = cache.values()
    k.zero_()
    v[:] = torch.ones_like(v)
    k[:, :, low:low + high, :, 0] = torch.full((1, 1, high, 64), 15.0, device=DEV).to(k.dtype)   # (the score's log2)
    k[:, :, low + high:, :, 0] = torch.full((1, 1, n - low - high, 64), -1.0, device=DEV).to(k.dtype)
    v[:, :, low:low + high] = torch.full((1, 1, high, 4, 4, 4, 64), 448.0, device=DEV).to(v.dtype)
    s[..., 0] = 1.0
    s[..., 1] = 2.0 ** -48
    s[:, :, low:low + high, 1] = 2.0 ** 47
    rows = B * new
    q = torch.zeros((1, rows, 1, 64), device=DEV, dtype=dtype)
    q[..., 0] = 0.5                                       # (15 / 2 above the first page: the reference does not move)
    row0 = i32(list(range(0, rows + 1, new)))
    got = paged.attend(params, cache, q, i32([64 * n - 1] * rows), row0, i32([list(range(n))] * B), i32([64 * n] * B), new,
                       64 * n, causal=False)
    weight = 2.0 ** torch.tensor([0.0] * low + [7.5] * high + [-0.5] * (n - low - high), dtype=torch.float64)
    value = torch.tensor([2.0 ** -48] * low + [448.0 * 2.0 ** 47] * high + [2.0 ** -48] * (n - low - high), dtype=torch.float64)
    want = float((weight * value).sum() / weight.sum())
    # weights to 2^-11 (fp16) each above and below, sums of 10240 terms in binary32, the result's own rounding
    tol = (2 * 2.0 ** -11 + 2 * 10304 * 2.0 ** -24 + torch.finfo(got.dtype).eps / 2) * abs(want)
    assert float((got.double() - want).abs().max()) <= tol


# -------------------------------------------------------------- bad pages
ENDS = {"few_four_waves": ([66, 130], [4, 4], 6, 2), "few_eight_waves": ([64 * 17 + 2], [4], 4, 4),
        "few_splits": ([8194], [4], 4, 1), "few_one_wave": ([66, 130] * 32, [4] * 64, 32, 32),
        "many_two_groups": ([130, 66], [70, 66], 2, 1), "many_splits": ([9002], [70], 2, 1),
        "many_one_group": ([130] * 32, [129] * 32, 12, 12)}


@pytest.mark.parametrize("dtype,rope", [(BF16, "none"), (F32, "pairs")])
@pytest.mark.parametrize("kind", list(ENDS))
def test_a_bad_page_touches_only_the_rows_that_see_it(kind, dtype, rope):
    """The last page of every sequence is not there, and page 0, which no sequence has, holds no numbers at all."""
    w = World(*ENDS[kind], dtype=dtype, rope=rope, seed=32)
    c, spare = w.cache, next(p for p in range(1, w.pages) if all(p not in row for row in w.table))
    for t in (c.k_codes, c.v_codes, c.scales):
        t[:, :, spare] = t[:, :, 0]
    w.table = [[spare if p == 0 else p for p in row] for row in w.table]
    fine = w.call()
    w.check(fine)
    table, sees = [list(row) for row in w.table], torch.zeros(w.rows, dtype=torch.bool, device=DEV)
    for b, n in enumerate(w.lens):
        last = (n - 1) // 64
        table[b][last] = (-1, w.pages, 2 ** 31 - 1)[b % 3]
        for t in range(w.row0[b], w.row0[b + 1]):
            sees[t] = w.pos[t] >= 64 * last
    assert bool(sees.any()) and not bool(sees.all())
    for codes, scales in ((0x7F, 0.0), (0xFF, float("nan")), (0x7F, float("inf"))):
        c.k_codes[:, :, 0], c.v_codes[:, :, 0], c.scales[:, :, 0] = codes, codes, scales
        got = w.call(table=i32(table))
        assert bool(got[:, sees].isnan().all()) and torch.equal(got[:, ~sees], fine[:, ~sees])


# ------------------------------------------------------------------ pages
def test_assign_of_as_many_rows_as_there_are_numbers():
    # 2^31 - 1 rows, all but 75 of them padding: a row number past the last does not come back as a negative one
    rows, before = 2 ** 31 - 1, 1 << 17
    slots = torch.full((before + rows,), 7, dtype=torch.int64, device=DEV)
    pos = torch.full((before + rows,), 7, dtype=torch.int32, device=DEV)
    pool, table, lens = paged.PagePool(8), torch.full((2, 2), -1, dtype=torch.int32, device=DEV), i32([0, 0])
    paged.assign(pool, table, lens, i32([5, 70]), rows, out=(slots[before:], pos[before:], i32([0] * 3), i32([0] * 2)))
    assert lens.tolist() == [5, 70] and table.tolist() == [[0, -1], [1, 2]] and pool.state.tolist() == [5, 0, 0, 0]
    want = list(range(5)) + list(range(64, 134))
    assert slots[before:before + 75].tolist() == want and pos[before:before + 75].tolist() == list(range(5)) + list(range(70))
    for t in (slots, pos):
        assert bool((t[:before] == 7).all())
        for i in range(before + 75, before + rows, 1 << 28):
            assert bool((t[i:i + (1 << 28)] == -1).all())


# ----------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_append_without_rope_needs_no_positions(dtype):
    g = torch.Generator(device=DEV).manual_seed(41)
    k, v = torch.randn((2, 1, 150, 2, 64), generator=g, device=DEV).to(dtype).unbind(0)
    slots, pos = torch.arange(64, 214, device=DEV), i32(list(range(150)))
    params = paged.Params(1, 4, 2, None, dtype)
    caches = [paged.Cache(1, 2, 4) for _ in range(3)]
    paged.append(params, caches[0], k, v, slots, pos)
    paged.append(params, caches[1], k, v, slots, None)
    paged.append(params, caches[2], k, v, slots)
    for c in caches[1:]:
        for name in ("k_codes", "v_codes", "scales"):
            assert torch.equal(getattr(c, name), getattr(caches[0], name)), name
    assert bool(caches[0].k_codes.any())
    with pytest.raises(TypeError):                # (with RoPE they are needed)
        paged.append(paged.Params(1, 4, 2, tq.rope_table(200), dtype), caches[0], k, v, slots)
    with pytest.raises(ValueError):               # (and what is given is looked at)
        paged.append(params, caches[0], k, v, slots, pos[:149])


def test_numbers_past_32_bits_are_refused_not_cut():
    w = World([100, 70], [2, 1], 4, 2, seed=42)
    before = w.call()
    kv = torch.zeros((1, w.rows, 2, 64), dtype=F16, device=DEV)
    slots, out = torch.full((w.rows,), -1, dtype=torch.int64, device=DEV), torch.full_like(before, 7.0)
    for wide in (2 ** 31, 2 ** 32, 2 ** 32 + 100, -2 ** 32):
        for kw in (dict(max_new=wide), dict(max_len=wide), dict(layer0=wide)):
            with pytest.raises(ValueError):
                w.call(out=out, **kw)
        with pytest.raises(ValueError):
            paged.append(w.params, w.cache, kv, kv, slots, i32(w.pos), layer0=wide)
        pool, table, lens = paged.PagePool(9), torch.full((2, 4), -1, dtype=torch.int32, device=DEV), i32([0, 0])
        room = (torch.empty(8, dtype=torch.int64, device=DEV), i32([0] * 8), i32([0] * 3), i32([0] * 2))
        with pytest.raises(ValueError):
            paged.assign(pool, table, lens, i32([2, 1]), wide, out=room)
        assert pool.state.tolist() == [9, 0, 0, 0] and lens.tolist() == [0, 0]
    assert bool((out == 7).all())
    with pytest.raises(tq.TQError):                # (what 32 bits hold the library itself refuses)
        w.call(layer0=-1)


# -------------------------------------------------------------- workspace
def test_only_the_counters_of_a_workspace_are_cleared():
    from torch.utils._python_dispatch import TorchDispatchMode

    class Fills(TorchDispatchMode):
        """Bytes that calls set to a value."""
        total = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            out = func(*args, **(kwargs or {}))
            if func.overloadpacket.__name__ in ("zeros", "zero_", "fill_", "full"):
                self.total += out.numel() * out.element_size()
            return out

    for w in (World([9000], [70], 2, 1, seed=43), World([8192], [1], 4, 1, seed=44)):
        need = paged.workspace_bytes(w.params, 1, 1, w.new[0], w.lens[0])
        want = w.call()
        w.check(want)
        args = dict(pos=i32(w.pos), row0=i32(w.row0), table=i32(w.table), seq_len=i32(w.lens))
        for size in (None, 1000):
            with Fills() as fills:
                got = w.call(workspace=None if size is None else torch.empty(size, dtype=torch.uint8, device=DEV), **args)
            assert torch.equal(got, want) and 0 < fills.total <= 16384 < need
        room = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)      # (what lies behind them may hold anything)
        room[:16384] = 0
        for _ in range(3):
            assert torch.equal(w.call(workspace=room), want) and int(room[:16384].count_nonzero()) == 0


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("case", range(6))
def test_append_across_many_skipped_rows(case, rope):
    """Runs of one page with thousands of skipped rows before, between and behind them, and other pages around."""
    gap = lambda n: [-1] * n
    slots = [[64] + gap(5000) + [65],
             gap(3000) + [64, 65, 66] + gap(1023) + [67] + gap(1025) + list(range(68, 128)) + gap(2000),
             list(range(192, 256)) + [130] + gap(4095) + [131, 132, 64] + gap(4096) + [65],
             [64 + i for i in range(10)] + gap(70000) + [74, 75] + gap(10) + [200],
             gap(2048) + [64] + gap(63) + [65] + gap(64) + [66] + gap(1984) + [320],
             [7 * 64 + 5] + gap(1500) + [10 ** 9, -5] + gap(1500) + [7 * 64 + 6] + gap(1100)][case]
    g = torch.Generator(device=DEV).manual_seed(60 + case)
    pages, N = 9, len(slots)
    pos = [i % 90 for i in range(N)]
    for i in range(0, N, 7):                       # (rows that only their position skips)
        if slots[i] < 0 and rope:
            slots[i], pos[i] = 3, (-1, 100)[i % 2]
    cache = random_cache(1, 2, pages, case)
    want = ref.CacheRef(cache)
    size = 2.0 ** torch.randint(-9, 6, (1, N, 1, 1), generator=g, device=DEV).float()
    k, v = (torch.randn((2, 1, N, 2, 64), generator=g, device=DEV) * size).unbind(0)
    cs = tq.rope_table(100) if rope else None
    paged.append(paged.Params(1, 2, 2, cs, F32), cache, k, v, torch.tensor(slots, device=DEV), i32(pos))
    live = [i for i in range(N) if 0 <= slots[i] < 64 * pages and 0 <= pos[i] < 100]
    # (one row after each is enough of a gap for the plain form)
    keep = sorted({j for i in live for j in (i, min(i + 1, N - 1))})
    want.append(k[:, keep].cpu().numpy(), v[:, keep].cpu().numpy(), [slots[i] for i in keep], [pos[i] for i in keep],
                None if cs is None else cs.cpu().numpy(), False)
    same_cache(cache, want)


@pytest.mark.parametrize("lens,new,heads,kv_heads", [([8192, 300], [1, 1], 4, 1), ([9000, 100], [70, 80], 2, 1)])
def test_a_captured_call_without_a_workspace(lens, new, heads, kv_heads):
    w = World(lens, new, heads, kv_heads, seed=45)
    # (tensors made beforehand: a copy from the host cannot be captured)
    args = (i32(w.pos), i32(w.row0), i32(w.table), i32(w.lens), max(new), max(lens))
    q, out = w.q.clone(), torch.empty_like(w.q)
    assert paged.workspace_bytes(w.params, 1, 2, max(new), max(lens)) > 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        paged.attend(w.params, w.cache, q, *args, out=out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        paged.attend(w.params, w.cache, q, *args, out=out)
    g = torch.Generator(device=DEV).manual_seed(46)
    for i in range(5):
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        out.fill_(7.0)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, paged.attend(w.params, w.cache, q, *args)), i
        if i % 2:
            torch.cuda.synchronize()
