"""The paged cache without a GPU: exports, struct layouts, what the entry points and the binding refuse, the wait states
of the built code, and the plain forms that the GPU tests compare with."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2603_26110_amd import TQError, paged
from test_code_hazards import OBJDUMP, _code_objects, _registers, too_early

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(paged.lib_path), reason="libturboesm_paged.so is not built")
FAKE = 0x10000          # aligned, not null, never dereferenced
P = ctypes.c_void_p


def _header():
    with open(os.path.join(ROOT, "include", "turboesm_paged.h")) as f:
        return re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)


def test_library_exports_exactly_the_declared_symbols():
    declared = sorted(set(re.findall(r"\bTQ_API\b[^;(]*?\b(tqp_\w+)\s*\(", _header())))
    assert declared == sorted(["tqp_assign", "tqp_release", "tqp_append", "tqp_attend", "tqp_workspace_bytes",
                               "tqp_cache_bytes", "tqp_last_error"])
    out = subprocess.run(["nm", "-D", "--defined-only", paged.lib_path], capture_output=True, text=True, check=True)
    assert sorted(ln.split()[-1] for ln in out.stdout.splitlines() if " T " in ln) == declared


def test_constants_and_layouts():
    h = _header()
    assert re.search(r"#define TQP_PAGE 64\b", h) and re.search(r"#define TQP_MAX_SEQS 4096\b", h)
    assert re.search(r"#define TQP_BF16 2\b", h) and paged._IO[torch.bfloat16] == 2
    assert (paged.PAGE, paged.MAX_SEQS) == (64, 4096)
    assert ctypes.sizeof(paged._Params) == 40 and paged._Params.rope_cs.offset == 32
    assert ctypes.sizeof(paged._Cache) == 32 and ctypes.sizeof(paged._Pool) == 24 and ctypes.sizeof(paged._Rows) == 32
    assert paged.cache_bytes(33, 20, 17) == 33 * 20 * 17 * 8200 and paged.cache_bytes(-1, 1, 1) == -1


def test_no_register_is_read_too_early(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump is missing")
    instructions = 0
    for i, obj in enumerate(_code_objects(paged.lib_path)):
        path = tmp_path / f"{i}.o"
        path.write_bytes(obj)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", str(path)], capture_output=True,
                                 text=True, check=True).stdout
        instructions += listing.count("\n\tv_")
        found = too_early(listing)
        assert not found, (len(found), found[:5])
        assert "v_pk_fma_f32" not in listing and "v_pk_mul_f32" not in listing and "v_pk_add_f32" not in listing
    assert instructions > 5000


def _params(**kw):
    p = dict(head_dim=64, num_layers=3, num_heads=8, kv_heads=2, io_dtype=1, flags=0, softmax_scale=0.125,
             rope_positions=100, rope_cs=FAKE)
    p.update(kw)
    return paged._Params(*[p[n] for n, _ in paged._Params._fields_])


def _cache(**kw):
    c = dict(k_codes=FAKE, v_codes=FAKE, scales=FAKE, pages=9)
    c.update(kw)
    return paged._Cache(*[c[n] for n, _ in paged._Cache._fields_])


def _rows(data=FAKE, layer=0, row=512, head=64):
    return paged._Rows(data, layer, row, head)


def _pool(stack=FAKE, state=FAKE, pages=9):
    return paged._Pool(stack, state, pages)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def assign(pool=_pool(), table=FAKE, width=4, B=2, seq_len=FAKE, new=FAKE, rows=5, slots=FAKE, pos=FAKE, row0=FAKE,
           granted=FAKE):
    return paged._load().tqp_assign(_ref(pool), P(table), width, B, P(seq_len), P(new), rows, P(slots), P(pos), P(row0),
                                    P(granted), None)


def release(pool=_pool(), table=FAKE, width=4, B=2, seq_len=FAKE, keep=FAKE):
    return paged._load().tqp_release(_ref(pool), P(table), width, B, P(seq_len), P(keep), None)


def append(p=_params(), c=_cache(), k=_rows(), v=_rows(), rows=5, layer0=0, nlayers=1, slots=FAKE, pos=FAKE):
    return paged._load().tqp_append(_ref(p), _ref(c), _ref(k), _ref(v), rows, layer0, nlayers, P(slots), P(pos), None)


def attend(p=_params(), c=_cache(), q=_rows(), rows=5, B=2, layer0=0, nlayers=1, pos=FAKE, row0=FAKE, table=FAKE, width=4,
           seq_len=FAKE, max_new=3, max_len=256, out=FAKE, ws=0, ws_bytes=0):
    return paged._load().tqp_attend(_ref(p), _ref(c), _ref(q), rows, B, layer0, nlayers, P(pos), P(row0), P(table), width,
                                    P(seq_len), max_new, max_len, 1, P(out), P(ws), ws_bytes, None)


@pytest.mark.parametrize("call,kw,code,msg", [
    (assign, dict(pool=None), -1, "pool"), (assign, dict(pool=_pool(stack=0)), -1, "NULL"),
    (assign, dict(pool=_pool(state=0)), -1, "NULL"), (assign, dict(pool=_pool(pages=0)), -5, "pages"),
    (assign, dict(pool=_pool(pages=2 ** 24 + 1)), -5, "pages"), (assign, dict(B=-1), -1, "B must"),
    (assign, dict(B=4097), -1, "4096"), (assign, dict(width=0), -1, "table_width"), (assign, dict(rows=-1), -1, "rows"),
    (assign, dict(table=0), -1, "NULL"), (assign, dict(seq_len=0), -1, "NULL"), (assign, dict(new=0), -1, "NULL"),
    (assign, dict(slots=0), -1, "NULL"), (assign, dict(pos=0), -1, "NULL"), (assign, dict(row0=0), -1, "NULL"),
    (assign, dict(granted=0), -1, "NULL"),
    (release, dict(pool=None), -1, "pool"), (release, dict(B=4097), -1, "4096"), (release, dict(width=-3), -1, "table_width"),
    (release, dict(keep=0), -1, "keep"), (release, dict(table=0), -1, "NULL"),
    (append, dict(p=None), -1, "params"), (append, dict(p=_params(head_dim=128)), -2, "head_dim"),
    (append, dict(p=_params(num_layers=0)), -1, "positive"), (append, dict(p=_params(kv_heads=0)), -1, "positive"),
    (append, dict(p=_params(num_heads=7)), -2, "multiple"), (append, dict(p=_params(io_dtype=3)), -1, "io_dtype"),
    (append, dict(p=_params(flags=1)), -1, "flag"), (append, dict(p=_params(flags=16)), -1, "flag"),
    (append, dict(p=_params(softmax_scale=float("nan"))), -1, "finite"),
    (append, dict(p=_params(rope_cs=FAKE + 8)), -3, "rope_cs"), (append, dict(p=_params(rope_positions=0)), -1, "rope_positions"),
    (append, dict(c=None), -1, "cache"), (append, dict(c=_cache(k_codes=0)), -1, "NULL"),
    (append, dict(c=_cache(v_codes=FAKE + 8)), -3, "16-byte"), (append, dict(c=_cache(scales=FAKE + 4)), -3, "8-byte"),
    (append, dict(c=_cache(pages=0)), -5, "pages"), (append, dict(rows=-1), -1, "rows"),
    (append, dict(layer0=3), -2, "layers"), (append, dict(layer0=-1), -2, "layers"), (append, dict(nlayers=-1), -1, "nlayers"),
    (append, dict(layer0=2 ** 31 - 1, nlayers=2 ** 31 - 1), -2, "layers"),
    (append, dict(k=None), -1, "k is"), (append, dict(v=_rows(data=0)), -1, "v is"),
    (append, dict(k=_rows(data=FAKE + 8)), -3, "aligned"), (append, dict(v=_rows(row=516)), -3, "strides"),
    (append, dict(k=_rows(head=4)), -3, "strides"), (append, dict(k=_rows(row=2 ** 23 + 8)), -1, "row strides"),
    (append, dict(v=_rows(row=-64)), -1, "row strides"), (append, dict(p=_params(rope_positions=2 ** 23 + 1)), -1, "2^23"), (append, dict(slots=0), -1, "NULL"), (append, dict(pos=0), -1, "NULL"),
    (append, dict(p=_params(num_layers=2 ** 20, num_heads=2 ** 20, kv_heads=2 ** 20), nlayers=2 ** 20), -1, "too many"),
    (attend, dict(p=None), -1, "params"), (attend, dict(c=None), -1, "cache"), (attend, dict(q=None), -1, "q is"),
    (attend, dict(rows=-1), -1, "rows"), (attend, dict(B=-1), -1, "B"), (attend, dict(max_len=-1), -1, "max_len"),
    (attend, dict(max_new=0), -1, "max_new"), (attend, dict(width=0), -1, "table_width"),
    (attend, dict(pos=0), -1, "NULL"), (attend, dict(row0=0), -1, "NULL"), (attend, dict(table=0), -1, "NULL"),
    (attend, dict(seq_len=0), -1, "NULL"), (attend, dict(out=0), -1, "NULL"), (attend, dict(out=FAKE + 8), -3, "out"),
    (attend, dict(q=_rows(layer=4)), -3, "strides"), (attend, dict(max_new=2 ** 30), -1, "too many"),
    (attend, dict(max_new=1, max_len=100000), -5, "workspace"),
    (attend, dict(max_new=1, max_len=100000, ws=FAKE, ws_bytes=64), -5, "too small"),
    (attend, dict(max_new=1, max_len=100000, ws=FAKE + 8, ws_bytes=1 << 40), -3, "workspace"),
])
def test_what_is_refused(call, kw, code, msg):
    assert call(**kw) == code, paged.last_error()
    assert msg in paged.last_error()


@pytest.mark.parametrize("call,kw", [
    (append, dict(rows=2 ** 31 - 1)), (append, dict(rows=2 ** 30, p=_params(kv_heads=1))),
    (append, dict(rows=64, p=_params(num_layers=2 ** 12, num_heads=2 ** 13, kv_heads=2 ** 13), nlayers=2 ** 12)),
    (attend, dict(B=2 ** 23)), (attend, dict(B=2 ** 15, max_new=2 ** 16)),
    (attend, dict(B=2 ** 20, p=_params(num_heads=64, kv_heads=16), max_new=1)),
    (attend, dict(B=2 ** 30, p=_params(num_layers=2 ** 30, num_heads=2 ** 30, kv_heads=2 ** 30), nlayers=2 ** 30)),
])
def test_launches_that_would_not_fit_are_refused(call, kw):
    assert call(**kw) == -1 and "too many" in paged.last_error()


def test_workspace_of_sizes_that_do_not_fit():
    L, p = paged._load(), _params(num_layers=2 ** 30, num_heads=2 ** 30, kv_heads=2 ** 30)
    assert L.tqp_workspace_bytes(ctypes.byref(p), 2 ** 30, 2 ** 30, 1, 8192) == 0
    assert L.tqp_workspace_bytes(ctypes.byref(p), 16, 2 ** 30, 1, 8192) == 0


def test_nothing_to_do_is_success():
    assert release(B=0, table=0, seq_len=0, keep=0) == 0
    assert append(rows=0, k=None) == 0 and append(nlayers=0) == 0
    assert attend(rows=0) == 0 and attend(B=0) == 0 and attend(nlayers=0) == 0
    assert paged.last_error() == ""
    L, p = paged._load(), _params()
    assert L.tqp_workspace_bytes(None, 1, 1, 1, 64) == 0
    for a in ((0, 1, 1, 64), (1, 0, 1, 64), (1, 1, 0, 64), (1, 1, 1, -1), (1, 1, 1, 64), (1, 1000, 1, 8192)):
        assert L.tqp_workspace_bytes(ctypes.byref(p), *a) == 0
    assert L.tqp_workspace_bytes(ctypes.byref(p), 1, 1, 1, 8192) > 16384


def test_binding_refuses_host_tensors():
    z = torch.zeros(4, dtype=torch.int32)
    pool = paged.PagePool(4, device="cpu")
    with pytest.raises(TypeError):
        paged.assign(pool, z.view(2, 2), z, z, 4)
    with pytest.raises(TypeError):
        paged.release(pool, z.view(2, 2), z, z)
    cache, params = paged.Cache(1, 2, 3, device="cpu"), paged.Params(1, 4, 2)
    x = torch.zeros((1, 4, 2, 64), dtype=torch.float16)
    with pytest.raises(TypeError):
        paged.append(params, cache, x, x, z.long(), z)
    with pytest.raises(TypeError):
        paged.attend(params, cache, x, z, z, z.view(2, 2), z, 1, 64)
    with pytest.raises(ValueError):
        paged.append(paged.Params(2, 4, 2), cache, x, x, z.long(), z)
    with pytest.raises(TypeError):
        paged.Params(1, 4, 2, io_dtype=torch.float64).c()
    with pytest.raises(ValueError):
        paged.Cache(1, 0, 3)
    with pytest.raises(ValueError):
        paged.PagePool(0)
    assert issubclass(TQError, RuntimeError)


# ---------------------------------------------------- the plain forms
def test_reference_e4m3_is_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.decode(codes.numpy()), want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 100001), np.random.default_rng(1).standard_normal(20000) * 0.01])
    x = x.astype(np.float32)
    assert np.array_equal(ref.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    for e in (-30, 0, 20):
        assert ref.exponent(448 * 2.0 ** e) == e and ref.exponent(448.001 * 2.0 ** e) == e + 1
    assert ref.exponent(0.0) == ref.exponent(1e-300) == -48 and ref.exponent(1e300) == 47


def test_reference_attend_is_softmax_attention():
    g = torch.Generator().manual_seed(1)
    k, v = torch.randn((2, 1, 2, 5, 64, 64), generator=g, dtype=torch.float64).unbind(0)
    q = torch.randn((1, 6, 4, 64), generator=g, dtype=torch.float64)
    table, lens, row0 = [[3, 0, 1], [4, -1, -1], [2, -1, -1]], [150, 0, 64], [0, 4, 5, 6]
    pos = [146, 147, 148, 149, 0, 63]
    out, spread, size = ref.attend(k, v, q, pos, row0, table, lens, True, 0.125)
    for row, b in ((0, 0), (3, 0), (5, 2)):
        for h in range(4):
            toks = [(table[b][t // 64], t % 64) for t in range(pos[row] + 1)]
            s = torch.stack([q[0, row, h] @ k[0, h // 2, p, t] for p, t in toks]) / 8
            o = sum(w * v[0, h // 2, p, t] for w, (p, t) in zip(torch.softmax(s, 0), toks))
            assert torch.allclose(out[0, row, h], o, rtol=1e-12, atol=1e-12)
    assert bool((out[0, 4] == 0).all()) and bool((spread[0][0, :4] >= out[0, :4].abs() - 1e-12).all()) and float(size.max()) > 0


def test_reference_pool_gives_back_what_it_took():
    g = np.random.default_rng(3)
    state = ref.Pool(range(30), [[-1] * 4 for _ in range(6)], [0] * 6)
    for _ in range(20):
        before = (list(state.stack), [list(r) for r in state.table], list(state.len))
        new = g.integers(0, 100, 6).tolist()
        _, _, _, granted = state.assign(new, sum(new), 30)
        state.release([n - m * ok for n, m, ok in zip(state.len, new, granted)])
        assert before == (state.stack, state.table, state.len)
        state.assign([1] * 6, 6, 30)


def test_a_cache_and_a_pool_keep_their_buffers():
    # (the library is given their addresses as they were made)
    cache, pool = paged.Cache(2, 3, 5, device="cpu"), paged.PagePool(5, device="cpu")
    for thing, names in ((cache, ("k_codes", "v_codes", "scales", "pages", "num_layers", "kv_heads", "device")),
                         (pool, ("stack", "state", "pages", "device"))):
        for name in names:
            was = getattr(thing, name)
            with pytest.raises(AttributeError):
                setattr(thing, name, was.clone() if isinstance(was, torch.Tensor) else object())
            with pytest.raises(AttributeError):
                delattr(thing, name)
            assert getattr(thing, name) is was
    pool.state[0] = 3                              # what they hold may change
    cache.scales[..., 1] *= 2
    assert pool.state[0] == 3 and float(cache.scales[0, 0, 0, 1]) == 2.0 ** -47


def test_numbers_past_32_bits_are_refused_not_cut():
    wide = 2 ** 32 + 1                             # (1 in 32 bits)
    for kw in (dict(num_layers=wide), dict(num_heads=wide), dict(kv_heads=wide), dict(num_layers=-2 ** 32 + 1),
               dict(flags=2 ** 32)):
        with pytest.raises(ValueError):
            paged.Params(**{**dict(num_layers=1, num_heads=1, kv_heads=1), **kw})
    params = paged.Params(1, 1, 1)
    for i in range(4):
        sizes = [1, 1, 1, 100_000]
        assert paged.workspace_bytes(params, *sizes) > 0
        sizes[i] = wide
        with pytest.raises(ValueError):
            paged.workspace_bytes(params, *sizes)
    for args in ((wide, 1, 1), (1, wide, 1)):
        with pytest.raises(ValueError):
            paged.cache_bytes(*args)
    assert paged.cache_bytes(1, 1, 2 ** 33) == 2 ** 33 * 8200


def stores_whose_data_is_written_next(listing):
    """(store, writer) of the stores of more than two words whose data the very next instruction writes (gfx9 wants a
    wait state between them, which the compiler keeps for its own stores but not for those in assembly)."""
    lines = [ln.split("//")[0].strip() for ln in listing.splitlines() if ln.startswith("\t")]
    found = []
    for store, after in zip(lines, lines[1:]):
        if re.match(r"(global|flat|scratch)_store_dwordx[34]\b", store) and after.startswith("v_"):
            data = _registers(store.split(",")[1].strip())
            if set(data) & set(_registers(after.partition(" ")[2].split(",")[0].strip())):
                found.append((store, after))
    return found


def test_no_store_loses_its_data(tmp_path):
    code = "\tglobal_store_dwordx4 v[0:1], v[4:7], off sc1   // 0:\n{}\tv_mov_b32_e32 v7, 0   // 8:\n"
    assert len(stores_whose_data_is_written_next(code.format(""))) == 1
    assert not stores_whose_data_is_written_next(code.format("\ts_nop 0\n"))
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump is missing")
    ours = 0
    for i, obj in enumerate(_code_objects(paged.lib_path)):
        path = tmp_path / f"{i}.o"
        path.write_bytes(obj)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", str(path)], capture_output=True,
                                 text=True, check=True).stdout
        assert not stores_whose_data_is_written_next(listing)
        lines = [ln.split("//")[0].strip() for ln in listing.splitlines() if ln.startswith("\t")]
        for store, after in zip(lines, lines[1:]):
            if re.match(r"global_store_dwordx4 .* sc1$", store):
                ours += 1
                assert re.match(r"s_nop", after), (store, after)
    assert ours > 0


def test_a_cache_and_a_pool_take_attributes_of_the_caller_s():
    for thing in (paged.Cache(1, 1, 2, device="cpu"), paged.PagePool(2, device="cpu")):
        thing.name = "mine"
        thing.name += " too"
        assert thing.name == "mine too"
        del thing.name
        assert not hasattr(thing, "name")
    cache = paged.Cache(1, 1, 2, device="cpu")
    cache.scales *= 2                              # (the tensor that is there already, changed in place)
    assert float(cache.scales[0, 0, 0, 0]) == 2.0 ** -47
