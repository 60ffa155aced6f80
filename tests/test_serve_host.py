"""The serving library without a GPU: exports, struct layouts, what the entry points and the binding refuse, the wait
states of the built code, and the plain forms that the GPU tests compare with."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_26110_amd import TQError, paged, serve
from test_code_hazards import OBJDUMP, _code_objects, too_early
from test_paged_host import FAKE, P, _params, _ref, _rows, stores_whose_data_is_written_next

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(serve.lib_path), reason="libturboesm_serve.so is not built")


def _header():
    with open(os.path.join(ROOT, "include", "turboesm_serve.h")) as f:
        return re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)


def test_library_exports_exactly_the_declared_symbols():
    declared = sorted(set(re.findall(r"\bTQ_API\b[^;(]*?\b(tqs_\w+)\s*\(", _header())))
    assert declared == sorted(["tqs_append", "tqs_attend", "tqs_cache_bytes", "tqs_last_error", "tqs_norm_rope", "tqs_read",
                               "tqs_verify", "tqs_verify_workspace_bytes", "tqs_workspace_bytes"])
    out = subprocess.run(["nm", "-D", "--defined-only", serve.lib_path], capture_output=True, text=True, check=True)
    assert sorted(ln.split()[-1] for ln in out.stdout.splitlines() if " T " in ln) == declared


def test_constants_and_layouts():
    assert re.search(r"#define TQS_MAX_AXES 4\b", _header()) and serve.MAX_AXES == 4
    assert ctypes.sizeof(serve._Cache4) == 32 and serve._Cache4.pages.offset == 24
    assert serve.cache_bytes(33, 20, 17) == 33 * 20 * 17 * 64 * 66 and serve.cache_bytes(-1, 1, 1) == -1


def test_no_register_is_read_too_early(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump is missing")
    instructions = 0
    for i, obj in enumerate(_code_objects(serve.lib_path)):
        path = tmp_path / f"{i}.o"
        path.write_bytes(obj)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", str(path)], capture_output=True,
                                 text=True, check=True).stdout
        instructions += listing.count("\n\tv_")
        found = too_early(listing)
        assert not found, (len(found), found[:5])
        assert not stores_whose_data_is_written_next(listing)
        assert "v_pk_fma_f32" not in listing and "v_pk_mul_f32" not in listing and "v_pk_add_f32" not in listing
    assert instructions > 5000


def _cache(**kw):
    c = dict(k_codes=FAKE, v_codes=FAKE, scales=FAKE, pages=9)
    c.update(kw)
    return serve._Cache4(*[c[n] for n, _ in serve._Cache4._fields_])


def norm(p=_params(), q=_rows(), k=_rows(), rows=5, nlayers=1, qw=FAKE, kw=FAKE, eps=1e-6, pos=FAKE, axes=1, sections=None,
         qo=_rows(), ko=_rows()):
    parts = None if sections is None else (ctypes.c_int32 * len(sections))(*sections)
    return serve._load().tqs_norm_rope(_ref(p), _ref(q), _ref(k), rows, nlayers, P(qw), P(kw), eps, P(pos), axes, parts,
                                       _ref(qo), _ref(ko), None)


def append(p=_params(), c=_cache(), k=_rows(), v=_rows(), rows=5, layer0=0, nlayers=1, slots=FAKE, pos=FAKE):
    return serve._load().tqs_append(_ref(p), _ref(c), _ref(k), _ref(v), rows, layer0, nlayers, P(slots), P(pos), None)


def read(p=_params(), c=_cache(), slots=FAKE, rows=5, layer0=0, nlayers=1, k=FAKE, v=FAKE):
    return serve._load().tqs_read(_ref(p), _ref(c), P(slots), rows, layer0, nlayers, P(k), P(v), None)


def attend(p=_params(), c=_cache(), q=_rows(), rows=5, B=2, layer0=0, nlayers=1, pos=FAKE, row0=FAKE, table=FAKE, width=4,
           seq_len=FAKE, max_new=3, max_len=256, out=FAKE, ws=0, ws_bytes=0):
    return serve._load().tqs_attend(_ref(p), _ref(c), _ref(q), rows, B, layer0, nlayers, P(pos), P(row0), P(table), width,
                                    P(seq_len), max_new, max_len, 1, P(out), P(ws), ws_bytes, None)


def verify(target=FAKE, ts=33, draft=FAKE, ds=33, io=0, vocab=33, rows=8, B=2, tokens=FAKE, row0=FAKE, u=FAKE, un=FAKE,
           seq_len=FAKE, accepted=FAKE, nxt=FAKE, keep=FAKE, ws=0, ws_bytes=0):
    return serve._load().tqs_verify(P(target), ts, P(draft), ds, io, vocab, rows, B, P(tokens), P(row0), P(u), P(un),
                                    P(seq_len), P(accepted), P(nxt), P(keep), P(ws), ws_bytes, None)


@pytest.mark.parametrize("call,kw,code,msg", [
    (norm, dict(p=None), -1, "params"), (norm, dict(p=_params(head_dim=128)), -2, "head_dim"),
    (norm, dict(p=_params(io_dtype=3)), -1, "io_dtype"), (norm, dict(p=_params(flags=1)), -1, "flag"),
    (norm, dict(rows=-1), -1, "rows"), (norm, dict(nlayers=4), -2, "layers"), (norm, dict(nlayers=-1), -1, "nlayers"),
    (norm, dict(eps=-1e-9), -1, "eps"), (norm, dict(eps=float("nan")), -1, "eps"), (norm, dict(eps=float("inf")), -1, "eps"),
    (norm, dict(axes=0), -1, "axes"), (norm, dict(axes=5, sections=[8, 8, 8, 8, 0]), -1, "axes"),
    (norm, dict(axes=2), -1, "sections"), (norm, dict(axes=2, sections=[16, 15]), -2, "32"),
    (norm, dict(axes=2, sections=[33, -1]), -2, "32"), (norm, dict(axes=2, sections=[-1, 33]), -1, "sections"),
    (norm, dict(axes=1, sections=[31]), -2, "32"), (norm, dict(axes=2, sections=[2 ** 31 - 1, 2 ** 31 - 1]), -2, "32"),
    (norm, dict(q=None), -1, "q is NULL"), (norm, dict(k=_rows(data=None)), -1, "k is NULL"),
    (norm, dict(qo=None), -1, "q_out"), (norm, dict(ko=_rows(data=FAKE + 8)), -3, "k_out"),
    (norm, dict(qo=_rows(row=0)), -1, "q_out: a stride"), (norm, dict(ko=_rows(head=0)), -1, "k_out: a stride"),
    (norm, dict(nlayers=2), -1, "q_out: a stride"), (norm, dict(q=_rows(row=500)), -3, "multiples of 8"), (norm, dict(pos=0), -1, "pos"),
    (norm, dict(qw=FAKE + 4), -3, "weights"), (norm, dict(kw=FAKE + 4), -3, "weights"),
    (norm, dict(rows=2 ** 31 - 1), -1, "too many"), (norm, dict(rows=2 ** 24, nlayers=3), -1, "too many"),
    (append, dict(p=None), -1, "params"), (append, dict(c=None), -1, "cache"), (append, dict(c=_cache(k_codes=0)), -1, "NULL"),
    (append, dict(c=_cache(scales=0)), -1, "NULL"), (append, dict(c=_cache(v_codes=FAKE + 8)), -3, "aligned"),
    (append, dict(c=_cache(scales=FAKE + 8)), -3, "aligned"), (append, dict(c=_cache(pages=0)), -5, "pages"),
    (append, dict(c=_cache(pages=2 ** 24 + 1)), -5, "pages"), (append, dict(rows=-1), -1, "rows"),
    (append, dict(layer0=3), -2, "layers"), (append, dict(layer0=-1), -2, "layers"), (append, dict(k=None), -1, "k is NULL"),
    (append, dict(v=_rows(data=FAKE + 2)), -3, "v must be"), (append, dict(v=_rows(head=63)), -3, "multiples"),
    (append, dict(slots=0), -1, "NULL"), (append, dict(pos=0), -1, "NULL"),
    (append, dict(rows=2 ** 29), -1, "too many"), (append, dict(p=_params(rope_positions=0)), -1, "rope_positions"),
    (append, dict(p=_params(rope_cs=FAKE + 4)), -3, "rope_cs"),
    (read, dict(p=None), -1, "params"), (read, dict(c=None), -1, "cache"), (read, dict(rows=-5), -1, "rows"),
    (read, dict(slots=0), -1, "NULL"), (read, dict(k=0), -1, "NULL"), (read, dict(v=0), -1, "NULL"),
    (read, dict(k=FAKE + 8), -3, "aligned"), (read, dict(nlayers=4), -2, "layers"), (read, dict(rows=2 ** 29), -1, "too many"),
    (attend, dict(p=None), -1, "params"), (attend, dict(p=_params(softmax_scale=float("inf"))), -1, "finite"),
    (attend, dict(c=_cache(pages=-1)), -5, "pages"), (attend, dict(rows=-1), -1, "rows"), (attend, dict(B=-1), -1, "rows, B"),
    (attend, dict(max_len=-1), -1, "max_len"), (attend, dict(width=0), -1, "table_width"), (attend, dict(max_new=0), -1, "max_new"),
    (attend, dict(q=None), -1, "q is NULL"), (attend, dict(pos=0), -1, "NULL"), (attend, dict(row0=0), -1, "NULL"),
    (attend, dict(table=0), -1, "NULL"), (attend, dict(seq_len=0), -1, "NULL"), (attend, dict(out=0), -1, "NULL"),
    (attend, dict(out=FAKE + 8), -3, "out"), (attend, dict(max_len=100_000, B=1), -5, "workspace"),
    (attend, dict(max_len=100_000, B=1, ws=FAKE, ws_bytes=1000), -5, "too small"),
    (attend, dict(max_len=100_000, B=1, ws=FAKE + 8, ws_bytes=2 ** 40), -3, "workspace"),
    (attend, dict(rows=2 ** 30), -1, "too many"), (attend, dict(B=2 ** 30), -1, "too many"),
    (attend, dict(max_new=2 ** 29), -1, "too many"), (attend, dict(B=2 ** 24, max_new=1), -1, "too many"),
    (verify, dict(io=3), -1, "io_dtype"), (verify, dict(vocab=0), -1, "vocab"), (verify, dict(vocab=2 ** 24 + 1), -1, "vocab"),
    (verify, dict(rows=-1), -1, "rows"), (verify, dict(B=-1), -1, "B must"), (verify, dict(B=4097), -1, "4096"),
    (verify, dict(target=0), -1, "NULL"), (verify, dict(tokens=0), -1, "NULL"), (verify, dict(row0=0), -1, "NULL"),
    (verify, dict(u=0), -1, "NULL"), (verify, dict(un=0), -1, "NULL"), (verify, dict(accepted=0), -1, "NULL"),
    (verify, dict(nxt=0), -1, "NULL"), (verify, dict(keep=0), -1, "NULL"), (verify, dict(ts=32), -1, "strides"),
    (verify, dict(ds=32), -1, "strides"), (verify, dict(target=FAKE + 2), -3, "aligned"),
    (verify, dict(draft=FAKE + 1, io=1), -3, "aligned"), (verify, dict(vocab=50_000, ts=50_000, ds=50_000), -5, "workspace"),
    (verify, dict(vocab=50_000, ts=50_000, ds=50_000, ws=FAKE, ws_bytes=16384), -5, "too small")])
def test_what_is_refused(call, kw, code, msg):
    assert call(**kw) == code, serve.last_error()
    assert msg in serve.last_error()


def test_nothing_to_do_is_success():
    assert norm(rows=0) == 0 and norm(nlayers=0) == 0 and append(rows=0) == 0 and append(nlayers=0) == 0
    assert read(rows=0, k=0, v=0) == 0 and read(nlayers=0) == 0
    assert attend(rows=0) == 0 and attend(B=0) == 0 and attend(nlayers=0) == 0 and verify(B=0) == 0
    assert serve.last_error() == ""


def test_workspaces():
    p = paged.Params(33, 40, 8)
    assert serve.workspace_bytes(p, 1, 0, 1, 100) == serve.workspace_bytes(p, 1, 2 ** 30, 1, 100) == 0
    assert serve.workspace_bytes(p, 1, 1, 1, 100_000) > 16384 and serve.workspace_bytes(p, 33, 64, 1, 100) == 0
    assert serve.verify_workspace_bytes(33, 4096) == serve.verify_workspace_bytes(2048, 5) == 0
    assert serve.verify_workspace_bytes(2049, 3) == 16384 + 3 * 2 * 8
    assert serve.verify_workspace_bytes(2 ** 24, 4096) <= 16384 + 4096 * 256 * 8
    assert serve.verify_workspace_bytes(0, 3) == serve.verify_workspace_bytes(2 ** 24 + 1, 3) == 0
    assert serve.verify_workspace_bytes(5000, 0) == serve.verify_workspace_bytes(5000, 4097) == 0


def test_binding_refuses():
    z = torch.zeros(4, dtype=torch.int32)
    cache, params = serve.Cache4(1, 2, 3, device="cpu"), paged.Params(1, 4, 2)
    x, q = torch.zeros((1, 4, 2, 64), dtype=torch.float16), torch.zeros((1, 4, 4, 64), dtype=torch.float16)
    p = torch.zeros((4, 7))
    for call in (lambda: serve.norm_rope(params, q, x), lambda: serve.append(params, cache, x, x, z.long()),
                 lambda: serve.read(params, cache, z.long()),
                 lambda: serve.attend(params, cache, q, z, z, z.view(2, 2), z, 1, 64),
                 lambda: serve.verify(p, p, z.long(), z, p[:, 0], p[:, 0]),
                 lambda: serve.append(params, paged.Cache(1, 2, 3, device="cpu"), x, x, z.long()),
                 lambda: paged.append(params, cache, x, x, z.long())):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(ValueError):
        serve.append(paged.Params(2, 4, 2), cache, x, x, z.long())
    with pytest.raises(ValueError):
        serve.Cache4(1, 2, 0)
    with pytest.raises(ValueError):
        serve.verify_workspace_bytes(2 ** 32 + 1, 1)
    with pytest.raises(ValueError):
        serve.cache_bytes(2 ** 32 + 1, 1, 1)
    assert issubclass(TQError, RuntimeError)


def test_a_cache_keeps_its_buffers():
    cache = serve.Cache4(2, 3, 5, device="cpu")
    assert cache.k_codes.shape == (2, 3, 5, 2048) and cache.scales.shape == (2, 3, 5, 128)
    for name in ("k_codes", "v_codes", "scales", "pages", "num_layers", "kv_heads", "device"):
        with pytest.raises(AttributeError):
            setattr(cache, name, object())
        with pytest.raises(AttributeError):
            delattr(cache, name)
    cache.label = "a caller's own"
    cache.scales += 1
    assert int(cache.scales[0, 0, 0, 0]) == 128


# ---------------------------------------------------- the plain forms
def test_reference_codes_are_the_nearest():
    x = np.concatenate([np.linspace(-8, 8, 32001), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -2.5, -3.5, -5.0]])
    got = ref.value_of(ref.e2m1(x))
    far = np.abs(np.clip(x, -6, 6)[:, None] - np.concatenate([ref.GRID, -ref.GRID])).min(1)
    assert np.array_equal(np.abs(np.clip(x, -6, 6) - got), far)
    assert list(got[-12:]) == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, -1.0, -2.0, -4.0, -4.0]
    assert list(ref.e2m1([1e30, -1e30, 2.0 ** 60])) == [7, 15, 7]
    for e in (-30, 0, 20):
        assert ref.exponent(6 * 2.0 ** e) == e and ref.exponent(6.0001 * 2.0 ** e) == e + 1
    assert ref.exponent(0.0) == ref.exponent(1e-300) == -48 and ref.exponent(1e300) == 47


def test_reference_hadamard_is_the_matrix_and_its_own_inverse():
    x = np.random.default_rng(1).standard_normal((50, 64)).astype(np.float32)
    # (six roundings of sums whose sizes are at most the sum of |x|)
    room = 7 * 2.0 ** -24 * np.abs(x.astype(np.float64)).sum(-1, keepdims=True) / 8
    assert (np.abs(ref.hadamard32(x) - x.astype(np.float64) @ ref.SIGNS / 8) <= room).all()
    assert np.allclose(ref.SIGNS @ ref.SIGNS, 64 * np.eye(64))


def test_reference_layout_gives_every_code_its_own_place():
    for where in (ref.KEY, ref.VALUE):
        nibbles = 2 * where + np.arange(64) % 2
        assert sorted(nibbles.ravel()) == list(range(4096))
    assert sorted([*ref.KEY_SCALE, *ref.VALUE_SCALE]) == list(range(128))


def test_reference_verify_draws_the_target():
    # over all pairs of random numbers on a grid the token after one draft is distributed as the target's
    p, q = np.array([[0.5, 0.25, 0.25, 0.0], [0.25, 0.25, 0.25, 0.25]]), np.array([[0.25, 0.5, 0.0, 0.25]] * 2)
    count, n = np.zeros(4), 0
    for d, weight in enumerate(q[0]):
        for i in range(64):
            for j in range(64):
                a, k, t = ref.verify(p, q, [0, d], [0, 2], [(i + 0.5) / 64, 0], [(j + 0.5) / 64], [10])
                assert k == [9 + a[0]]
                count[d if a[0] else t[0]] += weight / 4096
    assert np.allclose(count, p[0], atol=1e-12)
