"""Host-side checks of the operators over packed token rows (no GPU needed): their descriptor's C layout, what
is refused at creation, tile spaces, the rotary frequencies, the Python entry points' checks, and the float64
oracle against independent formulations."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import sequences as seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000000  # device addresses that nothing reads


@pytest.fixture(scope="module")
def L():
    from paper_2307_04339_amd import _lib
    _lib.load()
    return _lib


def _create(L, **fields):
    d = L.SeqDesc()
    for k, v in fields.items():
        setattr(d, k, v)
    h = ctypes.c_void_p()
    rc = L.load().miriam_seq_op_create(ctypes.byref(d), ctypes.byref(h))
    return rc, h


def _info(L, h):
    info = L.OpInfo()
    assert L.load().miriam_op_query(h, ctypes.byref(info)) == 0
    return info


def _at(i):
    return FAKE + i * (1 << 32)  # buffers of their own


NORM = dict(kind=16, dtype=2, tokens=10, n=768, scale=1.0, eps=1e-5, x=_at(1), y=_at(2), z=_at(3), residual=_at(4), pre=_at(5),
            post=_at(6))
ROT = dict(kind=17, dtype=1, tokens=10, seqs=2, heads=4, kv_heads=2, head_dim=64, rot=64, page=16, pages=8, max_pages=4, scale=1.0,
           cache_page=2048, cache_head=1024, cache_token=64, x=_at(1), y=_at(2), k_cache=_at(3), v_cache=_at(4), q_start=_at(5),
           kv_len=_at(6), page_table=_at(7), freq=_at(8))
ATT = dict(ROT, kind=18, flags=2, rot=0, scale=0.125)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_descriptor_matches_the_c_layout(L, tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "miriam.h"', "int main(void) {",
             '    printf("size %zu\\n", sizeof(miriam_seq_desc));']
    for name, _ in L.SeqDesc._fields_:
        lines.append(f'    printf("{name} %zu\\n", offsetof(miriam_seq_desc, {name}));')
    for name in ("MIRIAM_OP_BLOCK_NORM", "MIRIAM_OP_ROTARY", "MIRIAM_OP_ATTENTION", "MIRIAM_SEQ_INTERLEAVED", "MIRIAM_SEQ_CAUSAL",
                 "MIRIAM_SEQ_LAYER_NORM", "MIRIAM_GATE_NONE", "MIRIAM_GATE_CHANNEL", "MIRIAM_GATE_ROWS", "MIRIAM_GATE_SILU", "MIRIAM_GATE_SIGMOID"):
        lines.append(f'    printf("{name} %d\\n", (int){name});')
    lines += ["    return 0;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n") if l)
    assert int(got.pop("size")) == ctypes.sizeof(L.SeqDesc)
    for name, value in got.items():
        want = getattr(L, name[len("MIRIAM_"):]) if name.startswith("MIRIAM_") else getattr(L.SeqDesc, name).offset
        assert int(value) == want, name


# -------------------------------------------------------------------- refusals
@pytest.mark.parametrize("base,changes", [(b, c) for b, cs in [
    (NORM, [dict(tokens=0), dict(n=0), dict(x=None), dict(y=None, z=None, pre=None), dict(z=None), dict(pre=None),
            dict(post=None, post_bias=_at(9)), dict(gate=_at(9)), dict(gate_kind=3), dict(gate=_at(9), gate_kind=5),
            dict(gate=_at(9), gate_kind=-1), dict(flags=1), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
            dict(scale=math.nan), dict(ldx=767), dict(ldy=5), dict(ldr=1), dict(ldz=767), dict(ldg=767), dict(dtype=3), dict(dtype=-1),
            dict(y=_at(1)), dict(y=_at(4)), dict(z=_at(1)), dict(z=_at(2)), dict(z=_at(4) + 2 * 768 * 3), dict(x=_at(1) + 1),
            dict(post=_at(6) + 2), dict(tokens=1 << 31), dict(n=1 << 31), dict(kind=19), dict(kind=0),
            dict(gate=_at(2), gate_kind=2)]),
    (ROT, [dict(tokens=0), dict(seqs=0), dict(heads=0), dict(kv_heads=-1), dict(head_dim=0), dict(rot=3), dict(rot=66), dict(rot=-2),
           dict(freq=None), dict(freq=_at(8) + 4), dict(x=None), dict(y=None), dict(q_start=None), dict(kv_len=None), dict(page_table=None),
           dict(k_cache=None), dict(v_cache=None), dict(page=0), dict(pages=0), dict(max_pages=0), dict(ldt=3), dict(ldx=511), dict(ldy=255),
           dict(cache_page=0), dict(cache_head=0), dict(cache_token=0), dict(cache_token=32), dict(flags=2), dict(scale=math.inf),
           dict(y=_at(1)), dict(y=_at(1) + 64, ldy=512), dict(page=1 << 20, max_pages=1 << 11), dict(q_start=_at(5) + 2),
           dict(heads=1 << 29), dict(x=_at(1) + 1)]),
    (ATT, [dict(dtype=0), dict(heads=3), dict(kv_heads=0), dict(head_dim=4), dict(head_dim=264), dict(head_dim=68), dict(window=-1),
           dict(max_q=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(flags=1), dict(x=_at(1) + 2),
           dict(y=_at(2) + 8), dict(k_cache=_at(3) + 4), dict(v_cache=_at(4) + 2), dict(ldx=258), dict(ldy=260), dict(cache_page=2049),
           dict(cache_head=1028), dict(cache_token=68), dict(y=_at(1)), dict(page_table=None), dict(kv_len=None), dict(pages=0),
           dict(ldt=1), dict(tokens=1 << 28, heads=64, kv_heads=1)]),
] for c in cs])
def test_refusals(L, base, changes):
    rc, h = _create(L, **dict(base, **changes))
    assert rc == L.EINVAL and h.value is None, changes
    assert L.load().miriam_last_error()


@pytest.mark.parametrize("base,changes", [(b, c) for b, cs in [
    (NORM, [dict(y=_at(6)), dict(z=_at(5) - 64), dict(post_bias=_at(9), y=_at(9) + 16), dict(gate=_at(9), gate_kind=1, z=_at(9) + 764 * 4),
            dict(pre_bias=_at(9), z=_at(9) - 10 * 768 * 2 + 2)]),
    (ROT, [dict(v_cache=_at(3)), dict(x=_at(3)), dict(y=_at(4)), dict(y=_at(3) - 64), dict(x=_at(4) + 2 * 2048 * 7), dict(cache_page=1 << 60),
           dict(cache_head=1 << 62), dict(cache_token=1 << 60)]),
    (ATT, [dict(y=_at(3)), dict(y=_at(4) - 512), dict(y=_at(4) + 2 * (2048 * 7 + 1024 + 15 * 64)), dict(scale=3e38), dict(cache_page=1 << 60)]),
] for c in cs])
def test_overlaps_and_sizes_are_refused(L, base, changes):
    test_refusals(L, base, changes)


@pytest.mark.parametrize("base,changes", [
    (NORM, dict(post=_at(2) + 10 * 768 * 2)),                 # right behind the output
    (ROT, dict(v_cache=_at(3) + 2048, cache_page=4096)),      # keys and values of a page one after the other
    (ATT, dict(x=_at(3), v_cache=_at(3), y=_at(3) + 2 * 2048 * 8)),   # only read: may share memory
])
def test_neighbours_are_no_overlap(L, base, changes):
    rc, h = _create(L, **dict(base, **changes))
    assert rc == 0, L.load().miriam_last_error()
    L.load().miriam_op_destroy(h)


def test_null_arguments(L):
    h = ctypes.c_void_p()
    for fn in (L.load().miriam_seq_op_create, L.load().miriam_seq_op_create_noalloc):
        assert fn(None, ctypes.byref(h)) == L.EINVAL and fn(ctypes.byref(L.SeqDesc()), None) == L.EINVAL


@pytest.mark.parametrize("base,changes,tiles", [
    (NORM, {}, 3),                           # a logical wave per row
    (NORM, dict(n=512), 3), (NORM, dict(n=1024), 3),   # beyond, the four of a tile
    (NORM, dict(n=1025), 10), (NORM, dict(n=100000), 10),
    (NORM, dict(y=_at(1) + 1536, ldx=2000, ldy=2000), 3),   # columns of their own in rows of one buffer
    (NORM, dict(gate=_at(9), gate_kind=1), 3),
    (ATT, dict(max_q=1), 4),                 # without a device: a tile per sequence and cache head
    (ATT, {}, 4),                            # tiles of 128 rows: at most one per sequence here
    (ATT, dict(tokens=1000, max_q=500), 32),
])
def test_tile_spaces(L, base, changes, tiles):
    rc, h = _create(L, **dict(base, **changes))
    assert rc == 0, L.load().miriam_last_error()
    info = _info(L, h)
    assert info.num_tiles == tiles and info.path == L.PATH_OTHER and info.ksplit == 1
    for b, l, grid, block, want in [(-1, 1, 1, 256, L.ERANGE), (0, tiles + 1, 1, 256, L.ERANGE), (0, 1, 0, 256, L.ERANGE), (0, 1, 1, 32, L.ERANGE)]:
        assert L.load().miriam_elastic_launch(h, b, l, grid, block, None) == want
    assert L.load().miriam_op_destroy(h) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="device -1 is a host without one")
def test_launch_on_another_device_is_refused(L):
    rc, h = _create(L, **ATT)
    assert rc == 0
    assert L.load().miriam_op_run(h, None) == L.EINVAL
    assert b"another device" in L.load().miriam_last_error()
    L.load().miriam_op_destroy(h)


def test_work_of_the_operators(L):
    rc, h = _create(L, **dict(NORM, gate=_at(9), gate_kind=3))
    assert _info(L, h).bytes == 2 * 10 * 768 * 5 + 2 * 4 * 768
    L.load().miriam_op_destroy(h)
    rc, h = _create(L, **ROT)
    assert _info(L, h).bytes == 2 * 2 * 10 * 8 * 64
    L.load().miriam_op_destroy(h)


# ----------------------------------------------------------------- frequencies
def test_rotary_frequencies():
    from paper_2307_04339_amd import ops
    j = np.arange(32)
    f = 10000.0 ** (-j / 32)
    assert np.allclose(ops.rotary_freqs(64).numpy(), f, rtol=1e-15, atol=0)
    assert np.allclose(ops.rotary_freqs(64, 10000.0, 4.0).numpy(), f / 4, rtol=1e-15, atol=0)
    g = ops.rotary_freqs(64, 10000.0, 8.0, 4096, 1.0, 32.0).numpy()
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(g[turns >= 32], f[turns >= 32], rtol=1e-15) and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.any() and np.allclose(g[mid], f[mid] * keep + f[mid] / 8 * (1 - keep), rtol=1e-14)
    from paper_2307_04339_amd import _lib as L
    for bad in [(0,), (7,), (64, -1.0), (64, math.inf), (64, 1e4, 0.5), (64, 1e4, math.nan), (64, 1e4, 2.0, -1), (64, 1e4, 2.0, 10, 5.0, 5.0),
                (64, 1e4, 2.0, 10, -1.0, 5.0), (64, 1e4, 2.0, 10, 1.0, math.nan)]:
        with pytest.raises(L.MiriamError):
            ops.rotary_freqs(*bad)
    assert L.load().miriam_plan_rotary_freqs(64, 1e4, 1.0, 0, 1.0, 32.0, None) == L.EINVAL


# ------------------------------------------------------------ Python's own checks
def test_tensors_that_do_not_fit_are_refused():
    from paper_2307_04339_amd import ops
    x = torch.zeros(4, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="device memory"):
        ops.block_norm(x, z=torch.zeros(4, 64, dtype=torch.float16), pre=torch.ones(64))
    i = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    c = torch.zeros(2, 1, 16, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="device memory"):
        ops.attention(x, c, c, x.clone(), i(2), i(1), i(1).view(1, 1), heads=1)
    with pytest.raises(ValueError, match="go together"):
        ops.rotary(x, x.clone(), torch.zeros(4, dtype=torch.float64), i(2), i(1), heads=1, head_dim=64, kv_heads=1)
    for name, fn in [
        ("rows", lambda: ops._rows("x", x.t())), ("width", lambda: ops._rows("x", x, 65)), ("count", lambda: ops._rows("x", x, 64, 5)),
        ("type", lambda: ops._rows("x", x, 64, 4, torch.float32)), ("vector", lambda: ops._vector("w", torch.ones(64)[::2], 32, torch.float32)),
        ("starts", lambda: ops._sequences(i(3), i(3), None, None, None, x.dtype)),
        ("lengths", lambda: ops._sequences(i(4).long(), i(3), None, None, None, x.dtype)),
        ("caches", lambda: ops._sequences(i(2), i(1), i(1).view(1, 1), c, c[:1], x.dtype)),
        ("strides", lambda: ops._sequences(i(2), i(1), i(1).view(1, 1), c, c.expand(2, 1, 16, 64).transpose(1, 2).contiguous().transpose(1, 2)[..., ::1], torch.bfloat16)),
        ("values", lambda: ops._sequences(i(2), i(1), i(1).view(1, 1), c.transpose(2, 3), c.transpose(2, 3), x.dtype)),
        ("table", lambda: ops._sequences(i(2), i(1), i(2).view(2, 1), c, c, x.dtype)),
        ("table type", lambda: ops._sequences(i(2), i(1), i(1).view(1, 1).long(), c, c, x.dtype)),
    ]:
        with pytest.raises(ValueError):
            fn()


# ------------------------------------------------------------------- the oracle
def test_broadcast_rows_are_refused():
    """A row stride of 0 means dense rows to the library, and rows closer than their width are none."""
    from paper_2307_04339_amd import ops
    x = torch.zeros(64)
    for t in (x.expand(5, 64), x.as_strided((3, 16), (8, 1))):
        with pytest.raises(ValueError, match="share memory"):
            ops._rows("x", t)
    assert ops._rows("x", x.expand(1, 64)) == 64 and ops._rows("x", x.view(4, 16)[:, :8]) == 16
    c, i = torch.zeros(2, 1, 16, 64), lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="share memory"):
        ops._sequences(i(4), i(3), i(2).expand(3, 2), c, c.clone(), torch.float32)
    assert ops._sequences(i(2), i(1), i(2).expand(1, 2), c, c.clone(), torch.float32)["ldt"] == 2


def test_oracle_attention_against_a_masked_softmax():
    rng = np.random.default_rng(1)
    page, kv, d, heads = 4, 2, 8, 6
    k, v = rng.normal(size=(7, kv, page, d)), rng.normal(size=(7, kv, page, d))
    table = np.array([[3, 1, 6], [0, -1, 2]])
    x = rng.normal(size=(6, heads * d))
    got = seq.attention(x, k, v, [0, 4, 5], [9, 7], table, heads, window=5)
    for r, s, pos, n in [(0, 0, 5, 9), (3, 0, 8, 9), (4, 1, 6, 7)]:
        keys = [j for j in range(n) if pos - 5 < j <= pos and table[s, j // page] >= 0]
        q = torch.tensor(x[r]).view(heads, 1, d)
        kk = torch.tensor(np.stack([k[table[s, j // page], :, j % page] for j in keys])).permute(1, 0, 2).repeat_interleave(3, 0)
        vv = torch.tensor(np.stack([v[table[s, j // page], :, j % page] for j in keys])).permute(1, 0, 2).repeat_interleave(3, 0)
        want = torch.softmax(q @ kk.transpose(1, 2) / math.sqrt(d), -1) @ vv
        assert np.allclose(got[r][0], want.reshape(-1).numpy(), rtol=1e-12, atol=1e-13)
    assert set(got) == {0, 1, 2, 3, 4}


def test_oracle_rotary_is_a_rotation():
    freq = 100.0 ** (-np.arange(4) / 4)
    head = np.random.default_rng(2).normal(size=10)
    for inter in (False, True):
        out, _ = seq.rotate(head, 3, freq, inter, 2.0)
        back, _ = seq.rotate(out, -3, freq, inter, 0.5)
        assert np.allclose(back, head) and np.array_equal(out[8:], head[8:])
        a = (0, 1) if inter else (0, 4)
        w = complex(head[a[0]], head[a[1]]) * 2.0 * np.exp(3j * freq[0])
        assert np.allclose([out[a[0]], out[a[1]]], [w.real, w.imag])


def test_oracle_block_norm_against_torch():
    rng = np.random.default_rng(3)
    x, r, g = (rng.normal(size=(5, 40)) for _ in range(3))
    w, b, w2, b2 = (rng.normal(size=40) for _ in range(4))
    t = lambda a: torch.tensor(a)  # noqa: E731
    y, z, ey, ez = seq.block_norm(x, r, w, b, g, "silu", 0.3, w2, b2, "layer", 1e-5)
    want = t(r) + 0.3 * torch.nn.functional.layer_norm(t(x), (40,), t(w), t(b), 1e-5) * torch.nn.functional.silu(t(g))
    assert np.allclose(y, want.numpy()) and np.allclose(z, torch.nn.functional.layer_norm(want, (40,), t(w2), t(b2), 1e-5).numpy())
    y, z, _, _ = seq.block_norm(x, None, None, None, w, "none", 1.0, w2, None, "rms", 1e-6)
    assert np.allclose(y, x * w) and np.allclose(z, y / np.sqrt((y * y).mean(1, keepdims=True) + 1e-6) * w2)
    # the bounds hold for the same operations in fp32
    y32, z32, _, _ = (None if a is None else a for a in seq.block_norm(x.astype(np.float32), r.astype(np.float32), w.astype(np.float32),
                                                                       None, None, "none", 1.0, w2.astype(np.float32)))
    f = lambda a: a.astype(np.float32).astype(np.float64)  # noqa: E731
    y, z, ey, ez = seq.block_norm(f(x), f(r), f(w), None, None, "none", 1.0, f(w2))
    assert np.all(np.abs(y32 - y) <= ey) and np.all(np.abs(z32 - z) <= ez)
