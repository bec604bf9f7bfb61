"""Host-side checks of rotary positions, the paged bf16 cache and its attention that need no GPU: the table of steps, refusals before
any device work, workspace sizes, struct layouts, and the plain definitions the GPU tests rely on."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import _paged as P
from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NO_GPU = not torch.cuda.is_available()


@pytest.fixture(scope="module")
def lib():
    B.build_libgmlp()
    return gmlp.lib()


def call(entry, a, **kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return entry(ctypes.byref(a))


def changed(make, **kw):
    a = make()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def cache(**kw):
    return changed(lambda: gmlp.GmlpKvCache(0x10000, 0x20000, 10, 2, 64, 128, 0), **kw)


def rope(**kw):
    return changed(lambda: gmlp.GmlpRope(0x8000, 64, 0, 1.0, 0), **kw)


SCALINGS = [None, ("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 8192), ("ramp", 16.0, 32.0, 1.0, 4096), ("ramp", 1.0, 32.0, 1.0, 4096)]


@pytest.mark.parametrize("rot,base", [(4, 1e4), (20, 1e4), (64, 1e4), (128, 5e5), (256, 1e6)])
@pytest.mark.parametrize("scaling", SCALINGS)
def test_steps_are_the_frequencies(lib, rot, base, scaling):
    steps, amplitude = gmlp.rope_steps(rot, base, scaling)
    f, want = P.frequencies(rot, base, scaling)
    assert len(steps) == rot // 2 and amplitude == pytest.approx(want, rel=1e-7)
    for s, v in zip(steps, f):                               # a double's power is good to a few units of 2^-53
        assert 0 <= s < 1 << 64 and abs(s * 2.0 ** -64 - v / (2 * math.pi)) <= 2.0 ** -49 * v + 2.0 ** -64


def test_steps_refusals(lib):
    st, am = (ctypes.c_uint64 * 512)(), ctypes.c_float()
    f = lambda rot, base, s=None: lib.gmlp_rope_steps(rot, base, None if s is None else ctypes.byref(s), st, ctypes.byref(am))
    S = gmlp.GmlpRopeScaling
    for rot in (0, 2, -4, 6, 1028):
        assert f(rot, 1e4) == gmlp.ERR_SHAPE
    for base in (1.0, 0.0, -5.0, float("nan"), float("inf")):
        assert f(64, base) == gmlp.ERR_SHAPE
    assert f(64, 1e4, S(4, 0, 1, 1, 1, 1)) == gmlp.ERR_FLAGS and f(64, 1e4, S(1, 1, 2, 0, 0, 0)) == gmlp.ERR_FLAGS
    for bad in (S(1, 0, 0, 0, 0, 0), S(1, 0, float("nan"), 0, 0, 0), S(2, 0, 2, 4, 1, 100), S(2, 0, 2, 1, 4, 0), S(3, 0, 2, 0, 4, 100),
                S(3, 0, 2, 4, 1, 100), S(3, 0, 2, 1, 4, float("inf"))):
        assert f(64, 1e4, bad) == gmlp.ERR_SHAPE
    assert lib.gmlp_rope_steps(64, 1e4, None, None, ctypes.byref(am)) == gmlp.ERR_NULL
    assert lib.gmlp_rope_steps(64, 1e4, None, st, None) == gmlp.ERR_NULL
    with pytest.raises(ValueError):
        gmlp.rope_steps(64, 1e4, ("linear",))
    with pytest.raises(ValueError):
        gmlp.rope_steps(64, 1e4, ("other", 2.0))


BAD_ROPES = [(dict(rotary_dim=0), gmlp.ERR_SHAPE), (dict(rotary_dim=6), gmlp.ERR_SHAPE), (dict(rotary_dim=132), gmlp.ERR_SHAPE),
             (dict(amplitude=float("inf")), gmlp.ERR_SHAPE), (dict(amplitude=float("nan")), gmlp.ERR_SHAPE), (dict(interleaved=2), gmlp.ERR_FLAGS),
             (dict(reserved=1), gmlp.ERR_FLAGS), (dict(steps=0x8004), gmlp.ERR_ALIGN)]
BAD_CACHES = [(dict(head_dim=96), gmlp.ERR_UNSUPPORTED), (dict(head_dim=256), gmlp.ERR_UNSUPPORTED), (dict(page_size=24), gmlp.ERR_SHAPE),
              (dict(page_size=0), gmlp.ERR_SHAPE), (dict(page_size=8), gmlp.ERR_SHAPE), (dict(n_pages=0), gmlp.ERR_SHAPE), (dict(n_pages=-1), gmlp.ERR_SHAPE),
              (dict(n_pages=1 << 24), gmlp.ERR_SHAPE), (dict(n_pages=1 << 60), gmlp.ERR_SHAPE), (dict(n_kv_heads=0), gmlp.ERR_SHAPE),
              (dict(n_kv_heads=4097), gmlp.ERR_SHAPE), (dict(k=None), gmlp.ERR_NULL), (dict(v=None), gmlp.ERR_NULL), (dict(k=0x10008), gmlp.ERR_ALIGN),
              (dict(v=0x20002), gmlp.ERR_ALIGN), (dict(reserved=1), gmlp.ERR_FLAGS)]


def rope_args():
    return gmlp.GmlpRopeArgs(ctypes.sizeof(gmlp.GmlpRopeArgs), 0, 0x1000, 0x2000, 0x3000, 5, 8, 128, rope(), None)


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=1), gmlp.ERR_FLAGS), (dict(T=-1), gmlp.ERR_SHAPE),
                                       (dict(T=(1 << 24) + 1), gmlp.ERR_SHAPE), (dict(n_heads=0), gmlp.ERR_SHAPE), (dict(n_heads=65536), gmlp.ERR_SHAPE),
                                       (dict(head_dim=4), gmlp.ERR_SHAPE), (dict(head_dim=100), gmlp.ERR_SHAPE), (dict(head_dim=520), gmlp.ERR_SHAPE),
                                       (dict(T=0, X=None, Y=None, positions=None), gmlp.OK), (dict(X=None), gmlp.ERR_NULL), (dict(Y=None), gmlp.ERR_NULL),
                                       (dict(positions=None), gmlp.ERR_NULL), (dict(X=0x1008), gmlp.ERR_ALIGN), (dict(Y=0x2002), gmlp.ERR_ALIGN),
                                       (dict(positions=0x3004), gmlp.ERR_ALIGN), (dict(rope=rope(steps=None)), gmlp.ERR_NULL)] +
                         [(dict(rope=rope(**r)), s) for r, s in BAD_ROPES])
def test_rope_refusals(lib, kw, status):
    assert call(lib.gmlp_rope_apply, rope_args(), **kw) == status
    assert lib.gmlp_rope_apply(None) == gmlp.ERR_NULL


def append_args():
    return gmlp.GmlpKvAppendArgs(ctypes.sizeof(gmlp.GmlpKvAppendArgs), 0, 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 5, 8, 0, cache(), rope(), None)


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=1 << 4), gmlp.ERR_FLAGS), (dict(reserved=1), gmlp.ERR_FLAGS),
                                       (dict(T=-1), gmlp.ERR_SHAPE), (dict(T=(1 << 24) + 1), gmlp.ERR_SHAPE), (dict(n_q_heads=-1), gmlp.ERR_SHAPE),
                                       (dict(n_q_heads=0), gmlp.ERR_SHAPE), (dict(n_q_heads=65536), gmlp.ERR_SHAPE),
                                       (dict(T=0, K=None, V=None, slots=None), gmlp.OK), (dict(K=None), gmlp.ERR_NULL), (dict(V=None), gmlp.ERR_NULL),
                                       (dict(slots=None), gmlp.ERR_NULL), (dict(positions=None), gmlp.ERR_NULL), (dict(Q=None), gmlp.ERR_NULL),
                                       (dict(Qout=None), gmlp.ERR_NULL), (dict(rope=rope(steps=None)), gmlp.ERR_NULL), (dict(Q=0x1008), gmlp.ERR_ALIGN),
                                       (dict(Qout=0x2008), gmlp.ERR_ALIGN), (dict(K=0x3008), gmlp.ERR_ALIGN), (dict(V=0x4008), gmlp.ERR_ALIGN),
                                       (dict(positions=0x5004), gmlp.ERR_ALIGN), (dict(slots=0x6004), gmlp.ERR_ALIGN)] +
                         [(dict(rope=rope(**r)), s) for r, s in BAD_ROPES] + [(dict(cache=cache(**c)), s) for c, s in BAD_CACHES])
def test_append_refusals(lib, kw, status):
    assert call(lib.gmlp_kv_append, append_args(), **kw) == status
    assert lib.gmlp_kv_append(None) == gmlp.ERR_NULL


def attention_args():
    a = gmlp.GmlpKvAttentionArgs()
    a.struct_bytes = ctypes.sizeof(gmlp.GmlpKvAttentionArgs)
    a.Q, a.O, a.block_table, a.lengths, a.q_start = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000
    a.cache = cache()
    a.B, a.T, a.table_width, a.n_q_heads, a.scale = 3, 50, 4, 8, 0.1
    a.workspace, a.workspace_bytes = 0x100000, 1 << 40
    return a


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=1 << 5), gmlp.ERR_FLAGS), (dict(reserved=1), gmlp.ERR_FLAGS),
                                       (dict(scale=float("inf")), gmlp.ERR_FLAGS), (dict(scale=float("nan")), gmlp.ERR_FLAGS), (dict(scale=0.0), gmlp.ERR_FLAGS),
                                       (dict(scale=-0.1), gmlp.ERR_FLAGS), (dict(scale=3e38), gmlp.ERR_FLAGS), (dict(B=-1), gmlp.ERR_SHAPE),
                                       (dict(B=65536), gmlp.ERR_SHAPE), (dict(T=-1), gmlp.ERR_SHAPE), (dict(T=(1 << 24) + 1), gmlp.ERR_SHAPE),
                                       (dict(q_start=None, q_len=0), gmlp.ERR_SHAPE), (dict(q_start=None, q_len=16), gmlp.ERR_SHAPE),
                                       (dict(q_start=None, q_len=1 << 30, B=4, T=0), gmlp.ERR_SHAPE),
                                       (dict(n_q_heads=7), gmlp.ERR_SHAPE), (dict(n_q_heads=0), gmlp.ERR_SHAPE), (dict(n_q_heads=258), gmlp.ERR_UNSUPPORTED),
                                       (dict(table_width=0), gmlp.ERR_SHAPE), (dict(table_width=1 << 40), gmlp.ERR_SHAPE),
                                       (dict(table_width=(1 << 24) + 1), gmlp.ERR_SHAPE), (dict(B=0, Q=None, O=None), gmlp.OK),
                                       (dict(T=0, Q=None, O=None), gmlp.OK), (dict(Q=None), gmlp.ERR_NULL), (dict(O=None), gmlp.ERR_NULL),
                                       (dict(lengths=None), gmlp.ERR_NULL), (dict(block_table=None), gmlp.ERR_NULL), (dict(Q=0x1008), gmlp.ERR_ALIGN),
                                       (dict(O=0x2008), gmlp.ERR_ALIGN), (dict(block_table=0x3002), gmlp.ERR_ALIGN), (dict(lengths=0x4002), gmlp.ERR_ALIGN),
                                       (dict(q_start=0x5002), gmlp.ERR_ALIGN), (dict(workspace=0x100010), gmlp.ERR_ALIGN)] +
                         [(dict(cache=cache(**c)), s) for c, s in BAD_CACHES])
def test_attention_refusals(lib, kw, status):
    assert call(lib.gmlp_kv_attention, attention_args(), **kw) == status
    assert lib.gmlp_kv_attention(None) == gmlp.ERR_NULL


@pytest.mark.skipif(not NO_GPU, reason="checks the no-device behaviour")
def test_no_device_means_arch_error(lib):
    assert call(lib.gmlp_rope_apply, rope_args()) == gmlp.ERR_ARCH
    assert call(lib.gmlp_kv_append, append_args()) == gmlp.ERR_ARCH
    assert call(lib.gmlp_kv_append, append_args(), Q=None, Qout=None, n_q_heads=0, rope=rope(steps=None), positions=None) == gmlp.ERR_ARCH
    assert call(lib.gmlp_kv_attention, attention_args()) == gmlp.ERR_ARCH
    assert call(lib.gmlp_kv_attention, attention_args(), q_start=None, q_len=10, B=5) == gmlp.ERR_ARCH


def test_binding_refuses_host_tensors(lib):
    with pytest.raises(TypeError):
        gmlp.Rope(64, device="cpu")
    with pytest.raises(TypeError):
        gmlp.kv_cache(2, 2, device="cpu")
    with pytest.raises(ValueError):
        gmlp.KvCache(torch.zeros(2, 2, 16), torch.zeros(1))
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.Rope(30)
    assert e.value.status == gmlp.ERR_SHAPE


def test_struct_layouts_match_the_header(lib, tmp_path):
    names = dict(gmlp_rope_scaling=gmlp.GmlpRopeScaling, gmlp_rope=gmlp.GmlpRope, gmlp_rope_args=gmlp.GmlpRopeArgs, gmlp_kv_cache=gmlp.GmlpKvCache,
                 gmlp_kv_append_args=gmlp.GmlpKvAppendArgs, gmlp_kv_attention_args=gmlp.GmlpKvAttentionArgs)
    lines = []
    for c, py in names.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f[0]} %zu\\n", offsetof({c}, {f[0]}));' for f in py._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gmlp.h"\nint main(void) {' + "\n".join(lines) +
                   f"return (int)GMLP_KV_CAUSAL - {gmlp.KV_CAUSAL} + GMLP_ROPE_LINEAR - 1 + GMLP_ROPE_BANDS - 2 + GMLP_ROPE_RAMP - 3;" + "}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for c, py in names.items():
        assert int(got[c]) == ctypes.sizeof(py)
        for f in py._fields_:
            assert int(got[f"{c}.{f[0]}"]) == getattr(py, f[0]).offset
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gmlp.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(gmlp_(?:rope|kv)_[a-z_0-9]+)\s*\(", text))
    assert declared == {"gmlp_rope_steps", "gmlp_rope_apply", "gmlp_kv_append", "gmlp_kv_attention", "gmlp_kv_workspace_bytes"}
    assert all(hasattr(lib, n) for n in declared)


def test_plain_rotation_keeps_lengths_and_differences():
    g = torch.Generator().manual_seed(1)
    x, y = torch.randn(1, 1, 64, generator=g).double(), torch.randn(1, 1, 64, generator=g).double()
    for inter in (False, True):
        f, a = P.frequencies(32, 1e4)
        turn = lambda t, p: P.rotate(t, torch.tensor([p]), f, a, 32, inter)
        assert float((turn(x, 900).norm() - x.norm()).abs()) < 1e-12
        assert float((turn(x, 900) * turn(y, 893)).sum() - (turn(x, 7) * turn(y, 0)).sum()) == pytest.approx(0, abs=1e-11)
        assert torch.equal(turn(x, 900)[..., 32:], x[..., 32:])
        assert float((turn(turn(x, 900), -900) - x).abs().max()) < 1e-12


def test_plain_attention_of_hidden_rows():
    g = torch.Generator().manual_seed(2)
    Q, k, v = torch.randn(5, 4 * 64, generator=g), torch.randn(3, 2, 64, generator=g), torch.randn(3, 2, 64, generator=g)
    O, _, _ = P.attention(Q, k, v, 4, 0.125)
    assert bool((O[:2] == 0).all()) and torch.allclose(O[2].view(2, 2, 64), v[:1].double().transpose(0, 1).expand(2, 2, 64))
    full, _, _ = P.attention(Q, k, v, 4, 0.125, causal=False)
    assert torch.allclose(full[4], O[4])
