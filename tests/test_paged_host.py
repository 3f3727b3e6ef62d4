"""Rotary positions and the paged cache without a GPU: the oracle's pins, the
work arithmetic of the attention (tests/native/paged_plan_check.cpp), and the
refusals of the C ABI and the binding.  No kernel is launched."""
import ctypes
import math
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import paper_2404_00456_amd as q
from paged_cases import Batch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2404_00456_amd", "csrc")
OK, INVALID, UNSUPPORTED, ALIGN, WORKSPACE, NODEV, HIP = range(7)
P, P4, U = 1 << 20, (1 << 20) + 4, (1 << 20) + 2  # fake, never dereferenced


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_work_arithmetic():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "check")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-I", CSRC,
                        os.path.join(ROOT, "tests", "native", "paged_plan_check.cpp"), "-o", exe],
                       check=True, capture_output=True)
        res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
        assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr


# ---------------------------------------------------------------- oracle ----

def test_cos_sin_round_once(orc):
    """Against the C library's binary64 functions, whose error (below 1 ulp of
    binary64) moves the binary32 rounding of one angle in 2^28: none of these."""
    rng = np.random.default_rng(0)
    angles = np.concatenate([rng.uniform(-2.0 ** 31, 2.0 ** 31, 30000), rng.uniform(-7, 7, 30000),
                             np.arange(-50, 50) * math.pi / 4, [0.0, 2.0 ** 31, 1e-300]])
    for a in angles:
        c, s = orc.cos_sin(a)
        assert c == np.float32(math.cos(a)) and s == np.float32(math.sin(a)), a


def test_rope_is_a_rotation(orc):
    """Norms of pairs stay, equal shifts of a query and a key leave their
    product, and position 0 changes nothing."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 64)).astype(np.float16)
    fr = (1e4 ** (-np.arange(16) / 16)).astype(np.float32)
    axis = np.arange(16, dtype=np.uint8) % 2
    assert np.array_equal(orc.rope(x, np.zeros((2, 2), np.int32), fr, axis), x.astype(np.float32))
    dots = []
    for shift in (0, 5, 1 << 20):
        for inter in (False, True):
            y = orc.rope(x, np.array([[7, 3], [2, 9]]) + shift, fr, axis, inter).astype(np.float64)
            dots.append(((y[0] * y[1])[:, 32:].sum(-1), y))
            a, b = (y[..., 0:32:2], y[..., 1:32:2]) if inter else (y[..., :16], y[..., 16:32])
            u, v = (x[..., 0:32:2], x[..., 1:32:2]) if inter else (x[..., :16], x[..., 16:32])
            u, v = u.astype(np.float64), v.astype(np.float64)
            # two products and a sum, each half a step of binary32
            assert np.abs(np.hypot(a, b) - np.hypot(u, v)).max() <= 4 * 2.0 ** -24 * np.hypot(u, v).max()
            assert np.array_equal(y[..., 32:], x[..., 32:].astype(np.float64))
    for i in (0, 1):
        full = [(y[0] * y[1]).sum(-1) for _, y in dots[i::2]]
        for f in full[1:]:
            assert np.abs(f - full[0]).max() <= 64 * 16 * 2.0 ** -23


def test_paged_attention_is_dense_attention(orc):
    """Against the oracle of the dense cache for a single new token, and against
    softmax over explicit masks for chunks with a window."""
    bt = Batch(0, [1], [50], 2, 64, 32, 16)
    qh = bt.queries(4)
    got = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, 32)
    dense = [tuple(np.ascontiguousarray(c[bt.table[0]].swapaxes(0, 1).reshape(2, 64, -1)) for c in p)
             for p in (bt.k, bt.v)]
    ref = orc.kv_attention(qh[0], *dense, 50, 32)
    # the dense oracle takes sm_scale as binary32 and rounds its output to fp16
    assert np.abs(got[0] - ref.astype(np.float64)).max() <= 2.0 ** -11 * np.abs(ref).max() + 1e-6
    bt = Batch(1, [30, 0, 9], [60, 5, 9], 2, 64, 64, 32, behind=2)
    qh = bt.queries(6)
    for window, sinks in ((0, 0), (7, 3)):
        out = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, 64, window, sinks,
                                  out=np.full(qh.shape, 2.0))
        assert (out[39:] == 2.0).all()
        for b in (0, 2):
            n, total = bt.new[b], bt.total[b]
            k, v = (bt.values(p)[bt.table[b, :-(-total // 32)]].swapaxes(0, 1).reshape(2, -1, 64)[:, :total]
                    for p in (bt.k, bt.v))
            p, t = np.arange(total - n, total)[:, None], np.arange(total)[None]
            see = (t <= p) & ((window == 0) | (t > p - window) | (t < sinks))
            for h in range(6):
                s = qh[bt.cu[b]:bt.cu[b + 1], h].astype(np.float64) @ k[h // 3].T / 8.0
                s = np.where(see, s, -np.inf)
                w = np.exp(s - s.max(-1, keepdims=True))
                ref = w @ v[h // 3] / w.sum(-1, keepdims=True)
                assert np.abs(out[bt.cu[b]:bt.cu[b + 1], h] - ref).max() < 1e-12


# -------------------------------------------------------------- refusals ----

def cache(**kw):
    c = dict(k_codes=P, k_scale=P, k_zero=P, v_codes=P, v_scale=P, v_zero=P, page_table=P4,
             seq_lens=P4, cu_new=P4, batch=2, n_kv_heads=2, head_dim=128, group=128, n_pages=9,
             page_size=16, max_pages=4)
    c.update(kw)
    return ctypes.byref(q._PagedKV(**c))


AXES = (ctypes.c_uint8 * 64)(*([0] * 32 + [1] * 32))


def rotary(**kw):
    r = dict(positions=P4, pos_stride=8, inv_freq=P4, axis_map=None, n_axes=1, rot_dim=128,
             interleaved=0)
    r.update(kw)
    return ctypes.byref(q._Rotary(**r))


def has_gpu():
    return torch.cuda.device_count() > 0


def last(st):
    """What a call with valid arguments gives: no device here (with one, these
    calls are not made: the pointers are fake)."""
    assert st == NODEV


def test_rope_refusals():
    f = q.lib().quarot_rope
    S = None
    good = (P, 512, P, 512, rotary(), 8, 4, 128, 1)
    if not has_gpu():
        last(f(*good, S))
        last(f(P, 512, P, 512, rotary(axis_map=ctypes.cast(AXES, ctypes.c_void_p), n_axes=2), 8, 4, 128, 0, S))

    def g(i, v):
        a = list(good)
        a[i] = v
        return f(*a, S)

    assert g(5, 0) == OK
    assert g(5, -1) == INVALID and g(6, 0) == INVALID and g(7, 0) == INVALID
    assert g(7, 96) == UNSUPPORTED and g(7, 512) == UNSUPPORTED and g(6, 1 << 20) == UNSUPPORTED
    assert g(5, 9) == INVALID and g(5, 1 << 40) == UNSUPPORTED  # pos_stride; tokens
    assert f(P, 512, P, 512, rotary(pos_stride=1 << 28), 1 << 28, 4, 128, 1, S) == UNSUPPORTED
    assert g(0, None) == INVALID and g(2, None) == INVALID
    assert g(0, P4) == ALIGN and g(2, P4) == ALIGN
    assert g(1, 504) == INVALID and g(3, 504) == INVALID  # stride below a token
    assert g(1, 516) == ALIGN and g(1, 1 << 40) == UNSUPPORTED
    assert f(P, 512, P, 520, rotary(), 8, 4, 128, 1, S) == INVALID  # in place, other stride
    assert g(4, None) == INVALID
    for bad, st in ((dict(inv_freq=None), INVALID), (dict(positions=None), INVALID),
                    (dict(n_axes=0), INVALID), (dict(n_axes=5), UNSUPPORTED),
                    (dict(rot_dim=0), INVALID), (dict(rot_dim=8), UNSUPPORTED),
                    (dict(rot_dim=144), UNSUPPORTED), (dict(pos_stride=7), INVALID),
                    (dict(pos_stride=1 << 40), UNSUPPORTED),
                    (dict(positions=U), ALIGN), (dict(inv_freq=U), ALIGN),
                    (dict(axis_map=ctypes.cast(AXES, ctypes.c_void_p)), INVALID)):  # axis 1 of 1
        assert g(4, rotary(**bad)) == st, bad


BAD_CACHES = [(dict(batch=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
              (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED),
              (dict(group=0), INVALID), (dict(group=16), UNSUPPORTED),
              (dict(group=256), UNSUPPORTED), (dict(group=96), UNSUPPORTED),
              (dict(n_pages=0), INVALID), (dict(n_pages=1 << 31), UNSUPPORTED),
              (dict(page_size=0), INVALID), (dict(page_size=24), UNSUPPORTED),
              (dict(page_size=8), UNSUPPORTED), (dict(page_size=1 << 31), UNSUPPORTED),
              (dict(max_pages=0), INVALID), (dict(max_pages=(1 << 26) + 1), UNSUPPORTED),
              (dict(batch=1 << 24), UNSUPPORTED)]
BAD_CACHES += [({n: None}, INVALID) for n in ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale",
                                              "v_zero", "page_table", "seq_lens", "cu_new")]
BAD_CACHES += [({n: P4}, ALIGN) for n in ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale",
                                          "v_zero")]
BAD_CACHES += [({n: U}, ALIGN) for n in ("page_table", "seq_lens", "cu_new")]


def test_append_refusals():
    f = q.lib().quarot_kv_append_paged
    good = [P, 1024, P, 1024, P, 256, P, 256, cache(), rotary(), 8, 8, 1, 0, 0.95, None]

    def g(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)

    if not has_gpu():
        last(g())
        last(g(_9=None))
        last(g(_9=rotary(positions=None)))
        last(g(_0=None, _2=None, _11=0))
    assert g(_10=0) == OK and g(_10=-1) == INVALID
    assert g(_8=None) == INVALID
    for bad, st in BAD_CACHES:
        assert g(_8=cache(**bad)) == st, bad
    assert g(_14=0.0) == INVALID and g(_14=1.5) == INVALID and g(_14=float("nan")) == INVALID
    assert g(_0=None) == INVALID and g(_2=None) == INVALID and g(_11=0) == INVALID
    assert g(_4=None) == INVALID and g(_6=None) == INVALID and g(_11=-1) == INVALID
    assert g(_0=P4) == ALIGN and g(_4=P4) == ALIGN and g(_6=P4) == ALIGN
    assert g(_1=1016) == INVALID and g(_5=248) == INVALID and g(_7=260) == ALIGN
    assert g(_1=1032) == INVALID  # in place, other stride
    assert g(_9=rotary(positions=None, n_axes=2)) == INVALID
    assert g(_9=rotary(rot_dim=160)) == UNSUPPORTED


def test_attention_refusals():
    f = q.lib().quarot_kv_paged_attention
    good = [P, 1024, P, 1024, cache(), 8, 8, 64, 0, 0, 0.1, P, 1 << 30, None]

    def g(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)

    if not has_gpu():
        last(g())
    assert g(_5=0) == OK and g(_5=-1) == INVALID
    assert g(_4=None) == INVALID
    for bad, st in BAD_CACHES:
        assert g(_4=cache(**bad)) == st, bad
    assert g(_6=0) == INVALID and g(_6=7) == INVALID and g(_6=1 << 20) == UNSUPPORTED
    assert g(_5=1 << 28) == UNSUPPORTED  # T * n_heads
    assert g(_7=0) == INVALID and g(_8=-1) == INVALID and g(_9=-1) == INVALID
    assert g(_10=0.0) == INVALID and g(_10=float("inf")) == INVALID and g(_10=float("nan")) == INVALID
    assert g(_0=None) == INVALID and g(_2=None) == INVALID
    assert g(_0=P4) == ALIGN and g(_2=P4) == ALIGN and g(_1=1016) == INVALID and g(_3=1028) == ALIGN
    need = q.quarot_kv_paged_attention_workspace_size(8, 2, 8, 2, 128, 30000)
    assert need > 0
    long = dict(_7=30000)
    assert g(_11=None, **long) == WORKSPACE and g(_12=need - 1, **long) == WORKSPACE
    assert g(_11=P4, **long) == ALIGN
    if not has_gpu():
        last(g(_12=need, **long))


def test_workspace_size_of_bad_sizes():
    f = q.quarot_kv_paged_attention_workspace_size
    good = (8, 2, 8, 2, 128, 30000, 0, 0)
    assert f(*good) > 0
    assert f(8, 2, 8, 2, 128, 30000, group=0) == 0
    for i, bad in ((0, 0), (0, -3), (0, 1 << 62), (1, 0), (1, 1 << 62), (2, 0), (2, 7), (2, 1 << 62),
                   (3, 0), (4, 96), (5, 0), (6, -1), (7, -1)):
        a = list(good)
        a[i] = bad
        assert f(*a) == 0, (i, bad)
    assert f(8, 2, 8, 2, 128, 1 << 62, 1 << 62, 1 << 62) > 0
    assert f(1 << 30, 1, 65535, 1, 128, 1 << 62) >= 0


@pytest.mark.parametrize("T,batch,n_heads,n_kv_heads,D,group,most", [
    (8, 2, 8, 2, 128, g, 30000) for g in (1, 16, 31, 32, 48, 64, 96, 128, 256, 1 << 40)] + [
    (8, 2, 8, 2, 64, 128, 30000), (8, 2, 8, 2, 256, 256, 30000),
    (1 << 27, 2, 8, 2, 128, 128, 64), ((1 << 27) + 1, 2, 8, 2, 128, 128, 64),  # T * n_heads
    (1, 0xFFFFFF, 64, 64, 128, 128, 64), (1, 0xFFFFFF, 1, 1, 128, 128, 64),  # blocks
    (64, 64, 65535, 65535, 128, 128, 64), (1, 1, 65535, 65535, 128, 128, 1 << 20)])
def test_workspace_size_and_call_agree(T, batch, n_heads, n_kv_heads, D, group, most):
    """The query answers 0 for what the call refuses, and what the call needs for
    the rest."""
    size = q.quarot_kv_paged_attention_workspace_size(T, batch, n_heads, n_kv_heads, D, most, group=group)

    def call(bytes_):
        c = cache(batch=batch, n_kv_heads=n_kv_heads, head_dim=D, group=group)
        return q.lib().quarot_kv_paged_attention(P, n_heads * D, P, n_heads * D, c, T, n_heads, most, 0,
                                                 0, 0.1, P if bytes_ else None, bytes_, None)
    if size:
        assert call(0) == call(size - 1) == WORKSPACE
    if has_gpu():  # (the pointers are fake)
        return
    st = call(size)
    assert st == NODEV or (st in (INVALID, UNSUPPORTED) and size == 0)


def test_injected_error(monkeypatch):
    L = q.lib()
    for name, call in (
            ("quarot_rope", lambda: L.quarot_rope(P, 512, P, 512, rotary(), 8, 4, 128, 1, None)),
            ("quarot_kv_append_paged", lambda: L.quarot_kv_append_paged(
                P, 1024, P, 1024, P, 256, P, 256, cache(), None, 8, 8, 1, 0, 0.95, None)),
            ("quarot_kv_paged_attention", lambda: L.quarot_kv_paged_attention(
                P, 1024, P, 1024, cache(), 8, 8, 64, 0, 0, 0.1, P, 1 << 30, None))):
        monkeypatch.setenv("QUAROT_FAKE_HIP_ERROR", name)
        assert call() == HIP and L.quarot_last_hip_error() == 719


# --------------------------------------------------------------- binding ----

def f16(*s):
    return torch.zeros(s, dtype=torch.float16)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def pool(pages=5, heads=2, page=16, D=128, G=128):
    return (torch.zeros((pages, heads, page, D // 2), dtype=torch.uint8), f16(pages, heads, page, D // G),
            f16(pages, heads, page, D // G))


def app(k=None, v=None, kc=None, vc=None, table=None, lens=None, cu=None, **kw):
    return q.quarot_kv_append_paged(
        f16(8, 2, 128) if k is None else k, f16(8, 2, 128) if v is None else v, kc or pool(),
        vc or pool(), i32(3, 4) if table is None else table, i32(3) if lens is None else lens,
        i32(4) if cu is None else cu, **kw)


def att(x=None, kc=None, vc=None, table=None, lens=None, cu=None, **kw):
    return q.quarot_kv_paged_attention(
        f16(8, 4, 128) if x is None else x, kc or pool(), vc or pool(),
        i32(3, 4) if table is None else table, i32(3) if lens is None else lens,
        i32(4) if cu is None else cu, **kw)


FREQ = torch.zeros(64)
SHAPES = {
    "rope y": lambda: q.quarot_rope(f16(4, 2, 128), i32(4), FREQ, y=f16(4, 2, 64)),
    "rope 2-D": lambda: q.quarot_rope(f16(4, 128), i32(4), FREQ),
    "rope positions": lambda: q.quarot_rope(f16(4, 2, 128), i32(3), FREQ),
    "rope axes": lambda: q.quarot_rope(f16(4, 2, 128), i32(2, 4), FREQ, sections=[10, 10, 44]),
    "rope sections": lambda: q.quarot_rope(f16(4, 2, 128), i32(2, 4), FREQ, sections=[10, 53]),
    "rope negative section": lambda: q.quarot_rope(f16(4, 2, 128), i32(2, 4), FREQ, sections=[-1, 65]),
    "rope five sections": lambda: q.quarot_rope(f16(4, 2, 128), i32(5, 4), FREQ, sections=[12, 13, 13, 13, 13]),
    "rope width": lambda: q.quarot_rope(f16(4, 2, 64), i32(4), FREQ),
    "append v": lambda: app(v=f16(8, 1, 128)),
    "append heads": lambda: app(k=f16(8, 4, 128), v=f16(8, 4, 128)),
    "append width": lambda: app(k=f16(8, 2, 64), v=f16(8, 2, 64)),
    "append codes": lambda: app(vc=pool(pages=4)),
    "append scale": lambda: app(kc=(pool()[0], f16(5, 2, 16, 2), pool()[2])),
    "append group": lambda: app(group=96),
    "append table": lambda: app(table=i32(12)),
    "append lens": lambda: app(lens=i32(4)),
    "append cu": lambda: app(cu=i32(3)),
    "append q": lambda: app(q=f16(7, 4, 128)),
    "append q_out": lambda: app(q=f16(8, 4, 128), q_out=f16(8, 3, 128)),
    "append q_out alone": lambda: app(q_out=f16(8, 3, 128)),
    "append positions alone": lambda: app(positions=i32(8)),
    "attention width": lambda: att(x=f16(8, 4, 64)),
    "attention out": lambda: att(out=f16(8, 4, 64)),
    "attention cu": lambda: att(cu=i32(3)),
    "attention codes": lambda: att(vc=pool(page=32)),
}
SAYS = ("must have shape|must hold|must be [0-9]-D|must be a positive divisor|sections must|"
        "without q|need inv_freq")


@pytest.mark.parametrize("case", sorted(SHAPES))
def test_binding_refuses_before_launch(case):
    with pytest.raises(ValueError, match=SAYS):
        SHAPES[case]()


def test_binding_refuses_host_tensors():
    for call in (app, att, lambda: q.quarot_rope(f16(4, 2, 128), i32(4), FREQ)):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()


def test_binding_refuses_types():
    with pytest.raises(TypeError):
        q.quarot_rope(torch.zeros(4, 2, 128), i32(4), FREQ)
    with pytest.raises(TypeError):
        q.quarot_rope(f16(4, 2, 128), torch.zeros(4, dtype=torch.int64), FREQ)


def test_host_code_under_asan_ubsan():
    """The entry points' host code under both sanitizers, with no device, against
    counting stand-ins of the launchers (tests/native/paged_abi_check.cpp)."""
    import test_sanitizers as ts
    if not os.path.exists(ts.HIPCC) or ts.clang_asan_runtime() is None:
        pytest.skip("needs hipcc and clang's ASan runtime")
    csrc, native = (os.path.join(ROOT, *p) for p in (("paper_2404_00456_amd", "csrc"),
                                                     ("tests", "native")))
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host",
           "-fno-omit-frame-pointer"]
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "paged_abi_check")
        subprocess.run([ts.HIPCC, "-O1", "-g", "-std=c++17", *san, "-I", os.path.join(ROOT, "include"),
                        *(os.path.join(csrc, f) for f in ("capi.cpp", "capi_paged.cpp",
                                                          "host_rules.cpp")),
                        *(os.path.join(native, f) for f in ("launch_stubs.cpp",
                                                            "paged_abi_check.cpp")), "-o", exe],
                       check=True, capture_output=True, timeout=600)
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
                   HIP_VISIBLE_DEVICES="-1")
        res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
        assert res.returncode == 0 and res.stdout.strip().endswith("ok"), \
            res.stdout[-3000:] + res.stderr[-3000:]
