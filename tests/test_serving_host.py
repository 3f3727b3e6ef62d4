"""Scored attention, the cache's pages and the sampling without a GPU: the refusals of the
C ABI and of the binding, the host code under the sanitizers, and the arithmetic of a
scored block's steps.  No kernel is launched."""
import ctypes
import os
import shutil
import subprocess
import tempfile

import pytest
import torch

import paper_2404_00456_amd as q
from test_paged_host import (ALIGN, BAD_CACHES, CSRC, HIP, INVALID, NODEV, OK, P, P4, ROOT, U, UNSUPPORTED,
                             WORKSPACE, cache, f16, has_gpu, i32, last, pool)


def changed(f, good):
    def g(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    return g


def scoring(cap=0.0, slopes=None, begin=None, end=None):
    return ctypes.byref(q._Scoring(cap, slopes, begin, end))


def test_scored_refusals():
    g = changed(q.lib().quarot_kv_paged_attention_scored,
                [P, 1024, P, 1024, cache(), scoring(30.0, P4, P4, P4), 8, 8, 64, 0, 0, 0.1, P, 1 << 30, None])
    if not has_gpu():
        last(g())
        for s in (scoring(), scoring(1e-19), scoring(1e19), scoring(0.0, P4), scoring(0.0, None, P4),
                  scoring(0.0, None, None, P4)):
            last(g(_5=s))
    assert g(_5=None) == INVALID
    for cap in (-1.0, float("nan"), float("inf"), -float("inf")):
        assert g(_5=scoring(cap)) == INVALID
    for cap in (1e-30, 1e-40, 1e30):
        assert g(_5=scoring(cap)) == UNSUPPORTED
    for s in (scoring(0.0, U), scoring(0.0, None, U), scoring(0.0, None, None, U)):
        assert g(_5=s) == ALIGN
    # and all that the plain call refuses
    assert g(_6=0) == OK and g(_6=-1) == INVALID and g(_4=None) == INVALID
    for bad, st in BAD_CACHES:
        assert g(_4=cache(**bad)) == st, bad
    assert g(_7=0) == INVALID and g(_7=7) == INVALID and g(_7=1 << 20) == UNSUPPORTED
    assert g(_6=1 << 28) == UNSUPPORTED
    assert g(_8=0) == INVALID and g(_9=-1) == INVALID and g(_10=-1) == INVALID
    assert g(_11=0.0) == INVALID and g(_11=float("nan")) == INVALID
    assert g(_0=None) == INVALID and g(_2=None) == INVALID and g(_0=P4) == ALIGN
    need = q.quarot_kv_paged_attention_workspace_size(8, 2, 8, 2, 128, 30000)
    assert g(_8=30000, _12=None) == WORKSPACE and g(_8=30000, _13=need - 1) == WORKSPACE
    if not has_gpu():
        last(g(_8=30000, _13=need))


def table_refusals(g, B, P_, n):
    """What every call on a table says of its sizes, at argument numbers B, P_ and n."""
    for i in (B, P_, n):
        assert g(**{f"_{i}": 0}) == INVALID and g(**{f"_{i}": -1}) == INVALID
        assert g(**{f"_{i}": 1 << 62}) == UNSUPPORTED
    assert g(**{f"_{B}": 16385}) == UNSUPPORTED and g(**{f"_{n}": (1 << 30) + 1}) == UNSUPPORTED


def test_pages_refusals():
    L = q.lib()
    ws = L.quarot_kv_pages_workspace_size(100)
    assert ws == 1600 and L.quarot_kv_pages_workspace_size(1 << 30) == 1 << 34
    for n in (0, -1, (1 << 30) + 1, -(1 << 62), 1 << 62):
        assert L.quarot_kv_pages_workspace_size(n) == 0
    f = changed(L.quarot_kv_pages_fork, [P4, P4, P4, P4, 8, 10, 100, None])
    r = changed(L.quarot_kv_pages_reserve, [P4] * 8 + [8, 10, 100, 64, P, ws, None])
    c = changed(L.quarot_kv_pages_compact, [P4] * 5 + [8, 10, 100, P, ws, None])
    if not has_gpu():
        last(f())
        last(f(_4=16384))
        last(r())
        last(c())
        last(c(_2=None, _3=None, _7=1))
    for g, ints, at in ((f, 4, 4), (r, 8, 8), (c, 5, 5)):
        table_refusals(g, at, at + 1, at + 2)
        for i in range(ints):
            assert g(**{f"_{i}": None}) == INVALID and g(**{f"_{i}": U}) == ALIGN, i
    for g, w in ((r, 12), (c, 8)):
        assert g(**{f"_{w}": None}) == WORKSPACE and g(**{f"_{w + 1}": ws - 1}) == WORKSPACE
        assert g(**{f"_{w}": P4}) == ALIGN
    for size, st in ((0, INVALID), (-16, INVALID), (24, UNSUPPORTED), (8, UNSUPPORTED), (1 << 31, UNSUPPORTED)):
        assert r(_11=size) == st
    assert r(_9=1 << 25, _11=64) == UNSUPPORTED  # positions of a row


def test_copy_refusals():
    g = changed(q.lib().quarot_kv_pages_copy, [cache(), P4, P4, 5, None])
    if not has_gpu():
        last(g())
        last(g(_0=cache(page_table=None, seq_lens=None, cu_new=None, batch=0, max_pages=0)))
    assert g(_3=0) == OK and g(_3=-1) == INVALID and g(_3=(1 << 30) + 1) == UNSUPPORTED
    assert g(_0=None) == INVALID
    assert g(_1=None) == INVALID and g(_2=None) == INVALID and g(_1=U) == ALIGN and g(_2=U) == ALIGN
    for bad, st in BAD_CACHES:
        if set(bad) & {"page_table", "seq_lens", "cu_new", "batch", "max_pages"}:
            continue  # not read
        assert g(_0=cache(**bad)) == st, bad


def test_sample_refusals():
    g = changed(q.lib().quarot_sample, [P4, 1000, 1, P4, P4, P4, P4, P4, P4, 8, 1000, None])
    if not has_gpu():
        last(g())
        last(g(_4=None, _5=None, _6=None, _7=None))
        last(g(_0=U, _2=0))
        last(g(_9=1, _1=0))  # one row has no stride
    assert g(_9=0) == OK and g(_9=-1) == INVALID and g(_9=1 << 40) == UNSUPPORTED
    assert g(_10=0) == INVALID and g(_10=-5) == INVALID
    assert g(_10=(1 << 20) + 1, _1=1 << 21) == UNSUPPORTED
    assert g(_1=999) == INVALID and g(_1=(1 << 32) + 1) == UNSUPPORTED
    for i in (0, 3, 8):
        assert g(**{f"_{i}": None}) == INVALID
    for i in (3, 4, 5, 6, 7, 8):
        assert g(**{f"_{i}": U}) == ALIGN
    assert g(_0=U) == ALIGN and g(_0=(1 << 20) + 1, _2=0) == ALIGN


def test_injected_errors(monkeypatch):
    L = q.lib()
    for name, call in (
            ("quarot_kv_paged_attention_scored", lambda: L.quarot_kv_paged_attention_scored(
                P, 1024, P, 1024, cache(), scoring(3.0), 8, 8, 64, 0, 0, 0.1, P, 1 << 30, None)),
            ("quarot_kv_paged_attention_scored", lambda: L.quarot_kv_paged_attention_scored(
                P, 1024, P, 1024, cache(), scoring(), 8, 8, 64, 0, 0, 0.1, P, 1 << 30, None)),
            ("quarot_kv_pages_fork", lambda: L.quarot_kv_pages_fork(P4, P4, P4, P4, 8, 10, 100, None)),
            ("quarot_kv_pages_reserve", lambda: L.quarot_kv_pages_reserve(
                *[P4] * 8, 8, 10, 100, 64, P, 1600, None)),
            ("quarot_kv_pages_compact", lambda: L.quarot_kv_pages_compact(*[P4] * 5, 8, 10, 100, P, 1600, None)),
            ("quarot_kv_pages_copy", lambda: L.quarot_kv_pages_copy(cache(), P4, P4, 5, None)),
            ("quarot_sample", lambda: L.quarot_sample(P4, 9, 1, P4, None, None, None, None, P4, 2, 9, None))):
        monkeypatch.setenv("QUAROT_FAKE_HIP_ERROR", name)
        assert call() == HIP and L.quarot_last_hip_error() == 719


# --------------------------------------------------------------- binding ----

def att(x=None, **kw):
    return q.quarot_kv_paged_attention_scored(f16(8, 4, 128) if x is None else x, pool(), pool(), i32(3, 4),
                                              i32(3), i32(4), **kw)


def res(table=None, lens=None, refs=None, new=None, **kw):
    return q.quarot_kv_pages_reserve(i32(3, 4) if table is None else table, i32(3) if lens is None else lens,
                                     i32(9) if refs is None else refs, i32(3) if new is None else new, 16, **kw)


def smp(x=None, u=None, **kw):
    return q.quarot_sample(f16(5, 100) if x is None else x, torch.zeros(5) if u is None else u, **kw)


SHAPES = {
    "slopes": lambda: att(slopes=torch.zeros(3)),
    "begin": lambda: att(begin=i32(7)),
    "end": lambda: att(end=i32(8, 1)),
    "attention out": lambda: att(out=f16(8, 4, 64)),
    "fork parent": lambda: q.quarot_kv_pages_fork(i32(3, 4), i32(3), i32(9), i32(4)),
    "fork lens": lambda: q.quarot_kv_pages_fork(i32(3, 4), i32(4), i32(9), i32(3)),
    "fork table": lambda: q.quarot_kv_pages_fork(i32(12), i32(3), i32(9), i32(3)),
    "reserve new": lambda: res(new=i32(4)),
    "reserve lens": lambda: res(lens=i32(2)),
    "reserve refs": lambda: res(refs=i32(3, 3)),
    "reserve cu": lambda: res(cu_new=i32(3)),
    "reserve src": lambda: res(copy_src=i32(4)),
    "reserve missing": lambda: res(missing=i32(2)),
    "compact src": lambda: q.quarot_kv_pages_compact(i32(3, 4), i32(9), move_src=i32(5)),
    "compact live": lambda: q.quarot_kv_pages_compact(i32(3, 4), i32(9), n_live=i32(0)),
    "copy codes": lambda: q.quarot_kv_pages_copy(pool(), pool(pages=4), i32(2), i32(2)),
    "copy scale": lambda: q.quarot_kv_pages_copy((pool()[0], f16(5, 2, 16, 2), pool()[2]), pool(), i32(2), i32(2)),
    "copy groups": lambda: q.quarot_kv_pages_copy((pool()[0], f16(5, 2, 16, 3), pool()[2]), pool(), i32(2), i32(2)),
    "copy no groups": lambda: q.quarot_kv_pages_copy((pool()[0], f16(5, 2, 16, 0), pool()[2]), pool(), i32(2), i32(2)),
    "copy lists": lambda: q.quarot_kv_pages_copy(pool(), pool(), i32(2), i32(3)),
    "sample rows": lambda: smp(x=f16(100)),
    "sample u": lambda: smp(u=torch.zeros(4)),
    "sample top_k": lambda: smp(top_k=i32(4)),
    "sample temperature": lambda: smp(temperature=torch.zeros(5, 1)),
    "sample tokens": lambda: smp(tokens=i32(6)),
}


@pytest.mark.parametrize("case", sorted(SHAPES))
def test_binding_refuses_before_launch(case):
    with pytest.raises(ValueError, match="must have shape|must be [0-9]-D|must hold groups"):
        SHAPES[case]()


def test_binding_refuses_host_tensors():
    for call in (att, res, smp, lambda: q.quarot_kv_pages_fork(i32(3, 4), i32(3), i32(9), i32(3)),
                 lambda: q.quarot_kv_pages_compact(i32(3, 4), i32(9)),
                 lambda: q.quarot_kv_pages_copy(pool(), pool(), i32(2), i32(2))):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()


def test_binding_refuses_types():
    for call in (lambda: att(slopes=f16(4)), lambda: att(begin=torch.zeros(8)),
                 lambda: smp(x=torch.zeros((5, 100), dtype=torch.float64)),
                 lambda: q.quarot_kv_pages_fork(torch.zeros(3, 4), i32(3), i32(9), i32(3)),
                 lambda: res(new=[1, 2, 3]), lambda: q.quarot_sample(f16(5, 9), None)):
        with pytest.raises(TypeError):
            call()


# ----------------------------------------------------------------- host ----

def test_host_code_under_asan_ubsan():
    """The entry points' host code under both sanitizers, with no device, against counting
    stand-ins of the launchers (tests/native/serving_abi_check.cpp)."""
    import test_sanitizers as ts
    if not os.path.exists(ts.HIPCC) or ts.clang_asan_runtime() is None:
        pytest.skip("needs hipcc and clang's ASan runtime")
    native = os.path.join(ROOT, "tests", "native")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host",
           "-fno-omit-frame-pointer"]
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "serving_abi_check")
        subprocess.run([ts.HIPCC, "-O1", "-g", "-std=c++17", *san, "-I", os.path.join(ROOT, "include"),
                        *(os.path.join(CSRC, f) for f in ("capi.cpp", "capi_scored.cpp", "capi_pages.cpp",
                                                          "capi_sample.cpp", "host_rules.cpp")),
                        *(os.path.join(native, f) for f in ("launch_stubs.cpp", "serving_abi_check.cpp")),
                        "-o", exe], check=True, capture_output=True, timeout=600)
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
                   HIP_VISIBLE_DEVICES="-1")
        res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
        assert res.returncode == 0 and res.stdout.strip().endswith("ok"), \
            res.stdout[-3000:] + res.stderr[-3000:]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_scored_steps():
    """A block's steps hold the tokens that its rows see, once each
    (tests/native/scored_plan_check.cpp)."""
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "check")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-I", CSRC,
                        os.path.join(ROOT, "tests", "native", "scored_plan_check.cpp"), "-o", exe],
                       check=True, capture_output=True)
        res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
        assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
