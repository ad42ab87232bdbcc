"""Which kernels the decoder layer's operators launch at the sizes that their tests on a GPU compare with the definitions (layer_ops_sizes.py): every one
that the library has.  On a HIP runtime that launches nothing (fake_hip.c); each check runs in a process of its own."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
A = [(i + 1) << 44 for i in range(8)]          # addresses nothing reads


def ld8(n):
    return (n + 7) // 8 * 8


def _library():
    from test_host_side import Library
    return Library(1 << 50)


def _in_library(lib, part):
    """mangled names of the library's kernels that hold `part`, without the class of their parameters"""
    out = subprocess.run(["nm", lib.strp.LIB_PATH], capture_output=True, text=True, check=True).stdout
    return {n for n in re.findall(r"_ZN4strp\d+(\w*" + part + r"\w*)EvNS_\w+PE\b", out) if "__device_stub__" not in n}


def _short(name):
    return re.match(r"_ZN4strp\d+(\w+)EvNS_\w+PE$", name)[1]


def check_linear():
    import layer_ops_sizes as sizes
    lib = _library()
    strp, seen = lib.strp, set()
    kernels = _in_library(lib, "linear_")
    for of, pairs in ((sizes.LINEAR_BF16, [(0, 0)]), (sizes.LINEAR_F32, [(1, 1), (1, 0), (0, 1)])):
        for M, K, T in of:
            for w, x in pairs:
                for y in (0, 1):
                    a = strp.LinearIn(W=A[0], X=A[1], Y=A[4], w_dtype=w, x_dtype=x, y_dtype=y, M=M, K=K, T=T, ldw=ld8(K), ldx=ld8(T), ldy=ld8(T))
                    st, launches = lib.launches(lambda: lib.lib.strp_linear(lib.h, C.byref(a)))
                    assert st == strp.OK
                    names = [_short(n) for n, _ in launches]
                    seen |= {(names[0], len(names) > 1)} | {(n, True) for n in names[1:]}
    assert {n for n, _ in seen} == kernels and len(kernels) == 6 + 4 + 18 + 2, sorted(kernels - {n for n, _ in seen})
    # whole and in parts; few tokens are never in parts
    assert seen == {(n, s) for n in kernels for s in (False, True) if not (s and "few" in n) and (s or "join" not in n)}


def check_norm():
    import layer_ops_sizes as sizes
    lib = _library()
    seen, kernels = set(), _in_library(lib, "layer_norm_")
    for dt, name in enumerate(("bf16", "f32")):
        for d, T in sizes.NORM[name] + sizes.NORM_TALL:
            st, ((kernel, grid),) = lib.launches(lambda: lib.lib.strp_layer_norm(lib.h, A[0], dt, d, T, ld8(T), None, None, 1e-5, A[1], ld8(T)))
            assert st == lib.strp.OK
            chunks = -(-T // (4 if dt else 8))
            seen.add((_short(kernel), 0 if "tall" in kernel else [c for c in (16, 8, 4, 2, 1) if -(-chunks // c) == grid[0]][0]))
    assert {n for n, _ in seen} == kernels and len(kernels) == 10
    assert seen == {(n, c) for n in kernels for c in ((0,) if "tall" in n else (16, 8, 4, 2, 1))}


def check_logprobs():
    import layer_ops_sizes as sizes
    lib = _library()
    seen, kernels = set(), _in_library(lib, "logit_streams_") | _in_library(lib, "token_finish_")
    for V, T, k in sizes.LOGPROBS:
        for dt in (0, 1):
            st, launches = lib.launches(lambda: lib.lib.strp_token_logprobs(lib.h, A[0], dt, V, T, ld8(T), A[1], A[2], A[3], k, A[4], A[5], T))
            assert st == lib.strp.OK
            seen |= {_short(n) for n, _ in launches}
    assert seen == kernels and len(kernels) == 6


def check_attention():
    """by width and type, and for bf16 by the context's precision"""
    lib = _library()
    strp, seen = lib.strp, {}
    kernels = _in_library(lib, "attention_")
    for prec in (strp.PREC_FAST, strp.PREC_SPLIT):
        assert lib.lib.strp_set_precision(lib.h, prec) == strp.OK
        for dt in (strp.BF16, strp.F32):
            for dh in (1, 64, 65, 96, 97, 128):
                a = strp.AttentionIn(Q=A[0], K=A[1], V=A[2], C=A[3], dtype=dt, heads=4, kv_heads=2, d_head=dh, scale=1.0, T=300, ldq=304, ldk=304, ldv=304, ldc=304)
                st, ((kernel, _),) = lib.launches(lambda: lib.lib.strp_attention(lib.h, C.byref(a)))
                assert st == strp.OK
                seen[prec, dt, dh] = _short(kernel)
    assert set(seen.values()) == kernels and len(kernels) == 9
    for prec in (strp.PREC_FAST, strp.PREC_SPLIT):
        for a, b in ((1, 64), (65, 96), (97, 128)):
            assert seen[prec, strp.BF16, a] == seen[prec, strp.BF16, b] != seen[1 - prec, strp.BF16, a]
            assert seen[prec, strp.F32, a] == seen[prec, strp.F32, b] == seen[1 - prec, strp.F32, a]


def check_attention_scales():
    """in powers of two a scale has to be finite too"""
    lib = _library()
    strp = lib.strp
    for scale, want in ((1e-30, strp.OK), (2e38, strp.OK), (2.4e38, strp.EINVAL), (3.4e38, strp.EINVAL), (float("inf"), strp.EINVAL), (float("nan"), strp.EINVAL), (0.0, strp.EINVAL)):
        a = strp.AttentionIn(Q=A[0], K=A[1], V=A[2], C=A[3], dtype=strp.BF16, heads=4, kv_heads=2, d_head=64, scale=scale, T=300, ldq=304, ldk=304, ldv=304, ldc=304)
        st, launches = lib.launches(lambda: lib.lib.strp_attention(lib.h, C.byref(a)))
        assert st == want and len(launches) == (want == strp.OK), scale


CHECKS = [check_linear, check_norm, check_logprobs, check_attention, check_attention_scales]


@pytest.fixture(scope="session")
def fake_hip(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("fake") / "libfake_hip.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "fake_hip.c")], check=True, timeout=120)
    return so


@pytest.mark.parametrize("check", [c.__name__ for c in CHECKS])
def test_layer_ops_plans(fake_hip, check):
    from paper_2510_03246_amd import strp
    if not os.path.exists(strp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    out = subprocess.run([sys.executable, os.path.abspath(__file__), check], env=dict(os.environ, FAKE_HIP=fake_hip), capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr


if __name__ == "__main__":
    globals()[sys.argv[1]]()
