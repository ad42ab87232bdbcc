"""Refusals and launches of the paged cache's operators and of the verification of drafts on a HIP runtime that launches nothing (fake_hip.c), without a GPU.
Each check runs in a process of its own, where the stand-in is loaded before the library."""
import ctypes as C
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
A = [(i + 1) << 44 for i in range(14)]         # addresses nothing reads


def _library(ws_bytes=1 << 40):
    sys.path.insert(0, HERE)
    from test_host_side import Library
    return Library(ws_bytes)


def _cache(strp, **kw):
    a = dict(K=A[0], V=A[1], K_scale=A[2], V_scale=A[3], table=A[4], past=A[5], seq_start=A[6], format=strp.CACHE_BF16, kv_heads=2, d_head=64, page=16, pages=10, n_seq=3, ld_table=7)
    a.update(kw)
    return strp.Cache(**a)


# what both operators refuse of the cache and of T
BAD_CACHE = [dict(K=None), dict(V=None), dict(table=None), dict(past=None), dict(format=3), dict(format=-1), dict(format=1), dict(format=2, K_scale=None), dict(format=2, V_scale=None),
             dict(kv_heads=0), dict(kv_heads=1026), dict(d_head=0), dict(d_head=60), dict(d_head=136), dict(d_head=-8), dict(page=0), dict(page=8), dict(page=24), dict(page=131072),
             dict(page=-16), dict(pages=0), dict(n_seq=0), dict(n_seq=65537), dict(ld_table=0), dict(ld_table=(1 << 26) + 1), dict(seq_start=None), dict(K=A[0] + 8), dict(V=A[1] + 2),
             dict(format=2, K_scale=A[2] + 4)]
GOOD_CACHE = [dict(), dict(format=2), dict(seq_start=None, n_seq=1), dict(K_scale=None, V_scale=None), dict(d_head=8), dict(d_head=128), dict(page=65536, ld_table=1 << 14), dict(n_seq=65536),
              dict(pages=0x7fffffff), dict(kv_heads=1)]


def check_append():
    lib = _library()
    strp = lib.strp

    def call(cache=None, **kw):
        a = dict(K=A[7], V=A[8], Q=A[9], Qr=A[10], inv_freq=A[11], dtype=strp.BF16, heads=4, rot=8, pairs=0, T=20, ldk=24, ldv=24, ldq=24, ldqr=24)
        a.update(kw)
        return lib.launches(lambda: lib.lib.strp_cache_append(lib.h, C.byref(strp.CacheAppendIn(cache=_cache(strp, **(cache or {})), **a))))

    for good in [dict(cache=c) for c in GOOD_CACHE] + [dict(Q=None, Qr=None, ldq=0, ldqr=0, heads=0), dict(Qr=A[9]), dict(rot=0, inv_freq=None), dict(T=1, ldk=8, ldv=8, ldq=8, ldqr=8), dict(pairs=1),
                 dict(dtype=strp.F32, cache=dict(format=1)), dict(dtype=strp.F32, cache=dict(format=2)), dict(heads=1024), dict(T=65, ldk=72, ldv=72, ldq=72, ldqr=72),
                 dict(T=1 << 27, ldk=1 << 27, ldv=1 << 27, ldq=1 << 27, ldqr=1 << 27)]:
        st, launches = call(**good)
        assert st == strp.OK and len(launches) == 1, good
        assert launches[0][1][0] * 512 < 1 << 32 and 0 < launches[0][1][1] <= 65535
    for bad in [dict(cache=c) for c in BAD_CACHE] + [dict(K=None), dict(V=None), dict(Q=None), dict(Qr=None), dict(inv_freq=None), dict(dtype=2), dict(dtype=strp.F32), dict(heads=0), dict(heads=1025),
                dict(rot=7), dict(rot=-2), dict(rot=66), dict(T=0), dict(T=-1), dict(T=(1 << 27) + 1, ldk=1 << 28, ldv=1 << 28, ldq=1 << 28, ldqr=1 << 28), dict(ldk=16), dict(ldv=23), dict(ldq=19),
                dict(ldqr=16), dict(Qr=A[9], ldqr=32), dict(K=A[7] + 8), dict(V=A[8] + 2), dict(Q=A[9] + 4), dict(Qr=A[10] + 8)]:
        st, launches = call(**bad)
        assert st == strp.EINVAL and not launches and lib.lib.strp_last_error(lib.h), bad
    assert lib.lib.strp_cache_append(lib.h, None) == strp.EINVAL and lib.lib.strp_cache_append(None, C.byref(strp.CacheAppendIn(cache=_cache(strp)))) == strp.EINVAL


def check_attention():
    lib = _library()
    strp = lib.strp

    def make(cache=None, **kw):
        a = dict(Q=A[7], C=A[8], kv_of_head=None, dtype=strp.BF16, heads=4, scale=0.125, T=20, ldq=24, ldc=24)
        a.update(kw)
        return strp.CacheAttentionIn(cache=_cache(strp, **(cache or {})), **a)

    call = lambda **kw: lib.launches(lambda: lib.lib.strp_cache_attention(lib.h, C.byref(make(**kw))))
    for prec in (strp.PREC_FAST, strp.PREC_SPLIT):
        assert lib.lib.strp_set_precision(lib.h, prec) == strp.OK
        for good in [dict(cache=c) for c in GOOD_CACHE] + [dict(kv_of_head=A[9], heads=3), dict(kv_of_head=A[9], heads=1), dict(dtype=strp.F32, cache=dict(format=1)), dict(dtype=strp.F32, cache=dict(format=2)),
                     dict(T=1, ldq=8, ldc=8), dict(heads=1024), dict(T=1 << 20, ldq=1 << 20, ldc=1 << 20), dict(scale=2e38)]:
            st, launches = call(**good)
            assert st == strp.OK and launches, good
            assert all(g[0] * 512 < 1 << 32 and 0 < g[1] <= 65535 for _, g in launches), launches
    for bad in [dict(cache=c) for c in BAD_CACHE] + [dict(Q=None), dict(C=None), dict(dtype=2), dict(dtype=strp.F32), dict(heads=0), dict(heads=3), dict(heads=1026), dict(kv_of_head=A[9], heads=1025),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=2.4e38), dict(T=0), dict(ldq=16), dict(ldc=20), dict(Q=A[7] + 8), dict(C=A[8] + 2),
                dict(heads=1024, T=(1 << 20) + 1, ldq=1 << 21, ldc=1 << 21)]:
        st, launches = call(**bad)
        assert st == strp.EINVAL and not launches and lib.lib.strp_last_error(lib.h), bad
    assert lib.lib.strp_cache_attention(lib.h, None) == strp.EINVAL and lib.lib.strp_cache_attention(None, C.byref(make())) == strp.EINVAL
    # what it asks for is enough, and without it nothing is enqueued
    for dh in (8, 64, 80, 128):
        need = lib.lib.strp_cache_attention_workspace_bytes(dh)
        for T in (1, 300, 5000):
            args = dict(cache=dict(d_head=dh), T=T, ldq=5000, ldc=5000)
            lib.workspace(need)
            assert call(**args)[0] == strp.OK
            lib.workspace(need // 8)
            st, launches = call(**args)
            assert st == strp.ENOMEM and not launches
    bare = C.c_void_p()
    assert lib.lib.strp_create(C.byref(bare), 0, None) == strp.OK
    assert lib.lib.strp_cache_attention(bare, C.byref(make())) == strp.ENOMEM
    assert lib.lib.strp_cache_attention_workspace_bytes(0) == 0 and lib.lib.strp_cache_attention_workspace_bytes(129) == 0


def check_verify():
    lib = _library()
    strp = lib.strp

    def make(**kw):
        a = dict(target=A[0], draft=A[1], draft_id=A[2], u=A[3], u_next=A[4], draft_start=A[5], accepted=A[6], next_id=A[7], dtype=strp.BF16, V=1000, n_seq=3, temperature=0.7, T=12, ldt=16, ldd=16)
        a.update(kw)
        return strp.VerifyDraftIn(**a)

    call = lambda **kw: lib.launches(lambda: lib.lib.strp_verify_draft(lib.h, C.byref(make(**kw))))
    for good in (dict(), dict(dtype=strp.F32), dict(T=0, draft=None, draft_id=None, u=None, ldd=0), dict(T=0, draft=None, draft_id=None, u=None, ldd=0, draft_start=None), dict(n_seq=1, draft_start=None),
                 dict(V=1), dict(V=1 << 30), dict(T=1 << 20, n_seq=65536, ldt=(1 << 20) + 65536, ldd=1 << 20), dict(temperature=1e-30), dict(temperature=1e30)):
        st, launches = call(**good)
        assert st == strp.OK and launches, good
        assert all(g[0] * g[1] * 256 < 1 << 32 and 0 < g[1] <= 65535 for _, g in launches), launches
    for bad in (dict(target=None), dict(draft=None), dict(draft_id=None), dict(u=None), dict(u_next=None), dict(accepted=None), dict(next_id=None), dict(draft_start=None), dict(dtype=2), dict(V=0), dict(V=-3),
                dict(V=(1 << 30) + 1), dict(n_seq=0), dict(n_seq=65537, ldt=65560), dict(T=-1), dict(T=(1 << 20) + 8, ldt=1 << 21, ldd=1 << 21), dict(temperature=0.0), dict(temperature=-1.0),
                dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-31), dict(ldt=8), dict(ldt=17), dict(ldd=8), dict(ldd=20), dict(target=A[0] + 8), dict(draft=A[1] + 2)):
        st, launches = call(**bad)
        assert st == strp.EINVAL and not launches and lib.lib.strp_last_error(lib.h), bad
    assert lib.lib.strp_verify_draft(lib.h, None) == strp.EINVAL and lib.lib.strp_verify_draft(None, C.byref(make())) == strp.EINVAL
    for V in (1, 300, 50000, 130001):
        for T, n in ((0, 1), (4, 1), (300, 70), (4096, 512)):
            lib.workspace(lib.lib.strp_verify_draft_workspace_bytes(V, T, n))
            for dt in (strp.BF16, strp.F32):
                assert call(V=V, T=T, n_seq=n, ldt=8192, ldd=4096, dtype=dt)[0] == strp.OK, (V, T, n)
    lib.workspace(4096)
    st, launches = call(V=50000)
    assert st == strp.ENOMEM and not launches
    bare = C.c_void_p()
    assert lib.lib.strp_create(C.byref(bare), 0, None) == strp.OK
    assert lib.lib.strp_verify_draft(bare, C.byref(make())) == strp.ENOMEM
    for bad in ((0, 5, 1), (5, -1, 1), (5, 5, 0), ((1 << 30) + 1, 5, 1)):
        assert lib.lib.strp_verify_draft_workspace_bytes(*bad) == 0


def check_the_current_device_is_left_as_it_was():
    lib = _library()
    strp, fake = lib.strp, lib.fake
    h = C.c_void_p()
    assert lib.lib.strp_create(C.byref(h), 1, None) == strp.OK
    assert lib.lib.strp_set_workspace(h, 1 << 40, 1 << 30) == strp.OK
    append = strp.CacheAppendIn(cache=_cache(strp), K=A[7], V=A[8], dtype=strp.BF16, T=20, ldk=24, ldv=24)
    attention = strp.CacheAttentionIn(cache=_cache(strp), Q=A[7], C=A[8], dtype=strp.BF16, heads=4, scale=1.0, T=20, ldq=24, ldc=24)
    verify = strp.VerifyDraftIn(target=A[0], u_next=A[4], accepted=A[6], next_id=A[7], dtype=strp.BF16, V=10, n_seq=2, temperature=1.0, T=0, ldt=8)
    for current in (0, 1):
        fake.hipSetDevice(current)
        for f, a in ((lib.lib.strp_cache_append, append), (lib.lib.strp_cache_attention, attention), (lib.lib.strp_verify_draft, verify)):
            assert f(h, C.byref(a)) == strp.OK
            now = C.c_int(-1)
            assert fake.hipGetDevice(C.byref(now)) == 0 and now.value == current


def check_verify_workspace_is_near_what_a_call_takes():
    """At most twice what a call takes and 256 KB (slices are whole numbers, and so are the workgroups of few columns), and never less for larger sizes than for smaller ones: a program asks once, for its largest call."""
    lib = _library()
    strp = lib.strp
    need = lib.lib.strp_verify_draft_workspace_bytes

    def least(V, T, n):
        most = 0
        for dt in (strp.BF16, strp.F32):
            ld = (T + n + 7) // 8 * 8
            call = strp.VerifyDraftIn(target=A[0], draft=A[1], draft_id=A[2], u=A[3], u_next=A[4], draft_start=A[5], accepted=A[6], next_id=A[7], dtype=dt, V=V, n_seq=n, temperature=1.0,
                                      T=T, ldt=ld, ldd=ld)
            low, high = 4096, 1 << 34
            while high - low > 256:
                mid = (low + high) // 2
                lib.workspace(mid)
                st, _ = lib.launches(lambda: lib.lib.strp_verify_draft(lib.h, C.byref(call)))
                low, high = (low, mid) if st == strp.OK else (mid, high)
            most = max(most, high)
        return most

    for V in (300, 5003, 50000, 130001):
        for T, n in ((0, 1), (0, 64), (4, 1), (40, 9), (300, 70), (1024, 256), (4096, 1024), (8192, 2048), (1 << 20, 65536)):
            asked, taken = need(V, T, n), least(V, T, n)
            assert taken <= asked <= 2 * taken + (256 << 10), (V, T, n, asked, taken)
            for smaller in ((V, T // 2, n), (V, T, (n + 1) // 2), (V // 2, T, n), (V, T - 1 if T else 0, n), (V, T // 3, (n + 2) // 3)):
                assert need(*smaller) <= asked and least(*smaller) <= asked, (V, T, n, smaller)


CHECKS = [check_append, check_attention, check_verify, check_the_current_device_is_left_as_it_was]


@pytest.fixture(scope="session")
def fake_hip(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("fake") / "libfake_hip.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "fake_hip.c")], check=True, timeout=120)
    return so


@pytest.mark.parametrize("check", [c.__name__ for c in CHECKS])
def test_cache_host(fake_hip, check):
    from paper_2510_03246_amd import strp
    if not os.path.exists(strp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    out = subprocess.run([sys.executable, os.path.abspath(__file__), check], env=dict(os.environ, FAKE_HIP=fake_hip), capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr


def test_verify_workspace_is_near_what_a_call_takes(fake_hip):
    test_cache_host(fake_hip, "check_verify_workspace_is_near_what_a_call_takes")


def test_binding_structs_mirror_the_header(tmp_path):
    from paper_2510_03246_amd import strp
    pairs = [("strp_cache", "ld_table", strp.Cache), ("strp_cache_append_in", "ldqr", strp.CacheAppendIn), ("strp_cache_append_in", "pairs", strp.CacheAppendIn),
             ("strp_cache_attention_in", "ldc", strp.CacheAttentionIn), ("strp_cache_attention_in", "scale", strp.CacheAttentionIn),
             ("strp_verify_draft_in", "ldd", strp.VerifyDraftIn), ("strp_verify_draft_in", "temperature", strp.VerifyDraftIn)]
    src = tmp_path / "layout.c"
    body = "".join(f'  printf("%zu %zu\\n", sizeof({c}), offsetof({c}, {f}));\n' for c, f, _ in pairs)
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "strp.h"\nint main(void) {\n' + body + '  printf("%d %d %d\\n", STRP_CACHE_BF16, STRP_CACHE_F32, STRP_CACHE_Q4);\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(HERE), "include"), "-o", str(exe), str(src)], check=True, timeout=120)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=30).stdout.split("\n")
    for (cname, field, cls), line in zip(pairs, out):
        size, off = (int(x) for x in line.split())
        assert C.sizeof(cls) == size and getattr(cls, field).offset == off, (cname, field)
    assert out[len(pairs)] == f"{strp.CACHE_BF16} {strp.CACHE_F32} {strp.CACHE_Q4}"


if __name__ == "__main__":
    globals()[sys.argv[1]]()
