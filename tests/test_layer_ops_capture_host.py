"""What a context does with its workspace while its stream is being captured, on a HIP runtime that launches nothing (fake_hip.c) and
says that a stream is being captured as it is told to.  Each check runs in a process of its own."""
import ctypes as C
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
A = [(i + 1) << 44 for i in range(8)]          # addresses nothing reads
CAPTURE = """
static int status, error;
void set_capture(int s, int e) { status = s; error = e; }
int hipStreamIsCapturing(void* stream, int* out) { (void)stream; *out = status; return error; }
"""


def _library():
    capture = C.CDLL(os.environ["FAKE_CAPTURE"], mode=C.RTLD_GLOBAL)          # before the stand-in, whose streams are never captured
    sys.path.insert(0, HERE)
    from test_host_side import Library
    return Library(1 << 30), capture.set_capture


def check_no_workspace_is_set_while_the_stream_is_captured():
    """A clearing of the status word that a graph repeats would lose what calls outside it leave there."""
    lib, capture = _library()
    strp = lib.strp
    score = lambda: lib.launches(lambda: lib.lib.strp_gram(lib.h, A[0], strp.F32, 64, 512, 512, None, 64, A[1], 64, None, 0))
    for status, error in ((1, 0), (2, 0), (0, 900)):
        capture(status, error)
        st, launches = lib.launches(lambda: lib.lib.strp_set_workspace(lib.h, 1 << 41, 4096))
        assert st == strp.ESTATE and not launches and b"captured" in lib.lib.strp_last_error(lib.h)
        assert score()[0] == strp.OK            # the workspace it has, which is large enough
    capture(0, 0)
    assert lib.lib.strp_set_workspace(lib.h, 1 << 41, 4096) == strp.OK
    assert score()[0] == strp.ENOMEM


def check_every_call_that_uses_the_workspace_says_so():
    """Whether a graph has the workspace: after a captured call of each entry point that takes memory from it, not after the others, until another workspace is set."""
    lib, capture = _library()
    strp, dll, h = lib.strp, lib.lib, lib.h
    lib.workspace(1 << 50)
    sys.path.insert(0, HERE)
    from test_host_side import _module_calls
    refs = (strp.WeightRef * 2)(*[strp.WeightRef(1 << 50, strp.F32, 40, 64, 64) for _ in range(2)])
    score = strp.ScoreIn(A=A[0], a_dtype=strp.F32, ld=512, T=512, n_channels=64, group=8, mode=strp.WANDA, What=A[1], w_dtype=strp.F32, w_rows=64, ldw=64)
    linear = strp.LinearIn(W=A[0], X=A[1], Y=A[4], w_dtype=strp.BF16, x_dtype=strp.BF16, y_dtype=strp.BF16, M=512, K=4096, T=512, ldw=4096, ldx=512, ldy=512)
    init, step = _module_calls(lib, 136, 520, 3001, 260, strp.BF16)
    users = [lambda: dll.strp_gram(h, A[0], strp.F32, 64, 512, 512, None, 64, A[1], 64, None, 0),
             lambda: dll.strp_score_alloc(h, C.byref(score), A[2], A[3], 0, 1, None, None, 0.5, 1.0, 0.95, None, None),
             lambda: dll.strp_mask_topk(h, A[0], 3000000, 1000, 1, A[1], A[2], A[3]),
             lambda: dll.strp_weight_energy(h, refs, 2, 0.1, 0.1, 1.0, A[0]),
             lambda: dll.strp_refit(h, strp.SIDE_FC2, A[0], 64, 1.0, None, 0, A[1], strp.F32, 512, A[2], strp.F32, 512, 512, A[3], 64, A[4], 32, 64),
             init, step,
             lambda: dll.strp_linear(h, C.byref(linear)),
             lambda: dll.strp_token_logprobs(h, A[0], strp.F32, 100, 20, 24, None, None, A[3], 0, None, None, 0)]
    others = [lambda: dll.strp_layer_norm(h, A[0], strp.F32, 8, 8, 8, None, None, 0.0, A[1], 8),
              lambda: dll.strp_mask_topk_static(h, A[0], 30000, 1000, A[1], A[2], A[3])]
    assert init() == strp.OK
    for used, calls in ((1, users), (0, others)):
        for i, call in enumerate(calls):
            lib.workspace(1 << 50)
            assert call() == strp.OK and dll.strp_workspace_captured(h, 0) == 0, (used, i)
            capture(1, 0)
            assert call() == strp.OK and dll.strp_workspace_captured(h, 0) == used, (used, i)
            capture(0, 0)
            assert call() == strp.OK and dll.strp_workspace_captured(h, 0) == used, (used, i)
    capture(1, 0)
    assert users[0]() == strp.OK
    capture(0, 0)
    assert dll.strp_workspace_captured(h, 1) == 1 and dll.strp_workspace_captured(h, 0) == 0
    capture(1, 0)
    assert users[0]() == strp.OK
    capture(0, 0)
    lib.workspace(1 << 50)
    assert dll.strp_workspace_captured(h, 0) == 0 and dll.strp_workspace_captured(None, 0) == 0


CHECKS = [check_no_workspace_is_set_while_the_stream_is_captured, check_every_call_that_uses_the_workspace_says_so]


@pytest.fixture(scope="session")
def stand_ins(tmp_path_factory):
    at = tmp_path_factory.mktemp("fake")
    (at / "capture.c").write_text(CAPTURE)
    libs = {}
    for name, src in (("FAKE_HIP", os.path.join(HERE, "fake_hip.c")), ("FAKE_CAPTURE", str(at / "capture.c"))):
        libs[name] = str(at / (name.lower() + ".so"))
        subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-o", libs[name], src], check=True, timeout=120)
    return libs


@pytest.mark.parametrize("check", [c.__name__ for c in CHECKS])
def test_capture_host(stand_ins, check):
    from paper_2510_03246_amd import strp
    if not os.path.exists(strp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    out = subprocess.run([sys.executable, os.path.abspath(__file__), check], env=dict(os.environ, **stand_ins), capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr


if __name__ == "__main__":
    globals()[sys.argv[1]]()
