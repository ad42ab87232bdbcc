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


CHECKS = [check_no_workspace_is_set_while_the_stream_is_captured]


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
