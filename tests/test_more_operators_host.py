"""The host module and its build: what results hold, calls that are noted, a machine without a compiler for it."""
import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_operators_binding import BF, F, I32


@pytest.fixture
def noting(lib):
    host = ops._lib.host()
    host.pretend(True)
    yield host
    host.pretend(False)


def held(results):
    return max(t.untyped_storage().nbytes() for t in results), sum(-(-t.numel() * t.element_size() // 256) * 256 for t in results)


def test_results_hold_no_workspace(noting):
    # 136 KB of counts, 0.7 MB of sums and scores, a sum for each 2 KB
    r = noting.route(torch.zeros(3000, 200), 2, False, None)
    assert len(r) == 6 and held(r)[0] <= held(r)[1] + 8192
    r = noting.verify(torch.zeros(200, 6, 50), torch.zeros(200, 5, dtype=I32), torch.zeros(200, 5), torch.zeros(200, 50), None, 1.0, None)
    assert len(r) == 3 and held(r)[0] <= held(r)[1] + 8192
    r = noting.norm([torch.zeros(4, 3000, dtype=BF)] * 500, 1.0, 4, False)
    assert len(r) == 2 and held(r)[0] <= held(r)[1] + 8192 and r[0].dtype == F
    assert noting.pretend(True)[10] > 8192                   # (which is there all the same)


def test_the_library_is_built_without_the_host_modules_compiler(monkeypatch, tmp_path, capsys):
    import os

    from paper_1903_05133_gb300 import _build
    ran = []

    def run(cmd):
        """Each command's result is made; the host module's compiler finds no header."""
        ran.append(cmd)
        if os.path.join(_build.CSRC, "host.cpp") in cmd:
            raise RuntimeError("Python.h: No such file or directory")
        open(cmd[cmd.index("-o") + 1], "w").close()
        return ""

    def no_compiler(cmd):
        if os.path.join(_build.CSRC, "host.cpp") in cmd:
            raise FileNotFoundError("g++")
        return run(cmd)

    def no_pytorch(out):
        raise RuntimeError("PyTorch not found")
    monkeypatch.setattr(_build, "BUILD_DIR", str(tmp_path / "build"))
    monkeypatch.setattr(_build, "LIB_PATH", str(tmp_path / "libhier_avg.so"))
    monkeypatch.setattr(_build, "HOST_PATH", str(tmp_path / "_host.so"))
    for runs, command in ((run, None), (no_compiler, None), (run, no_pytorch)):
        (tmp_path / "_host.so").write_text("of an older build")
        monkeypatch.setattr(_build, "_run", runs)
        if command:
            monkeypatch.setattr(_build, "_host_command", command)
        assert _build.build() == str(tmp_path / "libhier_avg.so")
        assert (tmp_path / "libhier_avg.so").exists() and not (tmp_path / "_host.so").exists()
        assert "host module" in capsys.readouterr().err
        (tmp_path / "libhier_avg.so").unlink()
    monkeypatch.setattr(ops._lib, "_host", None)             # and its absence is an error where it is used
    with pytest.raises(RuntimeError, match="missing"):
        ops._lib.host()
    # what the library itself needs is an error still

    def no_nvcc(cmd):
        raise RuntimeError("command failed")
    monkeypatch.setattr(_build, "_run", no_nvcc)
    with pytest.raises(RuntimeError, match="command failed"):
        _build.build()
    assert not (tmp_path / "libhier_avg.so").exists()


def test_calls_are_noted_for_the_thread_that_asks(noting):
    import threading
    z = torch.zeros(3, 4)
    assert noting.route(z, 2, False, None) is not None
    other = []
    t = threading.Thread(target=lambda: other.append((noting.route(z, 2, False, None), noting.pretend(False))))
    t.start()
    t.join()
    assert other == [(None, None)]                           # a CPU tensor is none of a GPU there
    assert len(noting.pretend(True)) == 18                   # and the call that was noted here is still there


def test_rows_beyond_2_30_elements_are_refused(lib):
    # A row's columns are counted in 32 bits: with a thread for four single elements, the column behind a row of 2^31 - 1 is
    # the first, at most 2^29 - 1, and 2^31 more.
    from test_operators_abi import EUNSUPPORTED, P
    for width, status in ((1 << 30, 0), ((1 << 30) + 1, EUNSUPPORTED), ((1 << 31) - 1, EUNSUPPORTED)):
        for rows in (0, 1) if status else (0,):
            for kind in (0, 1):
                assert lib.hier_avg_dispatch(P, kind, rows, width, width, P, 1, P, 1, P, width, None) == status
                assert lib.hier_avg_combine(P, kind, rows, width, width, P, 1, P, P, width, kind, None) == status
                assert lib.hier_avg_combine_backward(P, kind, width, P, kind, rows, width, width, P, 1, P, P, 1, P, width, P, None) == status
    # what is allowed stays in 32 bits: V elements a part, U parts a thread, the last read of a thread without parts left
    for V, U in ((1, 4), (1, 8), (4, 1), (4, 2), (8, 1), (8, 2), (8, 4)):
        parts = (1 << 30) // V
        lanes = -(-parts // U)
        assert lanes - 1 + lanes * U < 1 << 31 and (lanes - 1 + (U - 1) * lanes) * V < 1 << 31
