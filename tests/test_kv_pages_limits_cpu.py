"""The largest calls on blocks that several rows hold, on the host alone (launches are noted by a stand-in for the HIP runtime, none runs): no launch has 2^32
threads, and lists that cannot be counted are refused.  In a process of its own."""
import ctypes as C
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from tests.test_kv_limits_cpu import INT_MAX, STAND_IN, THREADS, Library

P = 1 << 30


class Shared(Library):
    def context(self, **cfg):
        c = self.kv._config(self.kv.KvConfig(**cfg), workspace=1 << 20, workspace_bytes=1 << 62)
        self.ctx = C.c_void_p()
        rc = self.lib.br_kv_init_shared(C.byref(c), None, C.byref(self.ctx))
        self.launches()
        return rc

    def done(self, rc):
        got = self.launches()
        assert rc == 0 and got and all(0 < n < THREADS for _, n in got), (rc, got)
        return [name for name, _ in got]


def workers_and_rows_as_many_as_there_may_be(lib):
    kv = lib.kv
    for W, rows, width in ((2 ** 24 - 1, 1, 1), (2 ** 24 - 1, 4, 2), (2 ** 21, 31, 3), (2 ** 16 - 1, 1024, 1), (2 ** 16 - 1, 1000, 5), (2 ** 18, 255, 2), (1, 1024, 65536), (300, 97, 4000), (5000, 17, 9)):
        assert lib.context(n_workers=W, rows=rows, n_blocks=1, max_blocks=width) == 0
        forks, moves, fam = kv._Forks(from_=P, len=P), kv._Moves(src=P, dst=P, n=1), kv._Families(lead=P, members=4)
        lib.done(lib.lib.br_kv_fork(lib.ctx, C.byref(forks)))
        lib.done(lib.lib.br_kv_compact(lib.ctx, C.byref(moves)))
        lib.done(lib.lib.br_kv_copy(lib.ctx, C.byref(lib.layer), C.byref(moves)))
        lib.done(lib.lib.br_kv_plan(lib.ctx, C.byref(fam)))
        keep, out = kv._Lengths(keep=P, add=P), kv._StepOut(slot=P, token_cap=1)
        copies = kv._Moves(src=P, dst=P, n=rows)
        lib.done(lib.lib.br_kv_step_shared(lib.ctx, C.byref(keep), C.byref(out), C.byref(copies)))
        a = kv._Attention(q=P, out=P, q_token=64, q_head=64, out_token=64, out_head=64, n_tokens=3, max_count=1, dtype=0, scale=1.0)
        lib.done(lib.lib.br_kv_attend_shared(lib.ctx, C.byref(lib.layer), C.byref(a)))
        diff = kv._Diff(lam=P)
        lib.done(lib.lib.br_kv_attend_diff(lib.ctx, C.byref(lib.layer), C.byref(a), C.byref(diff)))
        lib.lib.br_kv_free(lib.ctx)
    for W, rows in ((2 ** 24, 1), (2 ** 16, 1024)):
        assert lib.context(n_workers=W, rows=rows, n_blocks=1, max_blocks=1) == -1 and not lib.ctx.value


def lists_as_long_as_their_places_can_be_counted(lib):
    kv = lib.kv
    for W, sizes in ((1, {}), (3, dict(n_kv_heads=8, n_q_heads=8, head_dim=256, block_tokens=128)), (1024, dict(head_dim=96))):
        assert lib.context(n_workers=W, rows=2, n_blocks=1, max_blocks=1, **sizes) == 0
        most = (INT_MAX - 256) // W
        for n, rc in ((most, 0), (most + 1, -1), (INT_MAX, -1), (-1, -1)):
            m = kv._Moves(src=P, dst=P, n=n)
            for call in (lambda: lib.lib.br_kv_copy(lib.ctx, C.byref(lib.layer), C.byref(m)), lambda: lib.lib.br_kv_compact(lib.ctx, C.byref(m))):
                got = call()
                assert got == rc, (W, n, got)
                if rc:
                    assert lib.launches() == []
                else:
                    lib.done(got)
        lib.lib.br_kv_free(lib.ctx)


def query_rows_that_can_be_counted(lib):
    """Two rows for each query head in differential attention."""
    kv = lib.kv
    assert lib.context(rows=2, n_blocks=1, max_blocks=1, n_kv_heads=1, n_q_heads=1024, head_dim=64) == 0
    a = dict(q=P, out=P, q_token=64, q_head=64, out_token=64, out_head=64, max_count=1, dtype=0, scale=1.0)
    diff, most = kv._Diff(lam=P), (INT_MAX - 256) // 2048
    for n, rc in ((most, 0), (most + 1, -1), (INT_MAX, -1)):
        assert lib.lib.br_kv_attend_diff(lib.ctx, C.byref(lib.layer), C.byref(kv._Attention(n_tokens=n, **a)), C.byref(diff)) == rc, n
        assert bool(lib.launches()) == (rc == 0)
    lib.lib.br_kv_free(lib.ctx)


SCENARIOS = [workers_and_rows_as_many_as_there_may_be, lists_as_long_as_their_places_can_be_counted, query_rows_that_can_be_counted]


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    at = tmp_path_factory.mktemp("hip")
    (at / "hip.cpp").write_text(STAND_IN)
    subprocess.check_call(["g++", "-shared", "-fPIC", "-O1", "-o", str(at / "hip.so"), str(at / "hip.cpp")])
    return str(at / "hip.so")


@pytest.mark.parametrize("scenario", SCENARIOS, ids=lambda f: f.__name__)
def test_limits(stand_in, scenario):
    run = subprocess.run([sys.executable, os.path.abspath(__file__), stand_in, scenario.__name__], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


if __name__ == "__main__":
    next(f for f in SCENARIOS if f.__name__ == sys.argv[2])(Shared(sys.argv[1]))
