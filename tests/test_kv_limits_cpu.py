"""The largest calls of the worker's part that are accepted, and the first that are not, on the host alone: the HIP runtime's entry points are taken by a
stand-in that notes the launches and runs none.  In a process of its own."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = r"""
#include <cstddef>
#include <cstdint>
#include <map>
#include <string>
struct D3 { uint32_t x, y, z; };
static std::map<const void *, std::string> names;
static std::string log_;
static D3 g, b; static size_t shm; static void *str;
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *n, unsigned, void *, void *, void *, void *, int *) { names[f] = n; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(D3 gg, D3 bb, size_t s, void *st) { g = gg, b = bb, shm = s, str = st; return 0; }
int __hipPopCallConfiguration(D3 *gg, D3 *bb, size_t *s, void **st) { *gg = g, *bb = b, *s = shm, *st = str; return 0; }
int hipLaunchKernel(const void *f, D3 gg, D3 bb, void **, size_t, void *) {
  log_ += names[f] + " " + std::to_string((uint64_t)gg.x * bb.x) + " " + std::to_string(gg.x) + "\n";
  return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int *v, int, int) { *v = 256; return 0; }
const char *stand_in_log() { static std::string out; out = log_; log_.clear(); return out.c_str(); }
}
"""
THREADS = 2 ** 32  # of a launch: fewer
INT_MAX = 2 ** 31 - 1


class Library:
    def __init__(self, so):
        self.fake = C.CDLL(so, mode=C.RTLD_GLOBAL)
        self.fake.stand_in_log.restype = C.c_char_p
        from paper_2605_06113_amd import kv
        self.kv, self.lib = kv, kv.load()
        self.layer = kv._Layer(k=1 << 30, v=1 << 30, k_scale=1 << 30, v_scale=1 << 30)

    def context(self, **cfg):
        c = self.kv._config(self.kv.KvConfig(**cfg), workspace=1 << 20, workspace_bytes=1 << 62)
        self.ctx = C.c_void_p()
        return self.lib.br_kv_init(C.byref(c), None, C.byref(self.ctx))

    def launches(self):
        found = re.findall(r"(br_kv_k_[a-z]+(?:_rows)?)\S* (\d+) (\d+)", self.fake.stand_in_log().decode())
        self.blocks = [int(n) for _, _, n in found]
        return [(name, int(n)) for name, n, _ in found]

    def tokens(self, call, **kw):
        a = self.kv._Tokens(**{**dict(k=1 << 30, v=1 << 30, slot=1 << 30, k_token=64, k_head=64, v_token=64, v_head=64, n_tokens=1, dtype=0), **kw})
        return getattr(self.lib, call)(self.ctx, C.byref(self.layer), C.byref(a))


def as_many_workers_as_a_launch_has_blocks_for(lib):
    for W, rows in ((2 ** 24 - 1, 1), (2 ** 24 - 1, 4), (2 ** 16 - 1, 1024)):
        assert lib.context(n_workers=W, rows=rows, n_blocks=1, max_blocks=1) == 0
        lib.launches()
        keep, out = lib.kv._Lengths(keep=1 << 30, add=1 << 30), lib.kv._StepOut(slot=1 << 30, token_cap=1)
        assert lib.lib.br_kv_step(lib.ctx, C.byref(keep), C.byref(out)) == 0
        done = lib.launches()
        assert [n for n, _ in done] == ["br_kv_k_step"] and all(n < THREADS for _, n in done)
        lib.lib.br_kv_free(lib.ctx)
    for W, rows in ((2 ** 24, 1), (2 ** 24 + 1, 3), (2 ** 16, 1024)):
        assert lib.context(n_workers=W, rows=rows, n_blocks=1, max_blocks=1) == -1 and not lib.ctx.value


def lists_as_long_as_their_places_can_be_counted(lib):
    for W in (1, 3, 1024):
        assert lib.context(n_workers=W, rows=2, n_blocks=1, max_blocks=1) == 0
        lib.launches()
        most = (INT_MAX - 256) // W
        for call in ("br_kv_append", "br_kv_read"):
            assert lib.tokens(call, n_tokens=most) == 0
            done = lib.launches()
            assert [n for n, _ in done] == ["br_kv_k_tokens"] and all(n < THREADS for _, n in done)
            for n in {most + 1, most + 100 // W + 1, max(most + 1, INT_MAX // W), INT_MAX}:
                assert lib.tokens(call, n_tokens=n) == -1 and lib.launches() == []
        lib.lib.br_kv_free(lib.ctx)


def a_workspace_holds_the_pieces_of_what_is_launched(lib):
    """Two pieces of 128 query rows for each block of the largest launch on 256 compute units, their maxima and sums, a counter a block, and
    the tables: no more than that and the places' alignment."""
    for dim in (64, 96, 128, 192, 256):
        cfg = dict(rows=3, n_blocks=4, max_blocks=5, head_dim=dim)
        assert lib.context(**cfg) == 0
        lib.launches()
        most = 0
        for queries in (1, 20, 40, 100):
            a = lib.kv._Attention(q=1 << 30, out=1 << 30, q_token=dim, q_head=dim, out_token=dim, out_head=dim, n_tokens=300, max_count=queries, dtype=0, scale=1.0)
            assert lib.lib.br_kv_attend(lib.ctx, C.byref(lib.layer), C.byref(a)) == 0
            assert [n for n, _ in lib.launches()] in (["br_kv_k_attend"], ["br_kv_k_attend_rows"])
            most = max([most] + lib.blocks)
        need = most * (2 * 128 * 4 * (dim + 2) + 4)
        assert need <= lib.kv.workspace_bytes(lib.kv.KvConfig(**cfg)) <= need + 4 * 512 + 9 * 256, (dim, most)
        lib.lib.br_kv_free(lib.ctx)


SCENARIOS = [a_workspace_holds_the_pieces_of_what_is_launched, as_many_workers_as_a_launch_has_blocks_for, lists_as_long_as_their_places_can_be_counted]


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
    sys.path.insert(0, ROOT)
    next(f for f in SCENARIOS if f.__name__ == sys.argv[2])(Library(sys.argv[1]))
