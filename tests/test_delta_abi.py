"""The C ABI of the gated delta rule (include/luna_delta.h) and its Python binding without a GPU: exports, refusals with their
status codes before anything is enqueued, workspace sizes, wait states of the compiled kernels."""
import concurrent.futures as cf
import ctypes
import os
import subprocess

import pytest

from paper_2512_08061_amd import luna
from test_matrix_waits import assembly, early, kernels
from test_seq_abi import FAKE, INV, NAN, OUTPUT, ROWS, UNS, WS, i64, ref


@pytest.fixture(scope="module")
def lib():
    return luna.load_library()


def test_exports(lib):
    names = luna.header_functions(luna.DELTA_HEADER)
    assert names == ["luna_delta_bwd", "luna_delta_fwd", "luna_delta_step", "luna_delta_workspace_bytes"]
    assert all(hasattr(lib, n) for n in names)


class Call:
    """Arguments that a call accepts, one of which a test replaces."""

    def __init__(self, **kw):
        self.H, self.Hk, self.D, self.d, self.n, self.B, self.dt = 4, 2, 64, 64, 100, 2, luna.LUNA_BF16
        self.scale, self.ws, self.wsn, self.m, self.off, self.lens = 1.0, FAKE, 1 << 40, 1, 0, 0
        self.S = self.g = self.beta = self.dg = self.db = FAKE
        self.rows = {}
        self.__dict__.update(kw)

    def row(self, name):
        heads, width = (self.Hk, self.D) if name in ("Q", "K", "dQ", "dK") else (self.H, self.d)
        return i64(*self.rows.get(name, (FAKE, self.n * heads * width, self.n * width, width)))

    def keep(self, *names):
        self.kept = [self.row(n) for n in names] + [i64(self.B, self.n, self.off, self.lens)]
        return [ref(x) for x in self.kept]

    def fwd(self, lib):
        r = self.keep("Q", "K", "V", "out")
        return lib.luna_delta_fwd(r[0], r[1], r[2], self.dt, r[4], self.H, self.Hk, self.D, self.d, self.g, self.beta, self.scale,
                                  self.S, r[3], self.ws, self.wsn, None)

    def step(self, lib):
        r = self.keep("Q", "K", "V", "out")
        return lib.luna_delta_step(r[0], r[1], r[2], self.dt, self.B, self.m, self.H, self.Hk, self.D, self.d, self.g, self.beta,
                                   self.scale, self.S, r[3], None)

    def bwd(self, lib):
        r = self.keep("Q", "K", "V", "dO", "dQ", "dK", "dV")
        return lib.luna_delta_bwd(r[0], r[1], r[2], r[3], self.dt, r[7], self.H, self.Hk, self.D, self.d, self.g, self.beta,
                                  self.scale, r[4], r[5], r[6], self.dg, self.db, self.ws, self.wsn, None)


def refused(lib, op, want, **kw):
    assert getattr(Call(**kw), op)(lib) == want, (op, kw)
    assert lib.luna_last_error()


@pytest.mark.parametrize("op", ["fwd", "step", "bwd"])
def test_refuses_arguments(lib, op):
    for kw, want in [(dict(H=0), INV), (dict(Hk=0), INV), (dict(Hk=3), INV), (dict(dt=7), INV), (dict(scale=NAN), INV), (dict(B=0), INV),
                     (dict(B=65536), UNS), (dict(H=65536, Hk=1, B=1), UNS), (dict(D=48), UNS), (dict(D=256), UNS), (dict(d=256), UNS),
                     (dict(d=0), INV), (dict(g=0), INV), (dict(beta=0), INV)]:
        refused(lib, op, want, **kw)
    if op != "bwd":
        refused(lib, op, INV, S=FAKE + 4)
    if op == "step":
        refused(lib, op, INV, S=0)
        refused(lib, op, INV, m=0)
        refused(lib, op, UNS, m=(1 << 30) + 1)
        refused(lib, op, UNS, B=65535, H=60, Hk=1)
    else:
        refused(lib, op, INV, n=-1)
        refused(lib, op, UNS, n=(1 << 30) + 64)
        refused(lib, op, INV, off=FAKE, lens=FAKE)
        refused(lib, op, WS, wsn=256, dt=luna.LUNA_F32)
        refused(lib, op, INV, ws=FAKE + 16, dt=luna.LUNA_F32)
        refused(lib, op, INV, ws=0, dt=luna.LUNA_F32)
    if op == "bwd":
        refused(lib, op, INV, dg=0)
        refused(lib, op, INV, db=0)


@pytest.mark.parametrize("op,names,outputs", [("fwd", "Q K V out", "out"), ("step", "Q K V out", "out"), ("bwd", "Q K V dO dQ dK dV", "dQ dK dV")])
def test_refuses_rows(lib, op, names, outputs):
    for name in names.split():
        for make, want in ROWS + (OUTPUT if name in outputs.split() else []):
            refused(lib, op, want, rows={name: make(64, 4)})
            assert name.encode() in lib.luna_last_error()


def test_workspace_sizes(lib):
    def nb(op, seqs, H=16, Hk=16, D=128, d=128, dt=luna.LUNA_F32):
        return lib.luna_delta_workspace_bytes(op, dt, ref(seqs), H, Hk, D, d)

    chunk = 64 * 64 * 4
    for op, least in ((luna.OP_DELTA_FWD, 2 * chunk), (luna.OP_DELTA_BWD, 2 * chunk + 2 * 128 * 128 * 4 + 2 * 64 * 128 * 4)):
        one = nb(op, i64(1, 64, 0, 0), H=1, Hk=1)
        assert one >= least and one % 256 == 0
        assert nb(op, i64(2, 2048, 0, 0)) >= 2 * 32 * 16 * least
        assert nb(op, i64(7, 5000, FAKE, 0)) >= 7 * 16 * least
        assert (nb(op, i64(2, 2048, 0, 0), dt=luna.LUNA_BF16) > 0) == (op == luna.OP_DELTA_BWD) and not lib.luna_last_error()
        for kw in (dict(D=48), dict(dt=5), dict(Hk=3)):
            assert nb(op, i64(2, 64, 0, 0), **kw) == 0 and lib.luna_last_error()
    assert nb(9, i64(1, 64, 0, 0)) == 0 and nb(0, None) == 0
    # 2^31 chunks, and launches of 2^32 threads
    assert nb(0, i64(1, 1 << 30, 0, 0), H=1, Hk=1) == 0 and b"too many" in lib.luna_last_error()
    assert nb(0, i64(65535, 16384, 0, 0), H=64, Hk=64) == 0 and b"too many" in lib.luna_last_error()


RULES = r"""
#include <cstdio>
#include "luna_delta.hpp"
int main() {
  for (int64_t chunks = 1; chunks <= 3000; ++chunks)
    for (int64_t group = 1; group <= 40; ++group) {
      int64_t together = 0, apart = 0;  // turns of 256 workgroups
      for (int64_t left = chunks; left > 0; left -= 256) together += group;
      for (int64_t left = chunks * group; left > 0; left -= 256) ++apart;
      if (luna::delta_grads_apart(chunks, group) != (apart <= together - (together + 3) / 4))
        return printf("%ld chunks, groups of %ld\n", (long)chunks, (long)group), 1;
    }
  return luna::delta_grads_apart((int64_t)1 << 20, 4) || luna::delta_grads_apart((int64_t)1 << 31, 65535);
}
"""


def host_program(tmp_path, text):
    src, exe = tmp_path / "rules.cpp", tmp_path / "rules"
    src.write_text(text)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["/opt/rocm/bin/hipcc", "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2512_08061_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True, capture_output=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout


WIDTH = r"""
#include "luna_delta.hpp"
int main() {
  for (int64_t groups = 1; groups <= 2000; ++groups)
    for (int64_t D = 32; D <= 128; D *= 2)
      for (int equal = 0; equal < 2; ++equal)
        if (!luna::delta_narrow(D, 32, groups, equal) || luna::delta_narrow(D, 128, groups, equal) != (groups <= (D < 128 && !equal ? 512 : 256)))
          return 1;
  return 0;
}
"""


def test_serial_passes_are_narrow_where_they_run_at_once(tmp_path):
    """32 columns a workgroup up to one for each of 256 compute units, or two where the lengths may differ."""
    host_program(tmp_path, WIDTH)


def test_value_heads_apart_where_a_quarter_of_the_turns_is_saved(tmp_path):
    host_program(tmp_path, RULES)


def test_workspace_sizes_are_those_of_the_header(lib):
    """Per chunk and value head, as luna_delta.h says."""
    for B, rows, off, chunks in ((8, 16384, 0, 8 * 256), (3, 65, 0, 6), (10000, 80000, FAKE, 11250), (1, 1, FAKE, 1)):
        for D, d in ((128, 128), (32, 64), (64, 32)):
            for op, dt, each in ((luna.OP_DELTA_BWD, luna.LUNA_BF16, 8 * D * d + 512 * d + 50688),
                                 (luna.OP_DELTA_BWD, luna.LUNA_F32, 8 * D * d + 512 * d + 34304), (luna.OP_DELTA_FWD, luna.LUNA_F32, 34304),
                                 (luna.OP_DELTA_FWD, luna.LUNA_BF16, 0)):
                assert lib.luna_delta_workspace_bytes(op, dt, ref(i64(B, rows, off, 0)), 16, 4, D, d) == chunks * 16 * each, (B, D, d, op)


def test_binding_refuses():
    """Shapes, types, devices and forms that do not go together, before the C call (CPU tensors are refused too)."""
    import torch

    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    off, q4, q3 = torch.tensor([0, 10], dtype=torch.int32), t(1, 2, 10, 32), t(10, 2, 32)
    g, S = t(1, 2, 10, dt=torch.float32), t(1, 2, 32, 32, dt=torch.float32)

    def bad(f, *a, **k):
        with pytest.raises(luna.LunaError) as e:
            f(*a, **k)
        assert e.value.status == INV

    for f in (lambda q, **k: luna.delta_attn(q, q, q, g, g, **k), lambda q, **k: luna.delta_attn_bwd(q, q, q, q, g, g, **k)):
        bad(f, q4)  # not on a GPU
        bad(f, q3)  # packed without offsets
        bad(f, q4, offsets=off)
        bad(f, q3, offsets=off, lens=off)
        bad(f, q3, offsets=off.long())
        bad(f, q4, lens=off)
        bad(f, t(10, 32))
    bad(luna.delta_attn_step, q3, q3, q3, g, g, S)
    bad(luna.delta_attn_step, q4, q4, q4, g, g, S)


SOURCES = ["luna_delta_gates.hip", "luna_delta_fwd.hip", "luna_delta_bf16.hip", "luna_delta_f32.hip", "luna_delta_grads.hip"]


def test_results_of_matrix_products_are_waited_for(tmp_path):
    with cf.ThreadPoolExecutor(4) as pool:
        texts = list(pool.map(lambda s: assembly(s, str(tmp_path / (s + ".s"))), SOURCES))
    found = [f"{s} {name}: {a} -> {b}: {n}" for s, text in zip(SOURCES, texts) for name, blocks in kernels(text)
             for a, b, n in early(blocks)]
    assert not found, "\n".join(found)
