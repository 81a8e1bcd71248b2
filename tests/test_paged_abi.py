"""The C ABI of attention over pages (include/luna_paged.h) and its Python binding without a GPU: exports, refusals with their status
codes before anything is enqueued, workspace sizes, the shares of the cache and the pages that a table may name, wait
states of the compiled kernels."""
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
    names = luna.header_functions(luna.PAGED_HEADER)
    assert names == ["luna_paged_append", "luna_paged_fwd", "luna_paged_workspace_bytes"]
    assert all(hasattr(lib, n) for n in names)


class Call:
    """Arguments that a call accepts, one of which a test replaces."""

    def __init__(self, **kw):
        self.H, self.Hk, self.d, self.n, self.B, self.dt = 4, 2, 64, 1, 2, luna.LUNA_BF16
        self.scale, self.ws, self.wsn, self.off, self.lens = 1.0, FAKE, 1 << 40, 0, 0
        self.pool, self.prows, self.width, self.table, self.plens = 50, 64, 10, FAKE, FAKE
        self.rot, self.freq, self.near, self.lse, self.pages = 64, FAKE, 0, FAKE, True
        self.rows, self.none = {}, ()
        self.__dict__.update(kw)

    def row(self, name):
        heads, n = (self.Hk, self.prows) if name.endswith("pages") else (self.Hk if name in ("K", "V") else self.H, self.n)
        return i64(*self.rows.get(name, (FAKE, n * heads * self.d, n * self.d, self.d)))

    def keep(self, *names):
        self.kept = [None if n in self.none else self.row(n) for n in names] + [i64(self.B, self.n, self.off, self.lens)]
        self.kept.append(i64(self.pool, self.prows, self.width, self.table, self.plens) if self.pages else None)
        return [ref(x) for x in self.kept]

    def append(self, lib):
        r = self.keep("K", "V", "Q", "k_pages", "v_pages", "q_out")
        return lib.luna_paged_append(r[0], r[1], r[2], self.dt, r[6], r[7], self.H, self.Hk, self.d, self.rot, self.freq, self.near, r[3],
                                     r[4], r[5], None)

    def fwd(self, lib):
        r = self.keep("Q", "k_pages", "v_pages", "out")
        return lib.luna_paged_fwd(r[0], r[1], r[2], self.dt, r[4], r[5], self.H, self.Hk, self.d, self.scale, r[3], self.lse, self.ws,
                                  self.wsn, None)


def refused(lib, op, want, **kw):
    assert getattr(Call(**kw), op)(lib) == want, (op, kw)
    assert lib.luna_last_error()


@pytest.mark.parametrize("op", ["append", "fwd"])
def test_refuses_arguments(lib, op):
    for kw, want in [(dict(H=0), INV), (dict(Hk=0), INV), (dict(Hk=3), INV), (dict(dt=7), INV), (dict(B=0), INV), (dict(n=-1), INV),
                     (dict(B=65536), UNS), (dict(n=(1 << 30) + 64), UNS), (dict(H=65536, Hk=1, B=1), UNS), (dict(d=48), UNS), (dict(d=256), UNS),
                     (dict(off=FAKE, lens=FAKE), INV), (dict(pages=False), INV), (dict(pool=0), INV), (dict(prows=0), INV),
                     (dict(width=0), INV), (dict(prows=8), UNS), (dict(prows=48), UNS), (dict(prows=1 << 17), UNS),
                     (dict(width=(1 << 24) + 1), UNS), (dict(pool=(1 << 31) + 1), UNS), (dict(table=0), INV), (dict(plens=0), INV)]:
        refused(lib, op, want, **kw)


def test_refuses_append_arguments(lib):
    for kw, want in [(dict(rot=-16), INV), (dict(rot=8), INV), (dict(rot=80), INV), (dict(rot=0), INV), (dict(freq=0), INV),
                     (dict(near=2), INV), (dict(none=("Q",)), INV), (dict(none=("q_out",)), INV), (dict(B=1, n=1 << 27), UNS)]:
        refused(lib, "append", want, **kw)


def test_refuses_attention_arguments(lib):
    refused(lib, "fwd", INV, scale=NAN)
    refused(lib, "fwd", WS, wsn=256)
    refused(lib, "fwd", INV, ws=FAKE + 16)
    refused(lib, "fwd", INV, ws=0)
    refused(lib, "fwd", UNS, B=65535, n=64, H=300, Hk=300)


@pytest.mark.parametrize("op,names,outputs", [("append", "K V Q k_pages v_pages q_out", "k_pages v_pages q_out"), ("fwd", "Q k_pages v_pages out", "out")])
def test_refuses_rows(lib, op, names, outputs):
    for name in names.split():
        for make, want in ROWS + (OUTPUT if name in outputs.split() else []):
            refused(lib, op, want, rows={name: make(64, 4)})
            assert name.encode() in lib.luna_last_error()


def nb(lib, seqs, pages, H=16, Hk=4, d=128, dt=luna.LUNA_BF16):
    return lib.luna_paged_workspace_bytes(dt, ref(seqs), ref(pages), H, Hk, d)


def test_workspace_sizes(lib):
    pages = i64(5000, 64, 128, FAKE, FAKE)
    part = 4 * (128 + 2) * 4  # a key head's rows
    got = nb(lib, i64(32, 1, 0, 0), pages)
    assert 4 * part * (32 + 1) <= got <= 4 * part * (32 + 1024) and got % 256 == 0
    assert nb(lib, i64(32, 512, 0, 0), pages) == 0 and not lib.luna_last_error()  # tiles
    assert nb(lib, i64(32, 40, FAKE, 0), pages) == 0 and not lib.luna_last_error()
    # it does not grow with the room for keys, only with the sequences
    assert nb(lib, i64(32, 1, 0, 0), i64(5000, 64, 1 << 20, FAKE, FAKE)) == got
    for kw in (dict(d=48), dict(dt=5), dict(Hk=3)):
        assert nb(lib, i64(2, 1, 0, 0), pages, **kw) == 0 and lib.luna_last_error()
    assert nb(lib, None, pages) == 0 and nb(lib, i64(2, 1, 0, 0), None) == 0


SHARES = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "luna_seq.hpp"
int main() {
  srand(2);
  for (int trial = 0; trial < 20000; ++trial) {
    const int count = 1 + rand() % 40, shares = 1 + rand() % (rand() % 2 ? 8 : 200), kind = rand() % 4;
    std::vector<int> units(count);
    std::vector<int64_t> before(count + 1, 0);
    for (int b = 0; b < count; ++b) {
      units[b] = rand() % 3 == 0 ? 0 : kind == 0 ? rand() % 4 : kind == 1 ? rand() % 300 : kind == 2 ? (rand() % 20 ? 1 : 5000) : 4 * (rand() % 9);
      before[b + 1] = before[b] + units[b];
    }
    const int64_t all = before[count], per = luna::paged_per(all, shares);
    if (per * shares < all) return printf("units left over\n"), 1;
    std::vector<int> owner(shares + count, -1);
    for (int b = 0; b < count; ++b) {
      const luna::PagedUnits h = luna::paged_holders(before[b], units[b], per);
      if (units[b] == 0 ? h.u1 >= h.u0 : h.u1 < h.u0 || h.u0 < 0 || h.u1 >= shares) return printf("trial %d: holders of %d\n", trial, b), 1;
      int seen = 0;
      for (int s = 0; s < shares; ++s) {
        if (s * per >= all) break;
        const luna::PagedUnits u = luna::paged_held(before[b], units[b], per, s, all);
        if (u.u0 >= u.u1) continue;
        if (u.u0 != seen || u.u1 > units[b] || s < h.u0 || s > h.u1) return printf("trial %d: share %d of %d\n", trial, s, b), 1;
        seen = u.u1;
        const int64_t part = luna::paged_part(s, b);
        if (part < 0 || part >= shares + count || owner[part] >= 0) return printf("trial %d: part %ld\n", trial, (long)part), 1;
        owner[part] = b;
      }
      if (seen != units[b]) return printf("trial %d: sequence %d: %d of %d units\n", trial, b, seen, units[b]), 1;
    }
  }
  const int32_t table[6] = {0, 6, 7, -1, 2147483647, -2147483647 - 1};
  const luna::PageSet p{table, 7, 3, 4};
  const int want[6] = {0, 6, -1, -1, -1, -1};
  for (int i = 0; i < 6; ++i)
    for (int row = 0; row < 16; ++row)
      if (luna::page_of(p, i / 3, i % 3 * 16 + row) != want[i]) return printf("page %d\n", i), 1;
  return 0;
}
"""


def test_shares_and_pages_on_the_host(tmp_path):
    """Each unit of the cache in one share, parts apart and within the workspace, the join's shares those that hold the sequence;
    table entries outside of the pool are no pages."""
    src, exe = tmp_path / "shares.cpp", tmp_path / "shares"
    src.write_text(SHARES)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["/opt/rocm/bin/hipcc", "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2512_08061_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True, capture_output=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout


def test_binding_refuses():
    """Shapes, types, devices and forms that do not go together, before the C call (CPU tensors are refused too)."""
    import torch

    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q4, q3, pages = t(1, 2, 10, 32), t(10, 2, 32), t(5, 2, 16, 32)

    def bad(f, *a, **k):
        with pytest.raises(luna.LunaError) as e:
            f(*a, **k)
        assert e.value.status == INV

    for f in (lambda q, p=pages, tb=i(1, 3), ln=i(1), **k: luna.paged_append(q, q, p, p, tb, ln, **k),
              lambda q, p=pages, tb=i(1, 3), ln=i(1), **k: luna.paged_attn(q, p, p, tb, ln, **k)):
        bad(f, q4)  # not on a GPU
        bad(f, q3)  # packed without offsets
        bad(f, q4, offsets=i(2))
        bad(f, t(10, 32))
        bad(f, q4, t(5, 2, 16))
        bad(f, q4, t(5, 2, 16, 32, dt=torch.float32))
        bad(f, q4, tb=i(2, 3))
        bad(f, q4, tb=i(3))
        bad(f, q4, ln=i(2))
        bad(f, q4, ln=i(1).long())
    bad(luna.paged_append, q4, q4, pages, pages, i(1, 3), i(1), q_out=q4)


SOURCES = ["luna_paged_tiles.hip", "luna_paged_split.hip"]


def test_results_of_matrix_products_are_waited_for(tmp_path):
    with cf.ThreadPoolExecutor(4) as pool:
        texts = list(pool.map(lambda s: assembly(s, str(tmp_path / (s + ".s"))), SOURCES))
    found = [f"{s} {name}: {a} -> {b}: {n}" for s, text in zip(SOURCES, texts) for name, blocks in kernels(text)
             for a, b, n in early(blocks)]
    assert not found, "\n".join(found)
