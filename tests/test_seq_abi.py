"""The C ABI of the operators over sequences (include/luna_seq.h) and its Python binding without a
GPU: exports, refusals with their status codes before anything is enqueued, workspace sizes."""
import ctypes

import pytest

from paper_2512_08061_amd import luna

FAKE = 0x10000  # non-null, aligned; validation never dereferences it
INV, UNS, WS = luna.LUNA_ERR_INVALID_ARG, luna.LUNA_ERR_UNSUPPORTED, luna.LUNA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return luna.load_library()


def test_exports(lib):
    names = luna.header_functions(luna.SEQ_HEADER)
    assert names == ["luna_decay_bwd", "luna_decay_fwd", "luna_decay_step", "luna_seq_workspace_bytes", "luna_softmax_bwd",
                     "luna_softmax_fwd"]
    assert all(hasattr(lib, n) for n in names)


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def ref(a):
    return None if a is None else ctypes.addressof(a)


class Call:
    """Arguments that a call accepts, one of which a test replaces."""

    def __init__(self, **kw):
        self.H, self.Hk, self.D, self.d, self.n, self.B, self.dt = 4, 2, 64, 64, 100, 2, luna.LUNA_BF16
        self.norm, self.scale, self.eps, self.ws, self.wsn = 1, 1.0, 1e-6, FAKE, 1 << 40
        self.S = self.z = self.den = self.g = self.lse = FAKE
        self.off = self.lens = 0
        self.keys = None
        self.rows = {}
        self.m = 1
        self.__dict__.update(kw)

    def row(self, name, width, heads):
        h = heads * width
        return i64(*self.rows.get(name, (FAKE, self.n * h, self.n * width, width)))

    def seqs(self):
        return i64(self.B, self.n, self.off, self.lens)

    def keep(self, *a):
        self.kept = a  # (alive during the call)
        return [ref(x) for x in a]

    def decay_fwd(self, lib):
        r = self.keep(*(self.row(n, w, self.H) for n, w in (("Q", self.D), ("K", self.D), ("V", self.d), ("out", self.d))),
                      self.seqs())
        return lib.luna_decay_fwd(r[0], r[1], r[2], self.dt, r[4], self.H, self.D, self.d, self.g, self.norm, self.scale,
                                  self.eps, self.S, self.z, r[3], self.den, self.ws, self.wsn, None)

    def decay_step(self, lib):
        r = self.keep(*(self.row(n, w, self.H) for n, w in (("Q", self.D), ("K", self.D), ("V", self.d), ("out", self.d))))
        return lib.luna_decay_step(r[0], r[1], r[2], self.dt, self.B, self.m, self.H, self.D, self.d, self.g, self.norm,
                                   self.scale, self.eps, self.S, self.z, r[3], None)

    def decay_bwd(self, lib):
        r = self.keep(*(self.row(n, w, self.H) for n, w in (("Q", self.D), ("K", self.D), ("V", self.d), ("dO", self.d),
                                                           ("out", self.d), ("dQ", self.D), ("dK", self.D), ("dV", self.d))),
                      self.seqs())
        return lib.luna_decay_bwd(r[0], r[1], r[2], r[3], self.dt, r[8], self.H, self.D, self.d, self.g, self.norm, self.scale,
                                  self.eps, r[4], self.den, r[5], r[6], r[7], self.ws, self.wsn, None)

    def softmax_fwd(self, lib):
        r = self.keep(self.row("Q", self.d, self.H), self.row("K", self.d, self.Hk), self.row("V", self.d, self.Hk),
                      self.row("out", self.d, self.H), self.seqs(), self.keys)
        return lib.luna_softmax_fwd(r[0], r[1], r[2], self.dt, r[4], r[5], self.H, self.Hk, self.d, self.scale, r[3], self.lse,
                                    self.ws, self.wsn, None)

    def softmax_bwd(self, lib):
        r = self.keep(*(self.row(n, self.d, self.H) for n in ("Q", "out", "dO", "dQ")),
                      *(self.row(n, self.d, self.Hk) for n in ("K", "V", "dK", "dV")), self.seqs(), self.keys)
        return lib.luna_softmax_bwd(r[0], r[4], r[5], r[1], self.lse, r[2], self.dt, r[8], r[9], self.H, self.Hk, self.d,
                                    self.scale, r[3], r[6], r[7], self.ws, self.wsn, None)


NAN = float("nan")
COMMON = [(dict(H=0), INV), (dict(dt=7), INV), (dict(scale=NAN), INV), (dict(B=0), INV), (dict(n=-1), INV),
          (dict(n=(1 << 30) + 64), UNS), (dict(B=65536), UNS), (dict(H=65536, Hk=1, B=1, n=1), UNS)]
SEQS = [(dict(off=FAKE, lens=FAKE), INV)]
ROWS = [(lambda w, h: (0, w * h, w, w), INV), (lambda w, h: (FAKE + 8, 100 * w * h, 100 * w, w), INV),
        (lambda w, h: (FAKE, 100 * w * h, 100 * w, w - 8), INV), (lambda w, h: (FAKE, 100 * w * h, 100 * w, w + 4), INV),
        (lambda w, h: (FAKE, 100 * w * h, -100 * w, w), INV), (lambda w, h: (FAKE, 100 * w * h, 100 * w, (1 << 20) + 8), UNS)]
OUTPUT = [(lambda w, h: (FAKE, 100 * w * h, 0, w), INV), (lambda w, h: (FAKE, 0, 100 * w, w), INV)]
DECAY = [(dict(D=48), UNS), (dict(d=256), UNS), (dict(D=512), UNS), (dict(g=0), INV), (dict(norm=2), INV), (dict(eps=-1.0), INV),
         (dict(eps=NAN), INV)]


def refused(lib, op, want, **kw):
    assert getattr(Call(**kw), op)(lib) == want, (op, kw)
    assert lib.luna_last_error()


@pytest.mark.parametrize("op", ["decay_fwd", "decay_step", "decay_bwd", "softmax_fwd", "softmax_bwd"])
def test_refuses_sizes(lib, op):
    for kw, want in COMMON:
        if op == "decay_step" and "n" in kw and kw.get("H") is None:
            kw = {"m": kw["n"]}
        refused(lib, op, want, **kw)
    if op != "decay_step":
        for kw, want in SEQS:
            refused(lib, op, want, **kw)


@pytest.mark.parametrize("op,names", [
    ("decay_fwd", ("Q", "K", "V", "out")), ("decay_step", ("Q", "K", "V", "out")),
    ("decay_bwd", ("Q", "K", "V", "dO", "out", "dQ", "dK", "dV")), ("softmax_fwd", ("Q", "K", "V", "out")),
    ("softmax_bwd", ("Q", "K", "V", "out", "dO", "dQ", "dK", "dV"))])
def test_refuses_rows(lib, op, names):
    outputs = ("out",) if op in ("decay_fwd", "decay_step", "softmax_fwd") else ("dQ", "dK", "dV")
    for name in names:
        for make, want in ROWS + (OUTPUT if name in outputs else []):
            refused(lib, op, want, rows={name: make(64, 4)})
            assert name.encode() in lib.luna_last_error()


def test_refuses_decay_arguments(lib):
    for op in ("decay_fwd", "decay_step", "decay_bwd"):
        for kw, want in DECAY:
            refused(lib, op, want, **kw)
    for op in ("decay_fwd", "decay_step"):
        refused(lib, op, INV, S=FAKE + 4)
        refused(lib, op, INV, z=0)  # a normalised state needs both
        refused(lib, op, INV, norm=0, den=0)  # and a plain one has no z
    refused(lib, "decay_fwd", INV, norm=0, z=0)  # den without normalize
    refused(lib, "decay_step", INV, S=0, z=0)
    refused(lib, "decay_step", INV, m=0)
    refused(lib, "decay_step", UNS, B=65535, H=60)
    refused(lib, "decay_bwd", INV, den=0)
    # pieces of long sequences, and the backward pass's row weights, need a workspace
    big = dict(n=20000, S=0, z=0)
    for op in ("decay_fwd", "decay_bwd"):
        refused(lib, op, WS, wsn=256, **big)
        refused(lib, op, INV, ws=FAKE + 16, **big)
        refused(lib, op, INV, ws=0, **big)


def test_refuses_softmax_arguments(lib):
    for op in ("softmax_fwd", "softmax_bwd"):
        refused(lib, op, UNS, d=48)
        refused(lib, op, UNS, d=256)
        refused(lib, op, INV, H=4, Hk=3)
        refused(lib, op, INV, Hk=0)
        refused(lib, op, INV, keys=i64(3, 100, 0, 0))
        refused(lib, op, INV, keys=i64(2, 100, FAKE, FAKE))
        refused(lib, op, INV, keys=i64(2, -1, 0, 0))
    refused(lib, "softmax_bwd", INV, lse=0)
    refused(lib, "softmax_bwd", WS, wsn=16)
    refused(lib, "softmax_bwd", INV, ws=FAKE + 4)


def ws_bytes(lib, op, seqs, H=16, Hk=16, Dq=128, Dv=128, keys=None, dt=luna.LUNA_BF16):
    return lib.luna_seq_workspace_bytes(op, dt, ref(seqs), ref(keys), H, Hk, Dq, Dv)


def test_workspace_sizes(lib):
    # one short sequence per workgroup needs none; long ones a state per piece and head
    assert ws_bytes(lib, luna.OP_DECAY_FWD, i64(64, 64, 0, 0)) == 0
    nb = ws_bytes(lib, luna.OP_DECAY_FWD, i64(1, 16384, 0, 0))
    assert 16 * (128 * 128 + 128) * 4 <= nb <= 16 * 256 * (128 * 128 + 128) * 4 and nb % 256 == 0
    rows = i64(2, 2048, 0, 0)
    assert ws_bytes(lib, luna.OP_DECAY_BWD, rows) >= 2 * 2 * 2048 * 16 * 4
    assert ws_bytes(lib, luna.OP_SOFTMAX_BWD, rows) >= 2 * 2048 * 16 * 4
    packed = i64(7, 5000, FAKE, 0)
    assert ws_bytes(lib, luna.OP_DECAY_FWD, packed) > 0
    for op, kw in [(9, {}), (luna.OP_DECAY_FWD, dict(Dq=48)), (luna.OP_DECAY_FWD, dict(dt=5)), (luna.OP_SOFTMAX_BWD, dict(Hk=3)),
                   (luna.OP_SOFTMAX_BWD, dict(Dv=64))]:
        assert ws_bytes(lib, op, rows, **kw) == 0 and lib.luna_last_error()
    assert ws_bytes(lib, luna.OP_DECAY_FWD, None) == 0


def test_binding_refuses(lib):
    """Shapes, types, devices and forms that do not go together, before the C call (CPU tensors are refused too)."""
    import torch

    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    off = torch.tensor([0, 10], dtype=torch.int32)
    g = torch.zeros(2)
    S = t(1, 2, 32, 32, dt=torch.float32)
    q4, q3 = t(1, 2, 10, 32), t(10, 2, 32)

    def bad(f, *a, **k):
        with pytest.raises(luna.LunaError) as e:
            f(*a, **k)
        assert e.value.status == INV

    for f in (lambda q, **k: luna.decay_attn(q, q, q, g, **k), lambda q, **k: luna.softmax_attn(q, q, q, **k),
              lambda q, **k: luna.decay_attn_bwd(q, q, q, q, g, **k),
              lambda q, **k: luna.softmax_attn_bwd(q, q, q, q, t(1, 2, 10, dt=torch.float32), q, **k)):
        bad(f, q4)  # not on a GPU
        bad(f, q3)  # packed without offsets
        bad(f, q4, offsets=off)
        bad(f, q3, offsets=off, lens=off)
        bad(f, q3, offsets=off.long())
        bad(f, q3, offsets=off[None])
        bad(f, q3, offsets=off[:0])
        bad(f, q4, lens=off)  # two lengths for one sequence
        bad(f, t(10, 32))
    bad(luna.decay_attn_step, q3, q3, q3, g, S)
    bad(luna.decay_attn_step, q4, q4, q4, g, S)
