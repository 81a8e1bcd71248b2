"""Which sizes the operators over sequences (include/luna_seq.h) take and how much workspace they ask for, without a GPU."""
import ctypes

import pytest

from paper_2512_08061_amd import luna

FAKE = 0x10000  # stands for offsets or lengths, which the host never reads
BF16, F32 = luna.LUNA_BF16, luna.LUNA_F32


def seqs(count, rows, offsets=False, lens=False):
    return (ctypes.c_int64 * 4)(count, rows, FAKE if offsets else 0, FAKE if lens else 0)


def workspace(op, q, keys=None, H=16, Hk=None, Dq=128, Dv=None, dt=BF16):
    """(bytes, error text) of an operation's query."""
    lib = luna.load_library()
    at = lambda a: None if a is None else ctypes.addressof(a)  # noqa: E731
    n = lib.luna_seq_workspace_bytes(op, dt, at(q), at(keys), H, Hk or H, Dq, Dv or Dq)
    return n, lib.luna_last_error().decode()


@pytest.mark.parametrize("count,rows,H,Hk,n", [(128, 65536, 64, 8, 1), (128, 32768, 128, 8, 1), (256, 16384, 128, 8, 1),
                                               (512, 32768, 32, 4, 1), (128, 65536, 64, 8, 8)])
def test_many_long_caches_are_taken(count, rows, H, Hk, n):
    """The next tokens over large caches: what is launched is a workgroup for 512 keys of a key head."""
    nb, why = workspace(luna.OP_SOFTMAX_FWD, seqs(count, n), seqs(count, rows, lens=True), H, Hk)
    assert nb == count * (rows // 512) * H * n * (128 + 2) * 4 and not why, why


@pytest.mark.parametrize("op,q,keys,H,Hk,d,dt", [
    # (a workgroup per 128 or 64 query rows of a head)
    (luna.OP_SOFTMAX_FWD, (1, 1 << 30, True), None, 1, 1, 64, BF16),
    (luna.OP_SOFTMAX_FWD, (1, 1 << 29, True), None, 1, 1, 32, BF16),
    (luna.OP_SOFTMAX_FWD, (1, 1 << 29, True), None, 1, 1, 128, F32),
    (luna.OP_SOFTMAX_FWD, (2048, 16384), None, 32, 4, 128, BF16),
    # (few queries: per 512 keys of a key head, and d threads per query row)
    (luna.OP_SOFTMAX_FWD, (65535, 1), (65535, 16384), 64, 8, 128, BF16),
    (luna.OP_SOFTMAX_FWD, (65535, 1), (65535, 512), 512, 8, 128, BF16),
    # (backward: query tiles of a head and key tiles of a key head; 512 threads for 128 keys)
    (luna.OP_SOFTMAX_BWD, (2048, 16384), None, 32, 4, 128, BF16),
    (luna.OP_SOFTMAX_BWD, (16, 64), (16, (1 << 26) - 128), 64, 1, 64, BF16)])
def test_sizes_whose_launches_fit_are_taken(op, q, keys, H, Hk, d, dt):
    _, why = workspace(op, seqs(*q), None if keys is None else seqs(*keys, lens=True), H, Hk, d, dt=dt)
    assert not why


@pytest.mark.parametrize("op,q,keys,H,Hk,d,dt", [
    (luna.OP_SOFTMAX_FWD, (1, 1 << 30, True), None, 2, 1, 64, BF16), (luna.OP_SOFTMAX_FWD, (1, 1 << 30, True), None, 1, 1, 32, BF16),
    (luna.OP_SOFTMAX_FWD, (1, 1 << 30, True), None, 1, 1, 64, F32),
    (luna.OP_SOFTMAX_FWD, (65535, 1), (65535, 16384), 128, 16, 128, BF16),
    (luna.OP_SOFTMAX_FWD, (65535, 64), (65535, 512), 9, 9, 128, BF16),
    (luna.OP_SOFTMAX_BWD, (1, 1 << 30, True), None, 2, 1, 64, BF16), (luna.OP_SOFTMAX_BWD, (1, 64), (1, 1 << 30), 2, 2, 64, BF16),
    (luna.OP_SOFTMAX_BWD, (16, 64), (16, 1 << 26), 64, 1, 64, BF16)])  # (2^23 workgroups of 512: 2^32)
def test_launches_of_too_many_threads_are_refused(op, q, keys, H, Hk, d, dt):
    nb, why = workspace(op, seqs(*q), None if keys is None else seqs(*keys, lens=True), H, Hk, d, dt=dt)
    assert nb == 0 and "too many" in why


@pytest.mark.parametrize("H,D,d,fits", [(128, 64, 64, True), (128, 128, 128, True), (129, 128, 128, False), (256, 64, 64, True),
                                        (128, 256, 64, True), (129, 256, 64, False)])
def test_many_short_sequences_of_the_decay_operators(H, D, d, fits):
    """A workgroup of 256 or 512 threads per sequence and head."""
    _, why = workspace(luna.OP_DECAY_FWD, seqs(65535, 4), H=H, Dq=D, Dv=d)
    assert ("too many" in why) != fits and bool(why) != fits
