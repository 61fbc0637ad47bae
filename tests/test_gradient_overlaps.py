"""Which tensors vsd_clip_gradients takes for overlapping, against the sets of their
bytes; every call here is refused, for its workspace if for nothing else."""
import ctypes
import os
import random

import pytest

from paper_2602_05774_amd import _lib

A = 0x10000  # a stand-in address; never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libvsd.so not built (run __graft_entry__.build())")
    return _lib.load()


def _table(items):
    return (_lib.VsdTensor * len(items))(*[_lib.VsdTensor(*i) for i in items])


def _overlap(lib, grads, out=None):
    """3 (they overlap): True, 7 (all that is missing is the workspace): False."""
    code = lib.vsd_clip_gradients(_table(grads), None if out is None else _table(out), len(grads), 1.0, None, None, None,
                                  None, 0, None)
    assert code in (3, 7), lib.vsd_last_error().decode()
    return code == 3


def _bytes(t):
    at, rows, cols, ld, dtype = t
    es = 2 if dtype else 4
    return {at + es * (r * (ld if rows > 1 else 0)) + k for r in range(rows) for k in range(es * cols)}


def _random(rng, span):
    dtype, rows, cols = rng.randint(0, 1), rng.choice((0, 1, 1, 2, 3, 7, 20)), rng.choice((0, 1, 2, 3, 5, 9, 30))
    ld = cols + rng.choice((0, 1, 2, 5, 17, 40))
    return (A + 4 * rng.randrange(span), rows, cols, max(ld, 1), dtype)


@pytest.mark.parametrize("seed", range(4))
def test_two_in_place(lib, seed):
    rng = random.Random(seed)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        pair = [_random(rng, 400), _random(rng, 400)]
        want = bool(_bytes(pair[0]) & _bytes(pair[1]))
        assert _overlap(lib, pair) == want, pair
        seen[want] += 1
    assert min(seen.values()) > 200  # both kinds of pairs are met


def test_out_of_place(lib):
    rng = random.Random(9)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        grads = [_random(rng, 300) for _ in range(2)]
        out = [(A + 4 * rng.randrange(600), rows, cols, cols + rng.choice((1, 3, 50)), rng.randint(0, 1)) for _, rows, cols, _, _ in grads]
        if any(o[0] == g[0] for o, g in zip(out, grads)):
            continue  # (in place, or refused for its type or stride)
        reads, writes = [_bytes(g) for g in grads], [_bytes(o) for o in out]
        want = bool(writes[0] & writes[1]) or any(w & r for w in writes for r in reads)
        assert _overlap(lib, grads, out) == want, (grads, out)
        seen[want] += 1
    assert min(seen.values()) > 200  # both kinds of pairs are met


def test_pieces_in_the_gaps_of_rows(lib):
    rows = (A, 1000, 60, 100, 0)              # 240 bytes of every 400
    assert not _overlap(lib, [rows, (A + 240, 1, 40, 40, 0)])          # one row in a gap
    assert not _overlap(lib, [rows, (A + 400 * 999 + 240, 1, 40, 40, 0)])
    assert _overlap(lib, [rows, (A + 240, 1, 41, 41, 0)])              # an element too many
    assert not _overlap(lib, [rows, (A + 240, 500, 40, 200, 0)])       # rows of twice the stride
    assert _overlap(lib, [rows, (A + 240, 500, 40, 150, 0)])
    assert not _overlap(lib, [rows, (A + 240, 400, 80, 200, 1)])       # of another type
    # far apart in size: strides of 2^40 elements
    far = (A, 1 << 4, 3, 1 << 40, 0)
    assert not _overlap(lib, [far, (A + 12, 1 << 30, 1, 2, 0)])
    assert _overlap(lib, [far, (A + 12, 1 << 30, 1, 3, 0), (A + (4 << 40) + 8, 1, 1, 1, 0)])
    # every one of many rows tried: 2^20 rows of stride 1009 against 1013, in gaps that meet once
    n = 1 << 20
    assert _overlap(lib, [(A, n, 1, 1009, 0), (A + 4, n, 1, 1013, 0)])
    hit = next(i for i in range(n) if (1009 * i - 1) % 1013 == 0)
    assert not _overlap(lib, [(A, hit, 1, 1009, 0), (A + 4, n, 1, 1013, 0)])
    assert _overlap(lib, [(A, hit + 1, 1, 1009, 0), (A + 4, n, 1, 1013, 0)])


def test_words_in_tensors(lib):
    """The given norm in what is written, what is returned in any tensor."""
    rows, flat = (A, 10, 60, 100, 0), (A + 8000, 1, 100, 100, 1)
    to = [(A + 10000, 10, 60, 60, 0), (A + 20000, 1, 100, 100, 1)]
    ws = A + (1 << 20)

    def refused(norm=None, norm_out=None, scale=None, out=None):
        code = lib.vsd_clip_gradients(_table([rows, flat]), None if out is None else _table(out), 2, 1.0, norm, norm_out,
                                      scale, ws, 1 << 30, None)
        return code == 3 and " lies in tensor " in lib.vsd_last_error().decode()

    inside = (A, A + 236, A + 400 * 9 + 8, A + 8000, A + 8198)
    assert all(refused(norm=at) for at in inside) and all(refused(norm_out=at) for at in inside)
    assert all(refused(scale=at) for at in inside) and all(refused(scale=at, out=to) for at in inside)
    assert all(refused(norm=at, out=to) for at in (A + 10000, A + 12396, A + 20000))
