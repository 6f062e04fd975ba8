"""The order in which a gather copies sequences, without a GPU.

A thread of the gather kernel takes the operations in batches of eight: it
loads a batch's sources, then stores its destinations, then goes on.  The
plans are executed that way here on a list that stands for the sequences.
"""
import ctypes as C
import itertools
import random

import numpy as np
import pytest

from paper_2609_04263_amd import configs

from test_host_abi import FAKE, FakeStorage, kvq  # noqa: F401  (kvq: the fixture)

BATCH = 8


def plan(kvq, rows, n_src, in_place):
    n = len(rows)
    r = (C.c_int32 * n)(*rows)
    pairs = (C.c_int32 * (2 * (3 * n + 2 * BATCH)))()
    dep = C.c_int(-1)
    count = kvq.lib().kvq_internal_gather_ops(r, n, n_src, int(in_place), pairs, C.byref(dep))
    assert 0 <= count <= 3 * n + 2 * BATCH and count % BATCH == 0
    ops = np.array(pairs[:2 * count]).reshape(-1, BATCH, 2)
    return ops, bool(dep.value)


def execute(ops, src, dst):
    for batch in ops:
        loaded = [src[s] if d >= 0 else None for s, d in batch]
        for v, (_, d) in zip(loaded, batch):
            if d >= 0:
                dst[d] = v


def check(kvq, rows, n_src, in_place, rng):
    ops, ordered = plan(kvq, rows, n_src, in_place)
    # a gap is only ever at the end of a batch (an operation may look at the one before it)
    for batch in ops:
        live = [d >= 0 for _, d in batch]
        assert live == sorted(live, reverse=True)
        assert all(0 <= s < n_src and d < len(rows) for s, d in batch)
    src = list(range(n_src))
    dst = src if in_place else [None] * len(rows)
    before = list(dst)
    ops = list(ops)
    if not ordered:
        rng.shuffle(ops)
    execute(ops, src, dst)
    assert dst == [before[b] if s < 0 else s for b, s in enumerate(rows)], rows
    moved = sum(s >= 0 and not (in_place and s == b) for b, s in enumerate(rows))
    assert in_place or sum(d >= 0 for batch in ops for _, d in batch) == moved
    return ordered


def test_every_small_map_in_place(kvq):
    rng = random.Random(1)
    for n in range(1, 6):
        for rows in itertools.product(range(-1, n), repeat=n):
            check(kvq, list(rows), n, True, rng)


@pytest.mark.parametrize("n", [2, 7, 8, 9, 15, 16, 17, 33, 100, 600])
def test_permutations_maps_and_mixtures_in_place(kvq, n):
    rng = random.Random(n)
    cycle = [(i + 1) % n for i in range(n)]
    assert check(kvq, cycle, n, True, rng)
    for _ in range(30):
        perm = rng.sample(range(n), n)
        check(kvq, perm, n, True, rng)
        check(kvq, [rng.randrange(-1, n) for _ in range(n)], n, True, rng)
        # a chain into a cycle, holes, fixed points
        mixed = [p if rng.random() < 0.7 else rng.choice([-1, i, rng.randrange(n)]) for i, p in enumerate(perm)]
        check(kvq, mixed, n, True, rng)


def test_a_beam_step_needs_no_order(kvq):
    # the ended beams take over another's cache, whose own stays: batches may run at once
    rows = list(range(32))
    for b, s in ((3, 1), (9, 1), (30, 2), (31, 4)):
        rows[b] = s
    ops, ordered = plan(kvq, rows, 32, True)
    assert not ordered and len(ops) == 1


@pytest.mark.parametrize("n_dst,n_src", [(1, 1), (4, 1), (5, 9), (9, 5), (64, 3), (300, 40)])
def test_between_caches(kvq, n_dst, n_src):
    rng = random.Random(n_dst)
    for _ in range(20):
        rows = [rng.randrange(-1, n_src) for _ in range(n_dst)]
        assert not check(kvq, rows, n_src, False, rng)
        ops, _ = plan(kvq, rows, n_src, False)
        sources = [s for batch in ops for s, d in batch if d >= 0]
        assert sources == sorted(sources)  # each source's copies are neighbours: it is loaded once per batch


def cache(kvq, f, B, H, D, T, n=0, addr=FAKE):
    c = kvq.Cache(f, B, H, D, T, storage=FakeStorage(kvq.cache_bytes(f, B, H, D, T), addr))
    c.restore(n)
    return c


def status(kvq, call):
    with pytest.raises(kvq.KvqError) as e:
        call()
    return e.value.status


def test_refusals_leave_both_caches_unchanged(kvq):
    f = configs.make_format()
    src = cache(kvq, f, 3, 2, 64, 100, n=90)
    far = FAKE + (1 << 30)
    dst = cache(kvq, f, 2, 2, 64, 80, n=7, addr=far)
    assert status(kvq, lambda: dst.gather(src, [0, 1], stream=0)) == kvq.ERR_CAPACITY   # 90 > 80 tokens
    assert status(kvq, lambda: dst.gather(src, [0, 3], n=8, stream=0)) == kvq.ERR_ARG   # no such sequence
    assert status(kvq, lambda: dst.gather(src, [0, -2], n=8, stream=0)) == kvq.ERR_ARG
    assert status(kvq, lambda: dst.gather(src, [0, 1 << 40], n=8, stream=0)) == kvq.ERR_ARG
    assert status(kvq, lambda: dst.gather(src, [0, 1], n=91, stream=0)) == kvq.ERR_ARG  # longer than the source
    assert status(kvq, lambda: dst.gather(src, [0, 1], n=-1, stream=0)) == kvq.ERR_ARG
    for bad in ([0], [0, 1, 2], [], [0.0, 1.0], [[0, 1]]):
        with pytest.raises(ValueError):
            dst.gather(src, bad, n=8, stream=0)
    for B, H, D in ((2, 3, 64), (2, 2, 128)):  # heads, head size
        assert status(kvq, lambda: cache(kvq, f, B, H, D, 100, addr=far).gather(src, [0, 1], stream=0)) == kvq.ERR_ARG
    other = cache(kvq, configs.make_format(2, 2), 2, 2, 64, 100, addr=far)
    assert status(kvq, lambda: other.gather(src, [0, 1], stream=0)) == kvq.ERR_FORMAT
    # storage that overlaps the source's, by a byte or wholly
    total = kvq.cache_bytes(f, 3, 2, 64, 100)
    for addr in (FAKE, FAKE + (total - 1) // 256 * 256):
        assert status(kvq, lambda: cache(kvq, f, 3, 2, 64, 100, addr=addr).gather(src, [0, 1, 2], n=8,
                                                                                  stream=0)) == kvq.ERR_ARG
    # a window only holds the newest tokens: no shorter copy
    w = configs.WORKLOADS["llama8b_kivi"].fmt
    ws, wd = cache(kvq, w, 2, 1, 128, 400, n=300), cache(kvq, w, 2, 1, 128, 400, addr=far)
    assert status(kvq, lambda: wd.gather(ws, [0, 1], n=299, stream=0)) == kvq.ERR_FORMAT
    assert status(kvq, lambda: ws.gather(ws, [1, 0], n=299, stream=0)) == kvq.ERR_FORMAT
    lib = kvq.lib()
    one = (C.c_int32 * 3)(0, 1, 2)
    for args in ((None, src.handle, one), (dst.handle, None, one), (dst.handle, src.handle, None)):
        assert lib.kvq_cache_gather(*args, 8, None) == kvq.ERR_ARG
    assert (src.n, dst.n, ws.n, wd.n) == (90, 7, 300, 0)


def test_nothing_to_copy_sets_the_length(kvq):
    f = configs.make_format()
    src, dst = cache(kvq, f, 3, 2, 64, 100, n=90), cache(kvq, f, 2, 2, 64, 80, n=7, addr=FAKE + (1 << 30))
    dst.gather(src, [0, 2], n=0, stream=0)       # no token: nothing is launched
    assert dst.n == 0
    dst.gather(src, [-1, -1], n=80, stream=0)    # no sequence
    assert dst.n == 80
    src.gather(src, [0, 1, 2], stream=0)         # every sequence its own
    assert src.n == 90
