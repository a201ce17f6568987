"""GPU parity of wedlm_cache_free, wedlm_cache_fork and wedlm_cache_compact
(include/wedlm_serve.h) with oracle/serve_oracle.py: all whole numbers, all
equal."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(x):
    return x.cpu().numpy()


def pool(rng, P, B, maxp, lens, spare=0):
    """A table whose rows own pages for their lengths and `spare` more."""
    bt = np.full((B, maxp), -1, np.int32)
    ids = rng.permutation(P)
    at = 0
    for b, n in enumerate(lens):
        m = min(maxp, -(-n // 16) + (spare if n else 0))
        bt[b, :m] = ids[at:at + m]
        at += m
    ref = np.bincount(bt[bt >= 0], minlength=P).astype(np.int32)
    plen = np.zeros(B, np.int32)
    plen[:len(lens)] = lens
    return bt, ref, plen


# pages of bytes, of 4-byte words and of 16-byte words, some not aligned
SHAPES = [(2, 3), (5,), (4, 16), (2, 16, 64), (3, 7, 4)]


def arrays(rng, L, P):
    return [rng.integers(0, 256, (L, P) + s).astype(np.uint8) for s in SHAPES]


def moved(arr, moves):
    arr = [a.copy() for a in arr]
    for a in arr:
        for s, d in moves:
            a[:, d] = a[:, s]
    return arr


def fork(parent, child, reserve, bt, ref, plen, arr, ws=None):
    from paper_2512_22737_amd import wedlm
    i32 = np.int32
    t = [dev(np.array(x, i32)) for x in (parent, child, reserve)]
    st = [dev(plen), dev(bt), dev(ref)]
    da = [dev(a) for a in arr]
    status = torch.full((len(parent),), 77, dtype=torch.int32, device="cuda")
    wedlm.wedlm_cache_fork(*t, *st, da, status, ws)
    want = O.fork(parent, child, reserve, plen, bt, ref)
    assert np.array_equal(host(status), want[3])
    assert np.array_equal(host(st[1]), want[0])
    assert np.array_equal(host(st[2]), want[1])
    assert np.array_equal(host(st[0]), want[2])
    for a, b in zip(da, moved(arr, want[4])):
        assert np.array_equal(host(a), b)
    return want


@pytest.mark.parametrize("P", [64, 5000, 20001])
@pytest.mark.parametrize("L", [1, 3])
def test_fork(P, L):
    rng = np.random.default_rng(P + L)
    bt, ref, plen = pool(rng, P, 12, 9, [37, 16, 0, 1, 128], spare=1)
    bt[2] = -1
    if P == 64:                    # whole batches of children fill the pool
        ref[:] = (ref > 0) | (rng.random(P) < 0.2)
    want = fork([0, 1, 4, 3, -1, 0, 2], [5, 6, 7, 8, 9, 10, 11],
                [37, 40, 100, 16, 33, 0, 0], bt, ref, plen,
                arrays(rng, L, P))
    assert want[3].tolist() == [0] * 7


def test_fork_runs_out_of_pages():
    """The first request that does not fit and every later one with a need is
    refused; those that need none still share."""
    rng = np.random.default_rng(1)
    bt, ref, plen = pool(rng, 20, 8, 6, [32, 80])
    ref[ref == 0] = 1
    ref[[3, 9, 11]] = 0
    bt[bt == 3] = bt[bt == 9] = bt[bt == 11] = 4
    want = fork([0, 0, 1, 0, 1], [2, 3, 4, 5, 6], [48, 80, 80, 48, 0], bt, ref,
                plen, arrays(rng, 1, 20))
    assert want[3].tolist() == [0, O.CAPACITY, 0, O.CAPACITY, 0]


def test_fork_extends_and_refuses():
    rng = np.random.default_rng(2)
    bt, ref, plen = pool(rng, 300, 14, 5, [33, 0, 50, 20, 64, 70], spare=0)
    bt[2, 1] = -1                               # a hole that is filled
    ref[:] = np.bincount(bt[bt >= 0], minlength=300)
    plen[1] = -3
    plen[5] = 81
    bt[3, 1] = 300
    want = fork(
        # extends; bad length; holes filled; bad page; full row as child;
        # parent beyond the table's width; twice one child; rows outside
        [0, 1, 2, 3, -1, 5, 4, 4, 14, -2, 4, 4],
        [0, 6, 2, 7, 4, 8, 9, 9, 10, 11, -1, 14],
        [70, 5, 66, 30, 5, 0, 64, 64, 1, 1, 1, 1], bt, ref, plen,
        arrays(rng, 2, 300))
    assert want[3].tolist() == [0, O.BAD_LEN, 0, O.BAD_PAGE, O.BAD_ROW,
                                O.BAD_LEN, O.BAD_ROW, O.BAD_ROW, O.BAD_ROW,
                                O.BAD_ROW, O.BAD_ROW, O.BAD_ROW]
    # more positions than the table has, lengths near the type's end
    want = fork([4, 4, -1], [6, 7, 8], [81, 2**31 - 1, -2**31], bt, ref, plen,
                arrays(rng, 1, 300))
    assert want[3].tolist() == [O.BAD_LEN, O.BAD_LEN, 0]


def test_fork_many_requests():
    """More requests than a workgroup has threads."""
    rng = np.random.default_rng(3)
    n = 2500
    bt, ref, plen = pool(rng, 9000, n + 3, 4, [37, 16, 20])
    parent = rng.integers(-1, 3, n)
    fork(parent, np.arange(3, n + 3), rng.integers(0, 65, n), bt, ref, plen,
         [rng.integers(0, 9, (1, 9000, 4)).astype(np.uint8)])


def test_fork_wants_2_31_pages_together():
    """1024 requests for 2^21 pages each, a pool that holds one of them and
    five pages: the sum of the needs passes 32 bits."""
    from paper_2512_22737_amd import wedlm
    n, maxp = 1024, 1 << 21
    i32 = dict(dtype=torch.int32, device="cuda")
    bt = torch.full((n, maxp), -1, **i32)
    ref = torch.zeros(maxp + 5, **i32)
    ref[7] = 1
    status = torch.full((n,), -1, **i32)
    wedlm.wedlm_cache_fork(
        torch.full((n,), -1, **i32), torch.arange(n, **i32),
        torch.full((n,), 16 * maxp, **i32), torch.zeros(n, **i32), bt, ref, [],
        status)
    assert host(status).tolist() == [0] + [O.CAPACITY] * (n - 1)
    ids = torch.arange(maxp + 1, **i32)
    assert torch.equal(bt[0], ids[ids != 7])
    assert all(bool((bt[b] == -1).all()) for b in range(1, n))
    assert bool((ref[:maxp + 1] == 1).all()) and not ref[maxp + 1:].any()


def test_fork_without_arrays_and_with_any_workspace():
    from paper_2512_22737_amd import wedlm
    rng = np.random.default_rng(4)
    bt, ref, plen = pool(rng, 50, 4, 5, [37, 16])
    n = wedlm.wedlm_cache_fork_workspace_size(2, 5, 50)
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        fork([0, 1], [2, 3], [64, 20], bt, ref, plen, [], ws)


@pytest.mark.parametrize("maxp", [3, 700])
def test_free(maxp):
    from paper_2512_22737_amd import wedlm
    rng = np.random.default_rng(maxp)
    P = 6 * maxp
    bt, ref, plen = pool(rng, P, 5, maxp, [16 * maxp, 17, 16 * maxp, 0, 9])
    bt[4, :2] = bt[0, :2]                        # shared pages
    ref[:] = np.bincount(bt[bt >= 0], minlength=P)
    bt[2, 0], bt[2, 1] = P, -5                   # outside the pool
    ref[bt[2, 2]] = 0                            # counted out already
    rows = [0, 2, 0, 5, -1, 4]
    st = [dev(bt), dev(ref), dev(plen)]
    wedlm.wedlm_cache_free(dev(np.array(rows, np.int32)), *st)
    for a, b in zip(st, O.free(rows, bt, ref, plen)):
        assert np.array_equal(host(a), b)
    # without the lengths
    st = [dev(bt), dev(ref)]
    wedlm.wedlm_cache_free(dev(np.array(rows, np.int32)), *st)
    for a, b in zip(st, O.free(rows, bt, ref, plen)):
        assert np.array_equal(host(a), b)


@pytest.mark.parametrize("P", [1, 2, 63, 1024, 1025, 9000, 300000])
@pytest.mark.parametrize("used", [0.0, 0.03, 0.5, 0.97, 1.0])
def test_compact(P, used):
    from paper_2512_22737_amd import wedlm
    print(f"compact P={P} used={used}", flush=True)
    rng = np.random.default_rng(P)
    ref = (rng.random(P) < used).astype(np.int32) * rng.integers(1, 5, P)
    ref = ref.astype(np.int32)
    if P > 60:
        ref[rng.integers(0, P, 3)] = -1          # counts as free
    bt = rng.integers(-2, P + 2, (7, 33)).astype(np.int32)
    L = 2 if P < 10000 else 1
    arr = arrays(rng, L, P) if P < 10000 else [
        rng.integers(0, 256, (1, P, 8)).astype(np.uint8)]
    want = O.compact(bt, ref)
    for in_place in (False, True):
        d, r, da = dev(bt), dev(ref), [dev(a) for a in arr]
        nt = d if in_place else torch.full_like(d, 9)
        nr = r if in_place else torch.full_like(r, 9)
        n = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        wedlm.wedlm_cache_compact(d, r, da, nt, nr, n)
        assert n.item() == want[2]
        assert np.array_equal(host(nt), want[0])
        assert np.array_equal(host(nr), want[1])
        for a, b in zip(da, moved(arr, want[3])):
            assert np.array_equal(host(a), b)
        if not in_place:
            assert np.array_equal(host(d), bt) and np.array_equal(host(r), ref)
