"""GPU parity of wedlm_cache8_append and wedlm_commit_cache8
(include/wedlm_serve.h) with oracle/serve_oracle.py: codes and exponents are
equal, every byte that is not written keeps its value."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(x):
    return x.cpu().numpy()


def rows(rng, L, B, T, H, D, spread=3.0):
    """bf16 rows of different ranges, with zeros and extremes among them."""
    x = rng.standard_normal((L, B, T, H, D)) * np.exp(
        spread * rng.standard_normal((L, B, T, H, 1)))
    x[rng.random(x.shape) < 0.02] = 0.0
    if x.size > 300:
        flat = x.reshape(-1)
        flat[rng.integers(0, x.size, 6)] = [np.nan, np.inf, -np.inf, 2e38,
                                            1e-39, -0.0]
    t = torch.from_numpy(x).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def cache(rng, L, P, H, D):
    return [rng.integers(0, 256, (L, P, H, 16, D)).astype(np.uint8),
            rng.integers(0, 256, (L, P, H, D, 16)).astype(np.uint8),
            rng.integers(100, 140, (L, P, H)).astype(np.uint8),
            rng.integers(100, 140, (L, P, H)).astype(np.uint8)]


def same(got, want):
    """NaN codes count as equal whatever their sign."""
    got, want = host(got), want
    if got.ndim == 5:
        got = np.where((got & 0x7f) == 0x7f, 0x7f, got)
        want = np.where((want & 0x7f) == 0x7f, 0x7f, want)
    return np.array_equal(got, want)


def check_append(L, B, T, H, D, start, count, bt, P, seed, status=0):
    from paper_2512_22737_amd import wedlm
    print(f"append L={L} B={B} T={T} H={H} D={D} {start} {count}", flush=True)
    rng = np.random.default_rng(seed)
    (k, kn), (v, vn) = (rows(rng, L, B, T, H, D) for _ in range(2))
    st = cache(rng, L, P, H, D)
    want = O.append(kn, vn, start, count, *st, bt)
    got = [dev(x) for x in st]
    told = torch.zeros(B, dtype=torch.int32, device="cuda")
    i32 = np.int32
    wedlm.wedlm_cache8_append(k, v, dev(np.array(start, i32)),
                              dev(np.array(count, i32)), *got, dev(bt), told)
    for a, b in zip(got, want[:4]):
        assert same(a, b)
    assert np.array_equal(host(told), want[4])
    return want[4]


def table(rng, B, maxp, P):
    return rng.permutation(P)[:B * maxp].reshape(B, maxp).astype(np.int32)


@pytest.mark.parametrize("H", [1, 2, 3, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_append_every_offset_and_count(H, D):
    rng = np.random.default_rng(H)
    start = list(range(16)) + [16, 31, 47]
    count = [(7 * i) % 20 for i in range(len(start))]
    B = len(start)
    check_append(2, B, 20, H, D, start, count, table(rng, B, 5, 5 * B + 3),
                 5 * B + 3, 10 + H)


@pytest.mark.parametrize("T,start,count", [
    (1, [0, 5, 15], [1, 1, 0]), (64, [0, 3, 16], [64, 64, 17]),
    (333, [0, 0, 9], [333, 1, 300])])
def test_append_lengths(T, start, count):
    rng = np.random.default_rng(T)
    check_append(1, 3, T, 2, 128, start, count, table(rng, 3, 24, 80), 80, T)


def test_append_refuses_what_has_no_page():
    """Positions behind the table, pages outside the cache, bad starts and
    counts: those rows are left out, every other is written."""
    rng = np.random.default_rng(5)
    bt = table(rng, 6, 3, 30)
    bt[1, 1], bt[2, 0] = 30, -1
    want = check_append(2, 6, 40, 2, 64, [10, 4, 14, -1, 3, 2**31 - 9],
                        [40, 30, 9, 5, 41, 9], bt, 30, 5)
    assert want.tolist() == [O.CAPACITY, O.BAD_PAGE, O.BAD_PAGE, O.BAD_LEN,
                             O.BAD_LEN, O.CAPACITY]


def test_append_in_steps_is_append_at_once_where_scales_agree():
    """Rows in one range: whatever the steps, the same codes."""
    from paper_2512_22737_amd import wedlm
    g = torch.Generator(device="cuda").manual_seed(1)
    k = 1 + torch.rand(1, 1, 50, 2, 64, generator=g, device="cuda")
    k = k.to(torch.bfloat16)
    bt = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    i32 = dict(dtype=torch.int32, device="cuda")
    outs = []
    for steps in ([50], [1] * 50, [7, 9, 16, 1, 17]):
        c = [torch.zeros(1, 4, 2, 16, 64, dtype=torch.uint8, device="cuda"),
             torch.zeros(1, 4, 2, 64, 16, dtype=torch.uint8, device="cuda"),
             torch.zeros(1, 4, 2, dtype=torch.uint8, device="cuda"),
             torch.zeros(1, 4, 2, dtype=torch.uint8, device="cuda")]
        at = 0
        for n in steps:
            x = k[:, :, at:at + n].contiguous()
            wedlm.wedlm_cache8_append(x, x, torch.tensor([at], **i32),
                                      torch.tensor([n], **i32), *c, bt)
            at += n
        outs.append(c)
    for c in outs[1:]:
        for a, b in zip(outs[0], c):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rule", [0, 1, 2])
@pytest.mark.parametrize("L,B", [(1, 1), (3, 5)])
def test_commit_is_the_bf16_commit_and_an_append(rule, L, B):
    """The window's part is that of wedlm_commit_layers, bit by bit; the
    caches get what an append of the committed rows gives them."""
    from paper_2512_22737_amd import wedlm
    print(f"commit rule={rule} L={L} B={B}", flush=True)
    W, H, D, P, maxp = 24, 2, 64, 60, 8
    rng = np.random.default_rng(rule + L)
    win = rng.integers(0, 99, (B, W)).astype(np.int32)
    for b in range(B):
        n = [0, W, 5, 1, 17][b]
        win[b, n:] = np.where(rng.random(W - n) < 0.6, -1, win[b, n:])
        if n < W:
            win[b, n] = -1
    start = rng.integers(0, 70, B).astype(np.int32)
    bt = table(rng, B, maxp, P)
    if B > 1:
        bt[2, start[2] // 16] = -1            # nothing is committed there
        win[2, 0] = 3
    (k, kn), (v, vn) = (rows(rng, L, B, W, H, D) for _ in range(2))
    ent = dev(rng.random((B, W)).astype(np.float32))
    am = dev(rng.integers(0, 99, (B, W)).astype(np.int32))
    st = cache(rng, L, P, H, D)

    def outs():
        z = dict(dtype=torch.int32, device="cuda")
        return [torch.full((B,), 9, **z), torch.full((B, W), 9, **z),
                torch.full((B, W), 9, **z),
                torch.full((B, W), 9, dtype=torch.uint8, device="cuda"),
                torch.full((B,), 9, **z)]
    w1, s1, o1 = dev(win), dev(start), outs()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    wedlm.wedlm_commit_layers(
        w1, s1, am, ent, 0.5, 0.01, k, v, torch.zeros(L, P, H, 16, D, **bf),
        torch.zeros(L, P, H, D, 16, **bf), dev(bt), *o1, rule)
    w2, s2, o2 = dev(win), dev(start), outs()
    got = [dev(x) for x in st]
    wedlm.wedlm_commit_cache8(w2, s2, am, ent, 0.5, 0.01, k, v, *got, dev(bt),
                              *o2, rule)
    for a, b in zip([w1, s1] + o1, [w2, s2] + o2):
        assert torch.equal(a, b)
    want = O.append(kn, vn, start, host(o1[0]), *st, bt)
    for a, b in zip(got, want[:4]):
        assert same(a, b)
