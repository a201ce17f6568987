"""Appends, forks and compactions (include/wedlm_serve.h) in arrays of more than
2^31 bytes: what is written at far pages and layers is what the same call
writes in a small pool."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [40, 200])
def test_append_beyond_2_31_bytes(D, T):
    from paper_2512_22737_amd import wedlm
    L, B, H, n, maxp = 3, 2, 8, 40, 20
    page = H * 16 * D
    P = (1 << 31) // page + 100               # one layer passes 2^31 bytes
    print(f"append D={D} T={T} P={P}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(D + T)
    rnd = lambda *s: torch.randint(0, 120, s, dtype=torch.uint8, generator=g,
                                   device="cuda")
    small = [rnd(L, n, H, 16, D), rnd(L, n, H, D, 16), rnd(L, n, H) + 60,
             rnd(L, n, H) + 60]
    big = [torch.zeros(L, P, *x.shape[2:], dtype=torch.uint8, device="cuda")
           for x in small]
    far = P - n
    for x, y in zip(big, small):
        x[:, far:] = y
    k, v = (torch.randn(L, B, T, H, D, generator=g, device="cuda").to(
        torch.bfloat16) for _ in range(2))
    bt = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    bt = bt.view(B, maxp).contiguous()
    start = torch.tensor([5, 32], **I32)
    count = torch.tensor([T, T - 9], **I32)
    wedlm.wedlm_cache8_append(k, v, start, count, *small, bt)
    wedlm.wedlm_cache8_append(k, v, start, count, *big, bt + far)
    for x, y in zip(big, small):
        assert torch.equal(x[:, far:], y)
        assert not x[:, :far].any()


# pages of words of 16, 4 and 1 bytes
@pytest.mark.parametrize("page_bytes", [1 << 23, (1 << 23) + 4, (1 << 23) + 1])
def test_pages_move_beyond_2_31_bytes(page_bytes):
    from paper_2512_22737_amd import wedlm
    L, P, maxp = 2, 260, 4                    # 2.2 GB a layer
    print(f"fork and compact, pages of {page_bytes} bytes", flush=True)
    x = torch.zeros(L, P, page_bytes, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    used = [3, 257, 259]
    held = torch.randint(0, 256, (L, len(used), page_bytes), dtype=torch.uint8,
                         generator=g, device="cuda")
    x[:, used] = held
    # row 0 holds pages 257 (whole) and 259 (partly filled), row 1 page 3
    table = torch.full((3, maxp), -1, **I32)
    table[0, :2] = torch.tensor([257, 259], **I32)
    table[1, 0] = 3
    plen = torch.tensor([20, 16, 0], **I32)
    ref = torch.ones(P, **I32)                # but for 258 all are in use
    ref[258] = 0
    status = torch.full((1,), 9, **I32)
    wedlm.wedlm_cache_fork(torch.tensor([0], **I32), torch.tensor([2], **I32),
                           torch.tensor([0], **I32), plen, table, ref, [x],
                           status)
    assert status.item() == 0
    assert table[2].tolist() == [257, 258, -1, -1]
    assert torch.equal(x[:, 258], held[:, 2])
    assert torch.equal(x[:, used], held)
    # only those four are in use: they move to 0, 1, 2; page 3 stays
    ref.zero_()
    ref[3] = ref[258] = ref[259] = 1
    ref[257] = 2
    n = torch.zeros(1, **I32)
    wedlm.wedlm_cache_compact(table, ref, [x], table, ref, n)
    assert n.item() == 4
    assert table[:, :2].tolist() == [[0, 2], [3, -1], [0, 1]]
    assert ref[:5].tolist() == [2, 1, 1, 1, 0] and not ref[5:].any()
    assert torch.equal(x[:, [3, 0, 2]], held)
    assert torch.equal(x[:, 1], held[:, 2])
    assert not x[:, 4:257].any()
    # the pages behind keep their bytes
    assert torch.equal(x[:, [257, 259]], held[:, 1:])
