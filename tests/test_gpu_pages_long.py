"""Forks of prefixes that end at the last positions of 32 bits
(include/wedlm_serve.h): every page of the parent is looked at."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MAXP = 1 << 27                                # pages of 2^31 positions


def fork(table, plen, ref):
    from paper_2512_22737_amd import wedlm
    i32 = dict(dtype=torch.int32, device="cuda")
    status = torch.full((1,), 9, **i32)
    wedlm.wedlm_cache_fork(torch.zeros(1, **i32), torch.ones(1, **i32),
                           torch.zeros(1, **i32), plen, table, ref, [], status)
    return status.item()


@pytest.mark.parametrize("short", [1, 16])
def test_fork_of_the_longest_prefix(short):
    """A bad page anywhere refuses the request and changes nothing; without
    one the child shares all whole pages."""
    i32 = dict(dtype=torch.int32, device="cuda")
    c = 2 ** 31 - short
    pages, full = -(-c // 16), c // 16
    table = torch.full((2, MAXP), -1, **i32)
    table[0, :pages] = 3
    plen = torch.tensor([c, 5], **i32)
    ref = torch.zeros(50, **i32)
    ref[3] = pages
    was = ref.clone()
    for at, bad in ((0, -1), (pages - 1, 50)):
        table[0, at] = bad
        print(f"fork c={c} entry {at} = {bad}", flush=True)
        assert fork(table, plen, ref) == 2
        assert torch.equal(ref, was) and plen.tolist() == [c, 5]
        assert bool((table[1] == -1).all())
        table[0, at] = 3
    assert fork(table, plen, ref) == 0
    assert plen.tolist() == [c, c]
    was[3] += full
    assert bool((table[1, :full] == 3).all())
    if full < pages:
        assert table[1, full].item() == 0
        was[0] = 1
    assert bool((table[1, pages:] == -1).all())
    assert torch.equal(ref, was)
