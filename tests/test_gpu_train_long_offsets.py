"""The attention backward on arrays of more than 2^31 elements whose sequences
all differ: an offset cut to fewer bits, or a sequence taken for another, reads
other values."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 100 GiB")
    yield
    torch.cuda.empty_cache()


def test_attention_backward_of_sequences_that_differ():
    from paper_2512_22737_amd import wedlm as W
    n, L, block, Hq, Hkv, D = 1040, 1024, 64, 16, 2, 64
    assert n * 2 * L * Hq * D > 1 << 31
    print("attention backward, 2^31 elements, sequences that differ",
          flush=True)
    g = torch.Generator(device="cuda").manual_seed(21)
    fill = lambda h: torch.empty(n, 2 * L, h, D, dtype=torch.bfloat16,
                                 device="cuda").normal_(generator=g)
    q, k, v, dout = fill(Hq), fill(Hkv), fill(Hkv), fill(Hq)
    out, lse = torch.empty_like(q), torch.empty(n, 2 * L, Hq, device="cuda")
    for i in range(0, n, 130):
        s = slice(i, i + 130)
        W.wedlm_dual_stream_attn(q[s], k[s], v[s], block, out[s], lse[s])
    got = [torch.full_like(x, float("nan")) for x in (q, k, v)]
    W.wedlm_dual_stream_attn_backward(q, k, v, block, out, lse, dout, *got)
    # 2^32 bytes are 1024 sequences of q, 2^31 are 512; 8 times as many of k
    for at in (0, 1, 15, 511, 512, 527, 1023, 1024, n - 1):
        s = slice(at, at + 1)
        one = [torch.empty_like(x[s]) for x in (q, k, v)]
        W.wedlm_dual_stream_attn_backward(q[s], k[s], v[s], block, out[s],
                                          lse[s], dout[s], *one)
        assert torch.equal(got[0][s], one[0]), at
        # sums in another order may round to the next bf16 value, 2^-7 away
        for x, y in zip(got[1:], one[1:]):
            err = (x[s].float() - y.float()).norm() / y.float().norm()
            assert err <= 2.0 ** -7, (at, err)
