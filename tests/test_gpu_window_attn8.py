"""GPU parity of wedlm_window_attn_cache8 (include/wedlm_serve.h) with the
fp64 attention of oracle/serve_oracle.py, element by element within the bounds
derived there."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def build(lens, W, Hq, Hkv, D, seed, extra=2, sharp=1.0, maxp=None):
    """Pages in random order; every code and scale that no prefix holds is
    NaN, so that whatever is used of them shows."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    need = [-(-n // 16) for n in lens]
    P = sum(need) + extra
    maxp = maxp or max(need) + 1
    ids = rng.permutation(P)
    bt = np.full((B, maxp), -1, np.int32)
    k8 = np.full((P, Hkv, 16, D), 0x7f, np.uint8)
    v8 = np.full((P, Hkv, D, 16), 0xff, np.uint8)
    ke = np.full((P, Hkv), 255, np.uint8)
    ve = np.full((P, Hkv), 255, np.uint8)
    at = 0
    for b, n in enumerate(lens):
        for j in range(need[b]):
            p = ids[at]
            at += 1
            bt[b, j] = p
            m = min(16, n - 16 * j)
            k8[p, :, :m] = O.encode(np.clip(
                rng.standard_normal((Hkv, m, D)) * 60, -448, 448))
            v8[p, :, :, :m] = O.encode(np.clip(
                rng.standard_normal((Hkv, D, m)) * 60, -448, 448))
            ke[p] = rng.integers(119, 123, Hkv)
            ve[p] = rng.integers(117, 125, Hkv)
    q = torch.from_numpy(rng.standard_normal((B, W, Hq, D)) * sharp)
    kw = torch.from_numpy(rng.standard_normal((B, W, Hkv, D)))
    vw = torch.from_numpy(rng.standard_normal((B, W, Hkv, D)))
    return dict(q=q.to(torch.bfloat16).cuda(), kw=kw.to(torch.bfloat16).cuda(),
                vw=vw.to(torch.bfloat16).cuda(), k8=k8, v8=v8, ke=ke, ve=ve,
                bt=bt, lens=lens)


def call(s, mp=None, lse=True, ws=None, scale=None):
    from paper_2512_22737_amd import wedlm
    B, W, Hq, D = s["q"].shape
    out = torch.full_like(s["q"], float("nan"))
    z = torch.full((B, W, Hq), float("nan"), device="cuda") if lse else None
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    wedlm.wedlm_window_attn_cache8(
        s["q"], s["kw"], s["vw"], dev(s["k8"]), dev(s["v8"]), dev(s["ke"]),
        dev(s["ve"]), dev(s["bt"]), dev(np.array(s["lens"], np.int32)),
        max(s["lens"]) if mp is None else mp, out, z, status, ws, scale)
    torch.cuda.synchronize()
    return out, z, status


def check(s, out, z, only=None, scale=None):
    B, W, Hq, D = s["q"].shape
    for b in only if only is not None else range(B):
        k, v = O.gather(s["k8"], s["v8"], s["ke"], s["ve"], s["bt"], b,
                        s["lens"][b])
        o, l, bo, bl = O.attention(
            s["q"][b].double().cpu().numpy(),
            s["kw"][b].double().cpu().numpy(),
            s["vw"][b].double().cpu().numpy(), k, v,
            D ** -0.5 if scale is None else scale)
        err = np.abs(out[b].double().cpu().numpy() - o)
        assert (err <= bo).all(), (b, (err / bo).max())
        if z is not None:
            err = np.abs(z[b].double().cpu().numpy() - l)
            assert (err <= bl).all(), (b, (err / bl).max())


# every residue of a prefix in a tile, splits that begin and end, one row to
# more rows than a workgroup takes
@pytest.mark.parametrize("lens", [
    [0], [1], [16, 15, 17], [31, 32, 33, 0], [64, 257, 5], [255, 256, 511],
    [600, 1300], [2049], [4000, 33, 0, 1]])
@pytest.mark.parametrize("W,Hq,Hkv,D", [
    (1, 4, 4, 64), (1, 32, 8, 128), (16, 4, 2, 64), (5, 28, 4, 128),
    (33, 8, 2, 128), (64, 8, 2, 64), (64, 16, 2, 128)])
def test_lengths(lens, W, Hq, Hkv, D):
    print(f"attention lens={lens} W={W} {Hq}/{Hkv} D={D}", flush=True)
    s = build(lens, W, Hq, Hkv, D, sum(lens) + W)
    out, z, status = call(s)
    assert not status.any()
    check(s, out, z)


@pytest.mark.parametrize("W", range(1, 65, 7))
def test_windows(W):
    s = build([100, 16], W, 4, 2, 64, W)
    out, z, _ = call(s)
    check(s, out, z)


def test_more_rows_than_one_workgroup_takes():
    s = build([70, 300], 64, 24, 1, 64, 3)      # 1536 rows of one kv head
    out, z, _ = call(s)
    check(s, out, z)


@pytest.mark.parametrize("W", [1, 32])
def test_bound_far_above_the_prefixes(W):
    """max_prefix_len sizes the split; sequences use as much of it as they
    have, and lse may be left out."""
    s = build([700, 40, 0], W, 8, 2, 128, 9, maxp=400)
    out, z, _ = call(s, mp=6000)
    check(s, out, z)
    again, _, _ = call(s, mp=6000, lse=False)
    assert torch.equal(out, again)
    one, _, _ = call(s, mp=700)
    check(s, one, None)


def test_growing_scores():
    """Keys that outgrow every earlier one by hundreds of log2 units, and a
    sharp softmax."""
    s = build([900, 900], 8, 4, 2, 64, 11, sharp=3.0)
    for b in range(2):
        for j in range(57):
            s["ke"][s["bt"][b, j]] = 115 + (j // 7 if b == 0 else 8 - j // 7)
    out, z, _ = call(s)
    check(s, out, z)


def test_scales_at_the_ends():
    """The smallest and largest scales of values and keys that meet: zero
    codes at the largest scale, a page of tiny values."""
    s = build([48, 48], 3, 4, 2, 64, 12)
    p = s["bt"][0, 1]
    s["k8"][p] = 0
    s["ke"][p] = 254
    s["v8"][p] = 0
    s["ve"][p] = 254
    s["ve"][s["bt"][0, 0]] = 1
    s["ke"][s["bt"][1, 2]] = 1
    out, z, _ = call(s)
    check(s, out, z)


def test_softmax_scale():
    s = build([130], 4, 4, 2, 64, 13)
    out, z, _ = call(s, scale=0.31)
    check(s, out, z, scale=float(np.float32(0.31)))


@pytest.mark.parametrize("W", [2, 40])
def test_bad_sequences_leave_the_others_alone(W):
    """A page outside the cache, a length beyond the bound, a negative one, one
    beyond the table: told by status, no other sequence changes."""
    s = build([600, 300, 290, 100, 310], W, 8, 2, 64, 14)
    want, _, _ = call(s, mp=600)
    bad = dict(s, bt=s["bt"].copy(), lens=list(s["lens"]))
    bad["bt"][1, 3], bad["bt"][1, 4] = len(s["k8"]), -7
    bad["lens"][2], bad["lens"][3] = 601, -1
    out, z, status = call(bad, mp=600)
    assert status.tolist() == [0, O.BAD_PAGE, O.BAD_LEN, O.BAD_LEN, 0]
    assert torch.equal(out[0], want[0]) and torch.equal(out[4], want[4])
    check(bad, out, z, [0, 4])
    short = dict(s, bt=np.ascontiguousarray(s["bt"][:, :20]))
    out, z, status = call(short, mp=600)
    assert status.tolist() == [O.BAD_LEN, 0, 0, 0, 0]
    check(short, out, z, [1, 2, 3, 4])


def test_same_bits_every_time_and_any_workspace():
    from paper_2512_22737_amd import wedlm
    s = build([3000, 1000], 16, 8, 2, 128, 15)
    n = wedlm.wedlm_window_attn_cache8_workspace_size(2, 16, 8, 2, 128, 3000)
    assert n > 0
    first = call(s)
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        again = call(s, ws=ws)
        assert torch.equal(first[0], again[0])
        assert torch.equal(first[1], again[1])


def test_pages_beyond_2_31_bytes():
    """Page offsets that pass 32 bits."""
    from paper_2512_22737_amd import wedlm
    s = build([90], 4, 16, 8, 128, 16)
    P, far = 135000, 134990                   # 16 KB each: 2.2 GB
    k8 = torch.zeros(P, 8, 16, 128, dtype=torch.uint8, device="cuda")
    v8 = torch.zeros(P, 8, 128, 16, dtype=torch.uint8, device="cuda")
    ke = torch.zeros(P, 8, dtype=torch.uint8, device="cuda")
    ve = torch.zeros_like(ke)
    n = len(s["k8"])
    for big, x in ((k8, "k8"), (v8, "v8"), (ke, "ke"), (ve, "ve")):
        big[far:far + n] = dev(s[x])
    out = torch.zeros_like(s["q"])
    bt = torch.where(dev(s["bt"]) >= 0, dev(s["bt"]) + far, -1)
    wedlm.wedlm_window_attn_cache8(
        s["q"], s["kw"], s["vw"], k8, v8, ke, ve, bt,
        dev(np.array([90], np.int32)), 90, out)
    check(s, out, None)
