"""sm_linear_w4 against oracle/paged.py.  Integers with power-of-two scales have exact sums, so the results there must be the rounded
exact ones; on random data a result may be off by half a bf16 step (2^-8) and the fp32 sums: a weight enters as an integer of at most
8 bits (143 with its offset, taken back per group), the sums of a group's 32 to 128 products and of the groups are chains of at most
K / 32 + 64 additions, so (K / 32 + 64) 2^-24 of sum 2 * 143 |x| s; GELU as approximated adds 3e-4 and changes its argument's error by at
most 1.13."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2404_13528_amd import binding as sm
from util import to_np

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def case(M, N, K, group, zeros, bias, residual, act, seed=0, exact=False):
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (N, K // group), generator=g, dtype=torch.uint8) if zeros else None
    if exact:
        s = 2.0 ** torch.randint(-3, 2, (N, K // group), generator=g)
        x = torch.randint(-4, 5, (M, K), generator=g).float()
        b, r = torch.randint(-9, 10, (N,), generator=g).float(), torch.randint(-9, 10, (M, N), generator=g).float()
    else:
        s = (0.5 + torch.rand(N, K // group, generator=g)) * K ** -0.5 / 4
        x, b, r = torch.randn(M, K, generator=g), torch.randn(N, generator=g), torch.randn(M, N, generator=g)
    s, x, b, r = (t.to(BF16) for t in (s, x, b, r))
    lin = sm.LinearW4(w.cuda(), s.cuda(), z.cuda() if zeros else None, group=group, bias=b.cuda() if bias else None)
    y = lin(x.cuda(), residual=r.cuda() if residual else None, act=act)
    assert torch.equal(y, lin(x.cuda(), residual=r.cuda() if residual else None, act=act))
    want = P.linear_w4(to_np(x), w.numpy(), to_np(s), z.numpy() if zeros else None, group, to_np(b) if bias else None,
                       to_np(r) if residual else None, act)
    got = to_np(y)
    if exact:
        assert np.array_equal(got, to_np(torch.from_numpy(want).float().to(BF16)))
        return
    tol = 2.0 ** -8 * np.abs(want) + (K / 32 + 64) * 2.0 ** -24 * 2 * 143 * 1.13 * (np.abs(to_np(x)) @ np.repeat(to_np(s), group, 1).T)
    if act == "gelu":
        tol = tol + 3e-4
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,steps", [(1, 1, 1), (1, 16, 2), (2, 17, 3), (3, 100, 5), (15, 33, 1), (16, 64, 8), (17, 31, 9), (31, 130, 2), (32, 48, 33),
                                       (33, 20, 4), (64, 16, 2), (65, 40, 3), (100, 96, 7)])
def test_exact_sums(M, N, steps, group):
    case(M, N, steps * group, group, True, True, True, "none", seed=M + N, exact=True)
    case(M, N, steps * group, group, False, False, False, "none", seed=M + N + 1, exact=True)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N", [(1, 20503), (3, 8219), (3, 24610), (8, 48005), (9, 2077), (9, 4112), (16, 8219), (9, 12289), (13, 16396), (17, 2743), (31, 4112), (17, 8219),
                                 (29, 12289), (17, 16396), (70, 4100)])
def test_exact_sums_of_many_features(M, N, group):
    """Enough features for every number of tiles that a workgroup may have, at 8, 16 and 32 rows."""
    case(M, N, 3 * group, group, True, True, True, "none", seed=M + N, exact=True)


def test_residual_may_be_the_result():
    g = torch.Generator().manual_seed(8)
    lin = sm.LinearW4(torch.randint(0, 256, (200, 64), generator=g, dtype=torch.uint8).cuda(), torch.rand(200, 2, generator=g).to(BF16).cuda(), group=64)
    x, y = torch.randn(20, 128, generator=g).to(BF16).cuda(), torch.randn(20, 200, generator=g).to(BF16).cuda()
    want = lin(x, residual=y)
    assert torch.equal(lin(x, residual=y, out=y), want)


@pytest.mark.parametrize("M,N,K,group,zeros,bias,residual,act", [
    (1, 4096, 4096, 128, True, False, False, "none"), (5, 1000, 2048, 64, False, True, False, "gelu"), (32, 515, 1024, 32, True, True, True, "gelu"),
    (8, 2048, 8192, 128, True, True, True, "none"), (1, 8, 16384, 32, False, False, True, "none"), (40, 300, 1152, 128, True, False, False, "gelu"),
    (1, 11008, 4096, 128, False, True, False, "none"), (17, 20000, 512, 64, True, True, False, "none")])
def test_random(M, N, K, group, zeros, bias, residual, act):
    case(M, N, K, group, zeros, bias, residual, act, seed=N)


@pytest.mark.parametrize("M", [1, 9, 20])
@pytest.mark.parametrize("residual", [False, True])
def test_gelu_of_exact_sums(M, residual):
    """The argument is exact (integers, one power of two as the scale), so the result may be off by the error function's 1.5e-7 of half the argument, a few
    roundings of fp32 and the store's half step (a GELU that is 3e-4 off would fail at the smaller values)."""
    g = torch.Generator().manual_seed(M)
    w, x = torch.randint(0, 256, (300, 64), generator=g, dtype=torch.uint8), torch.randint(-4, 5, (M, 128), generator=g).to(BF16)
    s, r = torch.full((300, 1), 2.0 ** -7).to(BF16), torch.randn(M, 300, generator=g).to(BF16)
    arg = P.linear_w4(to_np(x), w.numpy(), to_np(s), None, 128)
    want = P.linear_w4(to_np(x), w.numpy(), to_np(s), None, 128, None, to_np(r) if residual else None, "gelu")
    got = to_np(sm.LinearW4(w.cuda(), s.cuda())(x.cuda(), residual=r.cuda() if residual else None, act="gelu"))
    tol = 2.0 ** -8 * np.abs(want) + 0.5 * np.abs(arg) * (1.5e-7 + 2.0 ** -21) + 2.0 ** -23 * np.abs(want)
    assert np.abs(arg).max() > 3 and (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


def test_rows_do_not_touch_each_other():
    """A row of infinities or NaN stays in its row, and nothing is written around the result."""
    g = torch.Generator().manual_seed(3)
    w = torch.randint(0, 256, (70, 128), generator=g, dtype=torch.uint8).cuda()
    s = torch.rand(70, 2, generator=g).to(BF16).cuda()
    lin = sm.LinearW4(w, s, group=128)
    x = torch.randn(9, 256, generator=g).to(BF16).cuda()
    buf = torch.full((11, 70), 5.0, dtype=BF16, device="cuda").view(-1)
    out = buf[80:80 + 630].view(9, 70)                    # (16-byte aligned inside a larger buffer)
    want = lin(x, out=out).clone()
    assert (buf[:80] == 5).all() and (buf[710:] == 5).all()
    x[4] = float("nan")
    got = lin(x)
    keep = [0, 1, 2, 3, 5, 6, 7, 8]
    assert torch.equal(got[keep], want[keep]) and got[4].isnan().all()
    assert lin(x[:0]).shape == (0, 70)


def test_results_over_operands_are_refused():
    lin = sm.LinearW4(torch.zeros(128, 64, dtype=torch.uint8, device="cuda"), torch.ones(128, 1, dtype=BF16, device="cuda"), group=128)
    buf = torch.ones(64, 128, dtype=BF16, device="cuda")
    with pytest.raises(sm.SmError, match="overlap"):
        lin(buf[:8], out=buf[:8])
    with pytest.raises(sm.SmError, match="overlap"):
        lin(buf[:8], residual=buf[16:24], out=buf[17:25])
    # 128 weights of -8, and 1: -1023, in bf16 -1024
    assert (lin(buf[:8], residual=buf[8:16], out=buf[16:24]) == -1024).all() and (buf[:16] == 1).all() and (buf[24:] == 1).all()


def test_captured_and_replayed():
    g = torch.Generator().manual_seed(4)
    lin = sm.LinearW4(torch.randint(0, 256, (512, 512), generator=g, dtype=torch.uint8).cuda(), torch.rand(512, 8, generator=g).to(BF16).cuda(), group=128)
    x = torch.randn(3, 1024, generator=g).to(BF16).cuda()
    y = lin(x).clone()
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        lin(x, out=y)
    for i in range(3):
        x.copy_(torch.randn(3, 1024, generator=g).to(BF16))
        cg.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, lin(x))


def test_binding_refuses_wrong_tensors():
    w, s = torch.zeros(8, 64, dtype=torch.uint8, device="cuda"), torch.ones(8, 1, dtype=BF16, device="cuda")
    with pytest.raises(sm.SmError):
        sm.LinearW4(w, s, group=48)
    with pytest.raises(ValueError):
        sm.LinearW4(w, s, group=64)
    with pytest.raises(TypeError):
        sm.LinearW4(w, s.float(), group=128)
    with pytest.raises(ValueError):
        sm.LinearW4(w.t(), s, group=128)
    lin = sm.LinearW4(w, s, group=128)
    with pytest.raises(ValueError):
        lin(torch.zeros(2, 64, dtype=BF16, device="cuda"))
    with pytest.raises(sm.SmError):
        lin(torch.zeros(2, 128, dtype=BF16, device="cuda"), act="swiglu")
