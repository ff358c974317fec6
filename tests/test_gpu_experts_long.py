"""More tokens than one launch holds: the operators that stream run in several, each token once."""
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc

pytestmark = pytest.mark.gpu

T = (1 << 26) + 5


def _cycle(rows, n):
    """n rows, one after the other again and again."""
    return rows.repeat(-(-n // len(rows)), 1)[:n]


def test_gradient_of_the_sum():
    N = 8
    g = torch.Generator(device="cuda").manual_seed(1)
    whole = lambda n: torch.randint(-3, 4, (n, N), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    dO, Y = _cycle(whole(1013), T), _cycle(whole(1019), T)  # (whole numbers: every sum is exact)
    Wt = _cycle(torch.randint(-2, 3, (1021, 1), generator=g, device="cuda").float(), T)
    Place = (T - 1 - torch.arange(T, device="cuda")).to(torch.int32).view(T, 1)
    dY, dWt = torch.full_like(Y, float("nan")), torch.full_like(Wt, float("nan"))
    tc.tc_expert_sum_grad(dO, Y, Wt, Place, dY, dWt)
    assert torch.equal(dY.flip(0), (dO.float() * Wt).to(torch.bfloat16))
    assert torch.equal(dWt[:, 0], (dO.float() * Y.flip(0).float()).sum(dim=1))


def test_the_sum():
    n, N = (1 << 29) + 5, 7
    Y = torch.randn((5, N), device="cuda").to(torch.bfloat16)
    Place = (torch.arange(n, device="cuda", dtype=torch.int32) % 5).view(n, 1)
    O = torch.full((n, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    tc.tc_expert_sum(Y, None, Place, O)
    assert torch.equal(O[:n // 5 * 5].view(-1, 5 * N).amin(dim=0), Y.view(-1)) and torch.equal(O[:n // 5 * 5].view(-1, 5 * N).amax(dim=0), Y.view(-1))
    assert torch.equal(O[n // 5 * 5:], Y[:n % 5])


def test_gradient_of_the_router():
    E = 129  # (a wavefront a token)
    L = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    Id = (torch.arange(T, device="cuda", dtype=torch.int32) % E).view(T, 1)
    dWt = (1 + torch.arange(T, device="cuda", dtype=torch.int32) % 7).float().view(T, 1)
    dL = torch.full_like(L, float("nan"))
    tc.tc_route_grad(L, Id, dWt, dL)
    period = E * 7  # (everything comes again after so many tokens)
    first = dL[:period].double()
    want = -(dWt[:period].double() / E ** 2).expand(period, E).clone()
    want.scatter_(1, Id[:period].long(), dWt[:period].double() / E * (1 - 1 / E))
    assert bool(((first - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17 * 2 / E * 7).all())
    for at in range(period, T, period * 2000):
        some = dL[at:min(T, at + period * 2000)]
        whole = len(some) // period * period
        assert bool((some[:whole].view(-1, period, E) == dL[:period]).all()) and torch.equal(some[whole:], dL[:len(some) - whole])
