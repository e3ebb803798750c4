"""Sampling where sums and logits are at their limits: rows far from zero, infinities beside the largest finite values, and
rows that are cut into different numbers of parts."""
import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests.test_gpu_rows import DT, check_tokens, logits_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("temperature", [0.0371, 0.355, 0.71, 1.33])
def test_rows_far_from_zero(temperature, dtype):
    """|largest logit| / T up to 1500 of either sign: the logits times 1024 log2(e) / T have 22 digits before the point."""
    rows, vocab = 120, 300
    at = torch.linspace(1100, 1500, rows // 2, device="cuda") * temperature
    z = torch.cat([at, -at])[:, None] - 3 * temperature * torch.rand(rows, vocab, generator=torch.Generator().manual_seed(1)).cuda()
    z = z.to(DT[dtype])
    u = torch.rand(rows, generator=torch.Generator().manual_seed(2)).cuda()
    for how in ((temperature, 0, 1.0, 0.0), (temperature, 0, 0.6, 0.0), (temperature, 40, 0.9, 0.2)):
        check_tokens(z, u, how, lib.sample(z, u, *how, with_prob=True))


def test_infinities_beside_the_largest_values():
    """Infinite logits share the mass however large the finite ones are and whatever the temperature; a temperature of
    infinity leaves finite logits equal."""
    inf, nan, most = float("inf"), float("nan"), 3.4e38
    rows = [[inf, most, inf, -most], [most, inf, 1e36, nan], [-inf, nan, inf, most], [1.0, most, inf, inf],
            [1.0, -most, nan, 2.0], [-inf, 5.0, -5.0, most]]
    z = torch.tensor(rows, device="cuda")
    for v in (0.0, 0.3, 0.6, 0.99):
        u = torch.full((len(rows),), v, device="cuda")
        for t in (1.0, 1e-25, 1e25, inf):
            for how in ((t, 0, 1.0, 0.0), (t, 0, 0.45, 0.0), (t, 3, 0.8, 0.1)):
                check_tokens(z, u, how, lib.sample(z, u, *how, with_prob=True))


# A largest logit of 0, all others `x`, and top_p 1 - steps * 2^-24: the border lies among tokens that have bits below the
# last one of a mass, at places where their sum, rounded down in one piece or in eight, makes a token's difference.
BORDERS = [(-24.6891, 3), (-24.858887, 1), (-22.88196, 24), (-24.286236, 8), (-24.647385, 2), (-24.913706, 4), (-24.793331, 2),
           (-23.306297, 11), (-21.874956, 64), (-24.938128, 3), (-24.776915, 3), (-24.686554, 2), (-24.30417, 6), (-23.87952, 3),
           (-24.776066, 4), (-24.48427, 4), (-24.796192, 4), (-23.852974, 3), (-24.844908, 4), (-23.837873, 7), (-24.398659, 4),
           (-24.058304, 9), (-24.610064, 2), (-23.786625, 12)]


def alone_and_in_company(z, u, how):
    """A row of few is cut into as many parts as there are CTAs of a cluster, one of many stays whole."""
    assert len(z) >= 160
    token, prob = lib.sample(z, u, *how, with_prob=True)
    for r in range(len(z)):
        one = [h[r:r + 1].contiguous() if torch.is_tensor(h) else h for h in how]
        t, p = lib.sample(z[r:r + 1], u[r:r + 1], *one, with_prob=True)
        assert torch.equal(t[0], token[r]) and torch.equal(p[0], prob[r]), r


def test_borders_do_not_depend_on_a_rows_company():
    n, vocab = 168, 18000
    x = torch.tensor([x for x, _ in BORDERS], device="cuda").repeat(n // len(BORDERS))
    z = x[:, None].repeat(1, vocab)
    z[:, 0] = 0.0
    top_p = torch.tensor([1 - s * 2.0 ** -24 for _, s in BORDERS], device="cuda").repeat(n // len(BORDERS))
    alone_and_in_company(z, torch.ones(n, device="cuda"), (1.0, 0, top_p, 0.0))   # u = 1: the last of the kept


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_draws_do_not_depend_on_a_rows_company(dtype):
    n, vocab = 160, 17001
    g = torch.Generator().manual_seed(3)
    pick = lambda *v: torch.tensor(v)[torch.randint(0, len(v), (n,), generator=g)].cuda()  # noqa: E731
    how = (pick(0.3, 0.8, 1.0, 2.5), pick(0, 0, 60, 400).int(), pick(1.0, 0.999, 0.9, 0.5), pick(0.0, 0.0, 1e-4))
    alone_and_in_company(logits_of(n, vocab, 5, DT[dtype]), torch.rand(n, generator=g).cuda(), how)


def test_few_tokens_in_every_part_of_a_long_tail():
    """Masses of all octaves that have any, and below."""
    n, vocab = 160, 9000
    z = -40 * torch.rand(n, vocab, generator=torch.Generator().manual_seed(4)).cuda()
    top_p = 1 - torch.arange(n, device="cuda") % 16 * 2.0 ** -24
    alone_and_in_company(z, torch.ones(n, device="cuda"), (1.0, 0, top_p.float(), 0.0))
    u = np.float32(1 - 2.0 ** -24)
    check_tokens(z[:8], torch.full((8,), float(u), device="cuda"), (1.0, 0, 1.0, 0.0),
                 lib.sample(z[:8], torch.full((8,), float(u), device="cuda"), 1.0, 0, 1.0, 0.0, with_prob=True))
