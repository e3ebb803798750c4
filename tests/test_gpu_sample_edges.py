"""Sampling where sums and logits are at their limits."""
import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests.test_gpu_rows import DT, check_tokens

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
