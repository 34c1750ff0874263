"""Log probabilities at the ends of fp32's range, against the formulas in 64 bits (tolerances: as
in the other tests of them)."""
import math

import pytest

from test_gpu_log_probs import TYPES, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# a lane per row; few lanes, by rounds and by wavefronts; wavefronts; a workgroup; parts of rows
SIZES = [(18, 140000), (18, 300), (250, 40), (1000, 30), (1000, 4500), (3000, 700), (9000, 20),
         (9000, 2100), (131071, 3)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", SIZES)
@pytest.mark.parametrize("T", [1.0, 4.0, 2.0 ** 100])
def test_logits_further_apart_than_fp32_reaches(dtype, a, n, T):
    """3e38 and -3e38 differ by more than fp32's largest number; over T = 4 and 2^100 their
    difference fits again, and so do l and the lists' entries."""
    g = torch.Generator(device="cuda").manual_seed(a + n)
    x = torch.randn((n, a), generator=g, device="cuda")
    x[:, 20:] = torch.where(torch.rand((n, max(a - 20, 0)), generator=g, device="cuda") < 30 / a,
                            x[:, 20:], -math.inf)
    x[:, 3], x[:, 7], x[:, 11] = 3e38, -3e38, -1e38
    x[1::3, 3] = 2e30
    x = x.to(dtype)
    act = torch.tensor([7, 11, 3, 0, -1], dtype=torch.int32, device="cuda").repeat(n // 5 + 1)[:n]
    for top in (0, 5, 64, 256) if n < 100000 else (0, 18):
        stats = check(x, act, T=T, top=top, what="far")
        assert T == 1.0 or bool(torch.isfinite(stats).all())
