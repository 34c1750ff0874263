"""Lists of rows whose first tile says little of the rest: entries that are not legal, or low ones, in
one run (a padded head, actions of another phase), and rows that end within a tile."""
import math

import pytest

from test_gpu_log_probs import TYPES, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def rows_with_runs(n, a, dtype, g):
    """Rows of noise in which a run of entries is out, or low, or high; the runs' ends fall anywhere.
    Returns them and a mask that leaves the same runs out."""
    x = torch.randn((n, a), generator=g, device="cuda") * 2
    legal = torch.ones((n, a), dtype=torch.bool, device="cuda")
    for r in range(n):
        kind = r % 9
        to = int(torch.randint(1, a, (1,), generator=g, device="cuda"))
        if kind == 0:
            legal[r, :to] = False
        elif kind == 1:
            legal[r, :to // 2048 * 2048] = False
        elif kind == 2:
            legal[r, a - min(to, 70):] = True
            legal[r, :a - min(to, 70)] = False
        elif kind == 3:
            x[r, :to] -= 100
        elif kind == 4:
            x[r, to:] += torch.arange(a - to, device="cuda") / 8
        elif kind == 5:
            x[r, :to] = torch.finfo(dtype).min
        elif kind == 6:
            legal[r, to // 2:to] = False
            x[r, to:] += 50
        elif kind == 7:
            x[r, :to], x[r, to:] = 1.0, x[r, to:] + 5
            x[r, a - 1] = math.nan if r % 2 else math.inf
        else:
            x[r] += torch.arange(a, device="cuda") // 512 % 7 * 3.0
    return x.to(dtype), legal


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", [(1025, 27), (1200, 300), (1536, 27), (1537, 27), (2049, 300),
                                  (4100, 300), (8192, 54), (8193, 54), (20000, 54), (33333, 27),
                                  (65536, 270), (200000, 18)])
def test_lists_behind_runs(dtype, a, n):
    g = torch.Generator(device="cuda").manual_seed(a + n)
    x, legal = rows_with_runs(n, a, dtype, g)
    act = torch.randint(0, a, (n,), generator=g, device="cuda")
    for top in (1, 8, 64, 65, 256):
        check(x, act, mask=legal, top=top, what="mask")
        check(torch.where(legal, x, -math.inf), act, top=top, what="-inf")


def least_time(fn):
    fn()
    times = []
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(5):
            fn()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("dtype, n, a, top, prefix",
                         [(torch.bfloat16, 4096, 65536, 64, 8192),
                          (torch.bfloat16, 4096, 65536, 64, 16384),
                          (torch.float32, 2048, 32768, 64, 4096),
                          (torch.bfloat16, 8192, 8000, 8, 2048)])
def test_a_run_that_is_out_takes_no_search_of_the_row(dtype, n, a, top, prefix):
    """A first tile without entries: the exact search of all others took ten times as long as the
    row without the run; twice its way through memory is twice."""
    import paper_2106_07551_amd as M
    x = torch.randn((n, a), device="cuda").to(dtype)
    plain = least_time(lambda: M.log_probs(x, top=top))
    x[:, :prefix] = -math.inf
    assert least_time(lambda: M.log_probs(x, top=top)) <= 4 * plain


def test_rows_that_end_within_a_tile():
    """bf16 rows of 1025 to 1536 entries leave a wavefront without any: each list took the exact
    search (2000 x 1200, 100 places, 8 times as long as rows of 2048)."""
    import paper_2106_07551_amd as M
    x = torch.randn((2000, 2048), device="cuda").bfloat16()
    whole = least_time(lambda: M.log_probs(x, top=100))
    for a in (1025, 1200, 1536):
        y = x[:, :a].contiguous()
        assert least_time(lambda: M.log_probs(y, top=100)) <= 3 * whole
