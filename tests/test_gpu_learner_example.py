"""The learner's operators used together (examples/learner.py): one round of
population-based training with a best response from trajectory records and a
student distilled from the mixture, both added to the population."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import learner
    return learner


def test_round_of_training():
    lines = []
    out = _example().run(n_envs=256, horizon=6, policies=5, steps=12, say=lines.append)
    print("\n".join(lines), flush=True)
    assert len(lines) == 4
    assert np.isfinite(out["returns"]).all() and np.isfinite(out["losses"]).all()
    # a student that starts as the mean of the weights fits the mixture better
    assert out["losses"][-1] < 0.9 * out["losses"][0]
    assert torch.isfinite(out["stats"]).all() and (out["stats"][2] >= -1e-4).all()
    counts = out["table"]["counts"]
    assert counts.shape == (7, 7) and (counts[5:, :] > 0).all() and (counts[:, 5:] > 0).all()
    assert torch.isfinite(out["sigma"]).all()


def test_network_matches_the_populations_forward():
    """The example's network gives the logits that the population's kernels give
    for the same weights (bf16 operands, fp32 accumulation; a hidden value on the
    edge of a rounding may fall to either side, which 1e-2 of the largest logit
    covers, as in the parity tests)."""
    import paper_2106_07551_amd as M
    import workloads as W
    from paper_2106_07551_amd import workload_io as IO
    wl = W.team_variant(2, d=256, P=3, n_envs=64, horizon=1)
    pop, env = IO.make_population(wl), IO.make_env(wl)
    pairs = torch.ones((64, 2), dtype=torch.int32, device="cuda")
    logits = torch.empty((1, 128, wl.n_actions), device="cuda")
    states = torch.empty((64, wl.d), device="cuda")
    pop.rollout(env, 64, pairs, wl.seed, 1,
                trace=M.Trace(snap_steps=[0], logits=logits, states=states))
    net = _example().Net([torch.from_numpy(w[1]).cuda() for w in wl.weights],
                         [torch.from_numpy(b[1]).cuda() for b in wl.biases])
    own = net.forward(states.bfloat16())
    ref = logits[0].view(64, 2, -1)[:, 0]
    assert (own - ref).abs().max() <= 1e-2 * ref.abs().max()
    pop.close()
