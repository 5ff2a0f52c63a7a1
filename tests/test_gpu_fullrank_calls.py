"""Full-rank operators: what a call promises at the edges of its arguments."""
import numpy as np
import pytest

from tests import fullrank_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    from paper_2602_04396_amd import lordo
    lordo.load()
    return t


@pytest.mark.parametrize("state", ["f32", "q8"])
@pytest.mark.parametrize("rows", [40, 4200])
def test_the_new_weight_is_rounded_once(torch, state, rows):
    """With decay too: what is taken off a weight is formed at its own size, so the new fp32 weight is off by one rounding of itself and some of a change a
    thousand times smaller: of the update 17.5 (adamw_bounds) and 1 of its sum with the decay; of the decay 3 of lr sqrt(c2) / c1, 3 of the decay over
    sqrt(c2) / c1 and 1 of the sum."""
    from paper_2602_04396_amd import lordo
    gen, lr, wd, cols = torch.Generator(device="cuda").manual_seed(3), 1e-4, 0.1, 1031
    hp = lordo.adamw_hparams(weight_decay=wd, state_dtype=lordo.Q8 if state == "q8" else lordo.F32)
    opt = lordo.AdamW([(rows, cols)], hp, torch)
    W, G = [torch.randn(rows, cols, generator=gen, device="cuda")], [torch.randn(rows, cols, generator=gen, device="cuda")]
    w0, g = (x[0].double().cpu().numpy().reshape(-1) for x in (W, G))
    opt.local_step(W, G, lr)
    zero = np.zeros_like(w0)
    w, _, _, size = ref.adamw(w0, zero, zero, g, 1, lr, hp.beta1, hp.beta2, hp.eps, wd)
    got = W[0].double().cpu().numpy().reshape(-1)
    assert np.all(np.abs(got - w) <= ref.EPS32 * (np.abs(w) + lr * (22 * size + 8 * wd * np.abs(w0))))
