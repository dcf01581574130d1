"""Head gradients of a mean over many rows: all rows pass back the same gradient, so that a rounding which they share
does not average out."""

import pytest

torch = pytest.importorskip("torch")
import paper_2607_29678_amd as tt  # noqa: E402
from test_gpu_head_gradient_norms import MANY, TYPES, gradient, make, off_by, softmax  # noqa: E402

pytestmark = pytest.mark.gpu


# 1 / 510 and 1 / 1020 lie half way between two floats of 8 bits, 3 / 2048 * 1.0005 between two of 11
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,each,scale", [(510, 1 / 510, 1.0), (1020, 1 / 1020, 1.0), (300, 1 / 300, 0.85),
                                             (700, 3 / 2048 * (1 + 2.0**-11), 1.0), (510, 37.0, 1.0)])
@pytest.mark.parametrize("entropy_weight", [None, 0.01])
def test_norm_of_the_error(gpu, rows, each, scale, kind, entropy_weight):
    vocab, width = 20_011, 256
    hidden, weight, t, _, _ = make(rows, vocab, width, kind, "cuda")
    z, _ = softmax(hidden, weight)
    lp = (z * scale).log_softmax(1)
    m = z.amax(1)
    stats = torch.stack([m, ((z - m[:, None]) * scale).exp().sum(1).log()], 1).float()
    entropy = -(lp.exp() * lp).sum(1).float()
    a = torch.full((rows,), -each, device="cuda")
    b = None if entropy_weight is None else torch.full((rows,), entropy_weight * each, device="cuda")
    room = torch.full((tt.head_scores_grad_workspace(rows, vocab, width),), 255, dtype=torch.uint8, device="cuda")
    gh, gw = torch.full_like(hidden, 55.0), torch.full_like(weight, 55.0)
    tt.head_scores_grad(hidden, weight, t, stats, entropy, a, b, gh, gw, scale=scale, workspace=room)
    torch.cuda.synchronize()
    g = scale * gradient(lp, t, a, b)
    off = off_by(gh, g @ weight.double(), kind), off_by(gw, g.t().contiguous() @ hidden.double(), kind)
    assert max(off) <= MANY, off
