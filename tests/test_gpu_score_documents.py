"""The example runs the operators together: documents, a session, the cache, scores, a training step, alternatives."""

import pytest

pytestmark = pytest.mark.gpu


def test_example(gpu):
    from paper_2607_29678_amd import score_documents

    torch = gpu
    lines = []
    r = score_documents.main(say=lines.append)
    assert len(lines) == 4
    losses = r["losses"]
    assert losses[-1] < 0.9 * losses[0], losses
    # the session's tokens are where the plans put them: its whole text, in order, one position after the other
    more = r["more"]
    positions = more["positions"].tolist()
    assert positions == list(range(r["session_ids"][-1], int(more["lengths"][-1])))
    slots = more["slots"]
    assert len(set(slots.tolist())) == len(slots)
    # the second step's scores against plain products
    z = r["hidden"].float() @ r["weight"].float().t()
    lp = torch.log_softmax(z, 1)
    t = more["targets"].long()
    want = lp.gather(1, t.clamp(min=0)[:, None])[:, 0] * (t >= 0)
    assert torch.allclose(r["out"]["logprobs"], want, atol=1e-3)
    alt, alt_lp, g = r["alternatives"]
    z16 = z[-1].bfloat16().float()
    # a logit of 16 bits is off by at most 2^-8 of itself, and so is the sum under the logarithm
    room = 4 * 2.0**-8 * float(z16.abs().max())
    assert torch.allclose(alt_lp[0], torch.log_softmax(z16, 0).topk(alt.shape[1])[0], atol=room)
    assert float(z16[alt[0, 0].long()]) >= float(z16.max()) - room
    # the entropy's gradient does not change when all logits move together
    assert abs(float(g.float().sum())) < 1e-2
