"""GPU tests of the operators together: a small quantized language model trained through them, with its activations
kept in 8 bits and without."""
import pytest
import torch

from paper_2411_11038_b200 import binding as B
from paper_2411_11038_b200 import lm_step

pytestmark = pytest.mark.gpu

T, V, D, F = 512, 1000, 256, 1024


def batch(seed):
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=gen)
    labels = ((ids * 7 + 3) % V).to(torch.int32)
    labels[torch.rand((T,), generator=gen) < 0.1] = -1
    return ids.cuda(), labels.cuda()


@pytest.mark.parametrize("checkpoint", [True, False])
def test_training_lowers_the_loss(checkpoint):
    net = lm_step.QuantizedLm(T, V, D, F, blocks=2, checkpoint=checkpoint)
    losses = [float(net.step(*batch(k), lr=2.0)) for k in range(40)]
    assert net.ctx.device_status() == 0
    assert abs(losses[0] - torch.log(torch.tensor(float(V))).item()) < 1.5      # about log V before training
    assert losses[-1] < 0.8 * losses[0], losses


def test_gradients_from_checkpoints_follow_those_without():
    """One step from the same state.  A code step is a / 127 with a about 2.9 standard deviations (the largest of 128
    normal values), so an activation read back is off by 2.9 / 127 / sqrt(12) = 0.7 % of its standard deviation; the
    quantizer behind it turns that into steps of a similar size, and two blocks add theirs: 5 % of a gradient's norm
    is far above that and far below a wrong gradient."""
    nets = [lm_step.QuantizedLm(T, V, D, F, blocks=2, checkpoint=c) for c in (True, False)]
    ids, labels = batch(3)
    before = [[w.clone() for b in n.blocks for w in b.W] for n in nets]
    losses = [float(n.step(ids, labels, lr=0.5)) for n in nets]
    assert losses[0] == losses[1]                                    # the forward does not read the checkpoints
    for w0, w1, a, b in zip(before[0], before[1], [w for k in nets[0].blocks for w in k.W],
                            [w for k in nets[1].blocks for w in k.W]):
        assert torch.equal(w0, w1)
        da, db = (a - w0).double(), (b - w1).double()
        assert float(db.norm()) > 0
        assert float((da - db).norm()) <= 0.05 * float(db.norm())
        touched = (db.abs().sum(dim=1) > 0)
        assert torch.equal(touched, da.abs().sum(dim=1) > 0) and 0 < int(touched.sum()) <= 0.1 * touched.numel() + 1
    for k0, k1 in zip(nets[0].blocks, nets[1].blocks):
        for name in ("dgamma", "dbeta"):
            g0, g1 = k0.gn[name].double(), k1.gn[name].double()
            assert float((g0 - g1).norm()) <= 0.05 * float(g1.norm())
    kept = nets[0].kept_bytes()
    assert kept == 2 * (T * (D + F) + 4 * T * (D + F) // 128)
    assert kept * 3 < 2 * 2 * T * 2 * (D + F)                        # against the four bf16 activations of a block


def test_shared_norm_outputs_need_one_shape():
    ctx = B.Context(0)
    first = B.LayerNormPlan(ctx, 8, 128, torch.bfloat16, "cuda")
    second = B.LayerNormPlan(ctx, 8, 128, torch.bfloat16, "cuda", outputs=first)
    assert second.y is first.y and second.dx is first.dx and second.mean is not first.mean
    with pytest.raises(ValueError):
        B.LayerNormPlan(ctx, 9, 128, torch.bfloat16, "cuda", outputs=first)
