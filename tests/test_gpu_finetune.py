"""The fine-tuning example: every operator and the sparse layer in one training loop."""
import pytest
import torch

from paper_2501_08582_amd import finetune, ops, train

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,mask", [(train.RMS, ops.TWO_FOUR), (train.LAYER, ops.BITMAP)])
def test_preference_training_learns_and_serves(kind, mask):
    cfg = finetune.Config(vocab=512, width=128, hidden=256, pairs=6, length=33, prompt=5, kind=kind, mask=mask, lr=2e-3)
    trainer = finetune.Trainer(cfg)
    ids, targets = finetune.batch(cfg, 3)
    assert (ids < 0).any() and (targets < 0).any()
    ref = trainer.reference(ids, targets)
    # before any step the model is its reference: without dropout the loss is log 2
    loss, reward, _ = train.preference_loss(trainer.model.logits(ids), targets, ref, cfg.beta)
    assert abs(float(loss.detach()) - 0.693147) < 1e-6 and not reward.any()
    first, _ = trainer.step(ids, targets, ref)
    for _ in range(11):
        last, reward = trainer.step(ids, targets, ref)
    assert torch.isfinite(last) and float(last) < 0.5 * float(first)
    assert (reward[:cfg.pairs] > reward[cfg.pairs:]).all()
    assert any(p.detach().any() for k, p in trainer.params.items() if k.endswith(".B"))
    # one token at a time: the same model
    start = torch.arange(7, device="cuda").unsqueeze(1)
    told = trainer.model.generate(start, 3)
    assert told.shape == (7, 4)
    with torch.no_grad():
        logits = trainer.model.logits(told[:, :-1].contiguous())
    picked = logits.gather(2, told[:, 1:].unsqueeze(2)).squeeze(2)
    # the greedy token is the largest, up to the rounding of logits by calls of other lengths
    assert (picked >= logits.amax(2) - 2.0**-6 * logits.abs().amax(2)).all()
