"""The example that runs the cache's calls together: a step's committed rows are
what the caches hold, the budget is kept, and drafts are accepted."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from examples import verify_with_cache as example
    prompt, steps, keep, recent = 130, 12, 140, 32
    accepted, model = example.run(requests=2, prompt=prompt, steps=steps, keep=keep, recent=recent)
    torch.cuda.synchronize()
    assert accepted.float().mean() > 1
    committed = prompt + (accepted + 1).sum(0)
    for cache in model.caches:
        assert torch.equal(cache.state[:, 1].long(), committed)
        assert torch.equal(cache.lengths.long(), committed.clamp(max=keep))
        for b in range(2):
            n = int(cache.lengths[b])
            held = cache.positions[b, :, :n].long()
            young = torch.arange(int(committed[b]) - recent, int(committed[b]), device=held.device)
            for h in range(held.shape[0]):
                assert held[h].unique().numel() == n and torch.isin(young, held[h]).all()
            assert (cache.positions[b, :, n:] == -1).all()
        assert torch.isfinite(cache.weights).all() and (cache.weights >= 0).all() and cache.weights.sum() > 0
