"""The decoding loop with `sampling`, step by step against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import inputs, sampler

from .test_sample import DEV, choose

gpu = pytest.mark.gpu


def _replay(sampling, seed, mask_gain):
    """A run and, from the steps' logits, what each step had to reveal; the mask token's logits are `mask_gain` times as large as others."""
    from .parity_util import to_dev
    cfg = inputs.model_shape("tiny")
    weights = inputs.make_weights(cfg, 31, dtype=torch.float32)
    weights["lm_head"][-1] *= mask_gain
    B, N, n_prompt, block, steps, k = 2, 96, 64, 16, 16, 2
    ctx = SL.surelock_init(cfg, to_dev(weights), N, B)
    tokens, mask = (x.to(DEV) for x in inputs.make_tokens(B, N, n_prompt, cfg["vocab"], 6))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    seen, ran_into_mask = [], 0

    def look(t, out, lock_in, lock_out, tok, msk):
        nonlocal ran_into_mask
        n = int(out.n_active.item())
        u = torch.empty(B * N, device=DEV).uniform_(generator=gen).tolist()
        idx, logits = out.active_idx[:n].tolist(), out.logits[:n].cpu().double().numpy()
        before, m = tok.cpu().numpy().copy().reshape(-1), msk.cpu().numpy().copy().reshape(-1)
        if seen:
            assert np.array_equal(seen[-1][0], before) and np.array_equal(seen[-1][1], m)       # the last step revealed what it had to
        blk = t // (block // k)
        for b in range(B):
            rows = [r for r in range(n) if idx[r] // N == b and n_prompt + blk * block <= idx[r] % N < n_prompt + (blk + 1) * block and m[idx[r]]]
            drawn, conf = {}, {}
            for r in rows:
                T = float(np.float32(sampling.get("temperature", 1.0)))
                drawn[r] = choose(logits[r, :-1], float(np.float32(u[r])), T, sampling.get("top_k", 0), float(np.float32(sampling.get("top_p", 1.0))))[0]
                z = np.exp(logits[r] - logits[r].max())
                conf[r] = z[drawn[r]] / z.sum()
                ran_into_mask += int(logits[r].argmax() == cfg["vocab"] - 1)
            for r in sorted(rows, key=lambda r: -conf[r])[:k]:
                before[idx[r]], m[idx[r]] = drawn[r], 0
        seen.append((before, m))

    sampler.run(ctx, tokens, mask, n_prompt, block, steps, 1e-3, unmask_per_step=k, sampling=dict(sampling, seed=seed), observer=look)
    assert np.array_equal(seen[-1][0], tokens.cpu().numpy().reshape(-1)) and not mask.any()
    return tokens[:, n_prompt:].cpu(), ran_into_mask


@pytest.mark.parametrize("sampling", [dict(topk=4), dict(temperature=1.0, Seed=3)])
def test_unknown_settings_are_refused(sampling):
    with pytest.raises(SL.SurelockError, match="topk|Seed"):
        sampler.run(None, torch.zeros(1, 8, dtype=torch.int32), torch.ones(1, 8, dtype=torch.uint8), 4, 4, 1, 1e-3, sampling=sampling)


@gpu
@pytest.mark.parametrize("sampling", [dict(temperature=0.0), dict(top_k=1), dict(temperature=1.0), dict(temperature=0.7, top_k=40, top_p=0.9)])
@pytest.mark.parametrize("mask_gain", [1.0, 40.0])
def test_the_mask_token_is_not_drawn(sampling, mask_gain):
    """Its logits are made the largest of about every second row: it takes no place in the filters, is not drawn, and does not come out as
    token 0, which is what the unmasking writes for it."""
    tokens, ran_into_mask = _replay(sampling, 5, mask_gain)
    assert int(tokens.max()) < 2047 and (mask_gain == 1.0 or ran_into_mask > 50)
    assert int((tokens == 0).sum()) <= 1
