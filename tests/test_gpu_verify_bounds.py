"""Verification of drafts where its bounds are tight (B200 only)."""
import math

import numpy as np
import pytest

from test_gpu_cache8 import _verify, verified

pytestmark = pytest.mark.gpu


def test_a_draft_model_that_is_almost_the_target():
    """Two models that agree but for 2^-9 of their mass, and whose sums differ by a few 2^-27: what the common tokens have left over is all in that
    difference, and a draw falls among 2^18 small ones."""
    import torch
    B, V, common, small = 33, 270000, 3000, 1 << 18
    rng = np.random.default_rng(5)
    target = rng.uniform(-3, 3, (B, 2, V)).astype(np.float32)
    target[:, :, common:] = -math.inf
    draft = target[:, :1].copy()
    at = slice(common, common + small)
    for b in range(B):
        mass = np.exp(target[b, 0, :common].astype(np.float64)).sum()
        target[b, 0, at] = np.float32(math.log(mass * 2.0 ** -9 / small))
        # the draft's one token instead: the target's sum is larger by (b - 16) 2^-27
        only = np.exp(target[b, 0, at].astype(np.float64)).sum() - mass * (b - 16) * 2.0 ** -27
        draft[b, 0, V - 1] = np.float32(math.log(only))
    drafted = np.full((B, 1), V - 1, np.int32)  # (refused: the target does not have it)
    u, w = np.full((B, 1), 0.5, np.float32), (rng.random(B) * 0.5 + 0.5).astype(np.float32)
    dev = [torch.from_numpy(x).cuda() for x in (target, draft, drafted, u, w)]
    tokens, accepted = (x.cpu().numpy() for x in _verify(*dev))
    seen, wrong = 0, []
    for b in range(B):
        out, a, _ = verified(target[b], draft[b], drafted[b].tolist(), 1.0, u[b].tolist(), float(w[b]), False)
        p, q = (np.exp(x.astype(np.float64)) / np.exp(x.astype(np.float64)).sum() for x in (target[b, 0], draft[b, 0]))
        cum = np.cumsum(np.maximum(p - q, 0))
        # weights are good to 2^-39 of the sums, next to the 2^-9 that is left: 2^-28 of it holds (a small token has 2^-18 of it)
        if np.abs(cum - float(w[b]) * cum[-1])[at].min() > 2.0 ** -28 * cum[-1]:
            seen += 1
            if accepted[b] != a or tokens[b].tolist() != out:
                wrong.append((b, tokens[b].tolist(), out))
    assert not wrong and seen >= 0.9 * B, (seen, wrong)
