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


@pytest.mark.parametrize("V", [1, 2, 3, 4, 5, 6, 7, 8, 9, 30, 4097, 8191, 8193, 8200, 16390])
def test_rows_at_every_alignment(V):
    """Rows that start and end at every place of 16 bytes, the first and the last of their storage among them; their neighbours would win."""
    import torch
    B, n = 3, 2
    g = torch.Generator().manual_seed(V)
    for off in range(4):
        for pad in range(4):
            stride = V + pad
            rows = []
            for count in (n + 1, n):
                store = torch.full((off + B * count * stride - pad,), 1e30)  # (nothing behind the last row)
                view = store.cuda().as_strided((B, count, V), (count * stride, stride, 1), off)
                x = torch.randn(B, count, V, generator=g) * 2
                view.copy_(x)
                rows.append((x, view))
            drafted = torch.randint(0, V, (B, n), generator=g).int()
            u, w = torch.rand(B, n, generator=g) * 0.5, torch.rand(B, generator=g)
            for temp in (torch.tensor([1.0, 0.5, 0.0]), torch.tensor([0.0, 2.0, 1.0])):
                tokens, accepted = _verify(rows[0][1], rows[1][1], drafted.cuda(), u.cuda(), w.cuda(), temp.cuda())
                for b in range(B):
                    out, a, clear = verified(rows[0][0][b].numpy(), rows[1][0][b].numpy(), drafted[b].tolist(), float(temp[b]), u[b].tolist(), float(w[b]), False)
                    assert not clear or (int(accepted[b]) == a and tokens[b].tolist() == out), (off, pad, b, tokens[b].tolist(), out)
