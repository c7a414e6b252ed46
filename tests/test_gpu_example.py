"""GPU test (run with -m gpu): the decode worker of examples/ with few tokens; its last attention against 64-bit values of the rows
that the cache then held."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt,steps,drafts", [(100, 3, 7), (1, 1, 1), (33, 2, 64)])
def test_decode_worker(prompt, steps, drafts):
    import decode_worker
    tokens, back, (q, k, v, out, past) = decode_worker.run(prompt, steps, drafts, layers=2, kv_heads=2, q_heads=6)
    assert prompt + steps <= tokens <= prompt + steps * drafts
    assert torch.isfinite(back.float()).all()
    # the first draft sees the context and itself.  Against the rows as they are read back (K rounded once more) and its own row before
    # it was quantised (K in steps of a few hundredths, V in steps of a fifteenth of its range of some 5: half a step is 0.17)
    for h in range(6):
        keys = torch.cat([back[-1, 0, h // 3, :past], k[:1, h // 3]]).double().cpu().numpy()
        values = torch.cat([back[-1, 1, h // 3, :past], v[:1, h // 3]]).double().cpu().numpy()
        s = keys @ q[0, h].double().cpu().numpy() / np.sqrt(128)
        w = np.exp(s - s.max())
        assert np.abs(out[0, h].double().cpu().numpy() - w @ values / w.sum()).max() <= 0.25
