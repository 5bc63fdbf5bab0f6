"""The 8-bit rollout example without decode steps: prompts alone."""
import pytest
import torch

from examples import rollout_8bit as E
from paper_2602_09578_amd import binding as B

pytestmark = pytest.mark.gpu


def test_no_steps(monkeypatch):
    """No attention call has written the decoder's workspace, so its flags are not looked at, whatever the memory held before."""
    print("case: 8-bit rollout, no steps", flush=True)
    alloc = B.alloc_workspace
    monkeypatch.setattr(B, "alloc_workspace", lambda n, device: alloc(n, device).fill_(0xFF))
    r = E.run(2, 3, 40, 0, seed=1)
    assert r.out.shape == (6, E.HIDDEN) and bool(torch.isfinite(r.out.float()).all()) and not bool(r.decoder.suffix_lens.any())
