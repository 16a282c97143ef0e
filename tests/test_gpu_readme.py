"""The README's example as it stands there, with buffers that nobody has written holding NaN."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_example(repo_root, monkeypatch):
    empty = torch.empty

    def unwritten(*args, **kw):
        x = empty(*args, **kw)
        x.view(torch.uint8).fill_(0xff)
        return x

    monkeypatch.setattr(torch, "empty", unwritten)
    with open(os.path.join(repo_root, "README.md")) as f:
        parts = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    assert len(parts) == 2
    it = {}
    for part in parts:
        exec(part, it)
    torch.cuda.synchronize()
    n = it["small_lens"][0].tolist()
    assert torch.isfinite(it["out"]).all() and torch.isfinite(it["o32"]).all() and torch.isfinite(it["o1"]).all()
    for h in range(it["Hkv"]):
        weight = it["kept_weight"][0, h]
        # the token appended last has what the rows of one step gave it
        assert torch.isfinite(weight[:n[h]]).all() and 0 < weight[n[h] - 1] < it["Hq"] // it["Hkv"]
        # every token had all 32 rows' attention to share; some went with the tokens that left
        assert 0 < weight[:n[h]].sum() < 33.01 * it["Hq"] // it["Hkv"]
