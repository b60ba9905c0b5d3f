"""The command of the residual network beyond the losses that a run keeps."""
import re
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1908_11848_amd import residual_mlp as R             # noqa: E402


def losses(monkeypatch, capsys, pushes):
    monkeypatch.setattr(sys, "argv", ["residual_mlp", "--type", "fp32", "--width", "16", "--hidden", "16", "--depth", "0", "--batch", "2", "--workers", "1", "--pushes", str(pushes)])
    R.main()
    return re.search(r"%d pushes, .* mean loss (\S+) -> (\S+)" % pushes, capsys.readouterr().out).groups()


def test_more_pushes_than_losses_are_kept_by_default(monkeypatch, capsys):
    """A worker of 4100 iterations: the first loss is still the first one's, the last one is there."""
    first, last = losses(monkeypatch, capsys, 4100)
    assert first == losses(monkeypatch, capsys, 8)[0]
    assert float(last) < float(first)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
def test_a_step_copies_only_what_changes_its_type(type, monkeypatch):
    """fp32: no copy at all. bf16: the last norm's output is widened for the pooling, by torch; everything else is the launchers'."""
    t = R.Training(width=32, hidden=64, depth=1, batch=3, K=1, type=type)
    t.step(0, 0)                        # weights are whatever is there; only the calls count
    copies = []
    plain = torch.Tensor.copy_
    monkeypatch.setattr(torch.Tensor, "copy_", lambda self, src, *a: copies.append((src.dtype, self.dtype)) or plain(self, src, *a))
    t.step(0, 1)
    t.synchronize()
    t.close()
    assert copies == ([] if type == "fp32" else [(torch.bfloat16, torch.float32)])
