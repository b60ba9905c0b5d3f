"""The command of the residual network beyond the losses that a run keeps."""
import re
import sys

import pytest

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
