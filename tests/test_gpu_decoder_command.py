"""The decoder command's own use of streams."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_eager_steps_run_where_their_inputs_are_made(monkeypatch, capsys):
    """Positions, lengths and tokens are made on the current stream: a step on another
    one would have to wait for it."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_11357_amd import decoder
    seen, step = [], decoder.Stack.__call__

    def recorded(self, *args, **kw):
        if not torch.cuda.is_current_stream_capturing():
            seen.append(torch.cuda.current_stream())
        return step(self, *args, **kw)

    monkeypatch.setattr(decoder.Stack, "__call__", recorded)
    decoder.main(["--layers", "1", "--prompt", "64", "--batch", "2", "--steps", "2"])
    assert len(seen) == 5 and all(s == torch.cuda.current_stream() for s in seen)      # four prompts, one decode step
    assert "us a step" in capsys.readouterr().out
