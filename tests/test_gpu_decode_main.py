"""The decoding example as a command: its flags' ends, and the lengths that it ends with."""

import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from examples import decode as ex  # noqa: E402


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("prompt,chunk", [(0, 0), (1, 0), (1, 7), (80, 0), (80, 32), (80, 1000)], ids=str)
def test_prompts_and_chunks(prompt, chunk, cache, monkeypatch, capsys):
    """A prompt has one token at least, and is 37 tokens shorter than the one before it."""
    monkeypatch.setattr(sys, "argv", ["decode", "--batch", "3", "--prompt", str(prompt), "--chunk", str(chunk), "--new", "2",
                                      "--cache", cache])
    ex.main()
    lens = [max(1, prompt - 37 * b) for b in range(3)]
    out = capsys.readouterr().out
    assert f"prompts: {sum(lens)} tokens" in out and f"lengths {[n + 2 for n in lens]}" in out


@pytest.mark.parametrize("flags", [["--chunk", "-1"], ["--prompt", "-5"]], ids=" ".join)
def test_flags_that_are_refused(flags, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["decode", *flags])
    with pytest.raises(SystemExit):
        ex.main()
    assert flags[0] in capsys.readouterr().err
