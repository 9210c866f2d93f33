"""Options of the decoding loop's command that only models with a context have: refused without one, before anything runs."""
import sys

import pytest

from paper_2403_10444_b200 import specdec


class Reached(Exception):
    pass


def command(monkeypatch, *options):
    def stop():
        raise Reached

    monkeypatch.setattr(specdec.bv, "load_library", stop)
    monkeypatch.setattr(sys, "argv", ["specdec", *options])
    specdec.main()


@pytest.mark.parametrize("option", [["--top-k", "50"], ["--min-p", "0.1"], ["--rotary", "10000"], ["--packed"]])
def test_what_needs_a_context_is_refused_without(monkeypatch, capsys, option):
    with pytest.raises(SystemExit) as e:
        command(monkeypatch, *option)
    assert e.value.code == 2 and option[0] + ": only with --context" in capsys.readouterr().err
    with pytest.raises(Reached):
        command(monkeypatch, *option, "--context", "8")


@pytest.mark.parametrize("options", [[], ["--top-p", "0.9"], ["--top-k", "0", "--min-p", "0"], ["--context", "8", "--packed", "--top-k", "5", "--min-p", "0.1", "--rotary", "10000"]])
def test_what_does_not_is_not(monkeypatch, options):
    with pytest.raises(Reached):
        command(monkeypatch, *options)
