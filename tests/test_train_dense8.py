"""The example that trains and serves a stack of 8-bit dense blocks: few rows, no steps, and the figures that it prints."""
import re

import pytest


def run(*argv):
    pytest.importorskip("torch")
    import train_dense8
    train_dense8.main(list(argv))


@pytest.mark.parametrize("argv", [("--steps", "0"), ("--steps", "-3"), ("--rows", "0")])
def test_nothing_to_do_is_refused(argv, capsys):
    with pytest.raises(SystemExit) as e:
        run(*argv)
    assert e.value.code == 2 and argv[0] in capsys.readouterr().err


@pytest.mark.gpu
def test_a_batch_smaller_than_what_is_served(capsys):
    run("--rows", "32", "--steps", "2")
    out = capsys.readouterr().out
    assert re.search(r"single rows: \d+ of 32 right", out), out
    # h and the normed rows of five norms, the hidden rows of four blocks, two bytes a value
    whole = 32 * (5 * 2 * 1024 + 4 * 4096) * 2
    assert "(in storage type it would be %.1f)" % (whole / 1e6) in out, out
    run("--rows", "5", "--steps", "1", "--blocks", "0", "--dtype", "f32")         # a norm and the output layer
    assert "of 5 right" in capsys.readouterr().out
