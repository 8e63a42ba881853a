"""The example of a decode step at its smallest, and what its command line refuses (the steps need an MI355X)."""
import sys

import pytest

from test_gpu_serving_step import example


@pytest.mark.parametrize("args", [["--steps", "0"], ["--steps", "-3", "--check"], ["--batch", "0"], ["--prompt", "0"]])
def test_nothing_to_do_is_refused(args, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["shared_prefix_decode.py", *args])
    with pytest.raises(SystemExit) as e:
        example().main()
    assert e.value.code == 2 and "at least 1" in capsys.readouterr().err


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["e4m3", "same"])
@pytest.mark.parametrize("batch,prompt,steps", [(2, 70, 1), (3, 1, 1), (2, 70, 2), (1, 1, 3)])
def test_few_steps_are_checked_too(batch, prompt, steps, cache):
    """The bar of test_gpu_serving_step.py."""
    layer, us, error = example().run(batch, prompt, steps, cache, check=True)
    assert int(layer.suffix_lens[0]) == steps and error <= 2.0 ** -6 and (us is None) == (steps < 3)
