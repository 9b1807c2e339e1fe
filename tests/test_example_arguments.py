"""examples/speculative_decode.py refuses numbers that leave it nothing to do (before it touches a GPU)."""
import importlib.util
import os

import pytest

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")
_spec = importlib.util.spec_from_file_location("speculative_decode_arguments", _path)
sd = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(sd)


@pytest.mark.parametrize("option", ["--prompts", "--ways", "--length", "--rounds"])
@pytest.mark.parametrize("value", ["0", "-3"])
def test_numbers_have_to_be_above_zero(option, value, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["speculative_decode.py", f"{option}={value}"])
    with pytest.raises(SystemExit):
        sd.main()
    assert "is not above zero" in capsys.readouterr().err
