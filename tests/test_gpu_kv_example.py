"""The routed sessions of examples/routed_turns.py: what follows a hit equals the whole prompt's
outputs up to two roundings of the weights and the outputs (values of at most about 5)."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_routed_turns(dev, capsys):
    spec = importlib.util.spec_from_file_location("routed_turns", os.path.join(ROOT, "examples", "routed_turns.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    worst = m.main()
    assert worst <= 4 * 2.0 ** -8 * 5
    said = capsys.readouterr().out.splitlines()
    held = [int(line.split(" tokens, ")[1].split()[0]) for line in said if line.startswith("turn ")]
    assert held[0] == 0 and held[1] > 0 and held[2] > 0
