"""examples/paged_decode.py, up to where it needs a GPU."""
import importlib.util
import os

import pytest

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")


class Stop(Exception):
    pass


@pytest.mark.parametrize("prefix, steps", [(0, 1), (1000, 64), (32700, 64), (5, 40000)])
def test_every_position_has_its_rotation(prefix, steps, monkeypatch):
    """prefix + steps + 2 positions: a step before the graph, one before the clock and `steps` behind it."""
    spec = importlib.util.spec_from_file_location("paged_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    seen = {}

    def decoder(**kw):
        seen.update(kw)
        raise Stop

    default = m.Decoder.__init__.__defaults__[m.Decoder.__init__.__code__.co_varnames[1:].index("positions")]
    monkeypatch.setattr(m, "Decoder", decoder)
    with pytest.raises(Stop):
        m.main(["--prefix", str(prefix), "--steps", str(steps)])
    assert seen.get("positions", default) >= prefix + steps + 2
