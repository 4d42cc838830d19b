"""examples/sampled_serving.py, up to where it needs a GPU."""
import importlib.util
import os

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sampled_serving.py")


class Stop(Exception):
    pass


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("sampled_serving", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("prompts, steps", [("1", 1), ("300,41,120", 32), ("5,32700", 70), ("40,7", 40000)])
def test_every_position_and_token_has_its_place(example, prompts, steps, monkeypatch):
    seen = {}

    def model(**kw):
        seen.update(kw)
        raise Stop

    monkeypatch.setattr(example, "Model", model)
    with pytest.raises(Stop):
        example.main(["--prompts", prompts, "--steps", str(steps)])
    lengths = [int(n) for n in prompts.split(",")]
    assert seen["positions"] > max(int(example.places(n + steps).max()) for n in lengths)
    assert seen["pages"] * seen["page"] >= len(lengths) * (max(lengths) + steps)


@pytest.mark.parametrize("length", [1, 8, 9, 31, 32, 33, 500])
def test_places_of_text_and_image(example, length):
    p = example.places(length)
    assert p.shape == (3, length) and p.dtype == torch.int32 and int(p.min()) >= 0 and int(p.max()) < max(length, 14)
    for i in range(length):
        if i < 8:
            want = [i] * 3
        elif i < 32:
            want = [8, 8 + (i - 8) // 6, 8 + (i - 8) % 6]
        else:
            want = [14 + i - 32] * 3
        assert p[:, i].tolist() == want


def test_axes_cover_every_pair(example):
    assert len(example.AXES) == 64 and set(example.AXES) == {0, 1, 2}


def test_help(example, capsys):
    with pytest.raises(SystemExit) as e:
        example.main(["--help"])
    assert e.value.code == 0 and "--no-graph" in capsys.readouterr().out
