"""The example's decode loop: every text that it makes is one that its grammar accepts, and a second run makes the same texts."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")
    spec = importlib.util.spec_from_file_location("decode_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_decodes_what_its_grammar_accepts():
    import paper_2411_15100_amd as xgm

    example = _example()
    rows, steps, runs = 6, 40, []
    for _ in range(2):
        d = example.Decoder(rows, steps, seed=3)
        for k in range(steps):
            d.step(k)
        assert not d.states.status(example.wl.current_stream()).any()
        runs.append(d.texts())
    assert runs[0] == runs[1]
    assert len({tuple(t) for t in runs[0]}) > 1
    for ids in runs[0]:
        m = xgm.Matcher(cache=d.cache)
        assert ids and all(m.try_accept_token(t) == 0 for t in ids)
        assert len(ids) == steps or m.is_terminated()
