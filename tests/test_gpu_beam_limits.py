"""A beam search that runs into its cache's limits: the longest rows, and pools that run out."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _load(name, *path):
    spec = importlib.util.spec_from_file_location(name, os.path.join(ROOT, *path))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("window,sinks", [(None, 0), (21, 3), (33, 0)])
@pytest.mark.parametrize("heads,bs,most", [((4, 2, 64), 16, 40), ((28, 4, 128), 16, 33), ((8, 8, 64), 32, 64), ((4, 2, 64), 16, 15)])
def test_rows_grow_to_their_last_block(heads, bs, most, window, sinks):
    """Every step that gives a row a slot gives it an output too, up to whole blocks of
    ``max_length``; then its row finds no place and stays as it was."""
    room = -(-most // bs) * bs
    s = _load("beam_loop_search", "tests", "test_gpu_beam_loop.py").Search(heads, bs, window, sinks, (most - 2, most - 5), most, seed=most)
    s.prefill()
    for _ in range(room - (most - 2)):
        s.inputs()
        before = s.scores.clone()
        s.step()
        assert s.cache.stats[2].item() == 0 and s.cache.slots.ge(0).all()
        s.follow(before)
        assert s.fnpu.check() == 0
    assert s.cache.length.tolist() == [room] * 3 + [room - 3] * 3
    s.inputs()
    s.step()
    assert s.cache.stats[2].item() == 3 and s.cache.slots.view(-1)[:3].eq(-1).all() and s.cache.slots.view(-1)[3:].ge(0).all()
    assert s.cache.length.tolist() == [room] * 3 + [room - 2] * 3
    assert s.fnpu.check() == 0
    s.history = [s.history[p] for p in s.chosen[1].view(-1).tolist()]
    for layer in range(s.LAYERS):
        assert torch.isfinite(s.out[layer].float()).all() and torch.isfinite(s.lse[layer]).all()
        for r in range(3):                         # over the keys that they have
            s.check_row(r, layer, s.q[layer][r:r + 1], s.out[layer][r:r + 1], s.lse[layer][r:r + 1], room - 1)


def test_example_counts_the_rows_of_every_step(monkeypatch):
    """Rows that found no block in an early step are told, though later steps serve all."""
    import paper_2606_04415_gb300.beams as beams
    seen = []

    class Tight(beams.BeamCache):
        """A pool in which the first steps find no blocks: something else holds them until then."""

        def admit(self, lengths):
            got = super().admit(lengths)
            self.kept = self.refs.eq(0)
            self.refs[self.kept] = 1
            return got

        def advance(self, parents):
            if len(seen) == 3:
                self.refs[self.kept] -= 1
            super().advance(parents)
            seen.append(self.stats.clone())

    monkeypatch.setattr(beams, "BeamCache", Tight)
    got = _load("beam_search_loop", "examples", "beam_search_loop.py").main(
        ["--heads", "8", "2", "64", "--requests", "2", "--beams", "3", "--prompt", "32", "--tokens", "8", "--window", "40", "--vocab", "503", "--eager"])
    each = [int(x[2]) for x in seen]
    assert each[-1] == 0 and sum(each) > 0, each
    assert got["unserved"] == sum(each)
    assert np.isfinite(got["scores"]).all()
