"""Replicas with little room: what fits is served, what does not is refused by name."""
import pytest

from paper_2609_29160_gb300 import served

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages,positions,chunk", [(8, 64, 128), (512, 256, 128), (5, 4096, 16), (2, 32, 1)])
def test_small_replicas_serve_what_fits(pages, positions, chunk):
    rep = served.Replica(pages=pages, page=16, max_positions=positions, chunk=chunk)
    done = rep.serve([(0, 12, 4), (0, 20, 5), (1, 1, 1)])
    assert sorted(r["L_in"] for r in done) == [1, 12, 20]
    assert sorted(rep.free) == list(range(pages))


def test_prompt_weight_wants_its_place():
    for size in (dict(pages=8, max_positions=4096), dict(pages=512, max_positions=256)):
        rep = served.Replica(page=16, chunk=128, **size)
        with pytest.raises(ValueError, match="prompt_weight"):
            rep.prompt_weight()
        assert sorted(rep.free) == list(range(size["pages"]))
        assert rep.prompt_weight(requests=2, context=0, times=1) > 0 if size["pages"] > 8 else True


def test_no_pages_at_all():
    with pytest.raises(ValueError, match="pages"):
        served.Replica(pages=0, page=16).serve([(0, 1, 1)])
