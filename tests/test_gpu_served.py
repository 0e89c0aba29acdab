"""A served replica's requests: what its steps compute, and that the records and service
times it leaves are the library's own inputs."""
import numpy as np
import pytest
import torch

import paper_2609_29160_gb300 as tre
from paper_2609_29160_gb300 import served

pytestmark = pytest.mark.gpu

ARRIVALS = [(0, 70, 5), (0, 1, 1), (3, 200, 9), (10, 33, 20), (400, 16, 2)]


def test_chunks_and_batches_do_not_change_what_is_computed():
    """Last rows of a prompt in chunks beside other requests, against the prompt whole and
    alone: the same sums in another order, over keys rounded to bfloat16."""
    rows = {}
    for chunk in (16, 256):
        rep = served.Replica(chunk=chunk, seed=4)
        rep.serve(ARRIVALS[:2], seed=1)
        r = {"pages": [], "L_in": 200, "tokens": torch.arange(200, device="cuda") % 256}
        for at in range(0, 200, chunk):
            n = min(chunk, 200 - at)
            x = rep.forward(r["tokens"][at:at + n], rep._batch([(r, at, n)]))
        rows[chunk] = x[-1].double()
    # two layers, each of a handful of bfloat16 roundings of values of this size
    assert (rows[16] - rows[256]).norm() <= 2 * 8 * 2.0 ** -8 * rows[256].norm()


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "i8"])
def test_requests_run_to_their_ends(cache):
    rep = served.Replica(chunk=64, cache=cache, time_scale=4.0)
    done = rep.serve(ARRIVALS)
    assert len(done) == len(ARRIVALS) and sorted(rep.free) == list(range(512))
    assert 0 < rep.prompt_weight() < 100 and sorted(rep.free) == list(range(512))
    for r in done:
        assert r["t_arr"] <= r["t_start"] <= r["t_first"] <= r["t_end"]
        assert len(r["tokens"]) == r["L_in"] + r["L_out"]
    assert sum(p for p, _, _ in rep.steps) == sum(a[1] for a in ARRIVALS)
    # a request's last token is not fed back
    assert sum(d for _, d, _ in rep.steps) == sum(a[2] - 1 for a in ARRIVALS)


def test_few_pages_make_requests_wait():
    rep = served.Replica(pages=40, page=16, chunk=64, max_positions=640)
    done = rep.serve([(0, 400, 5), (0, 100, 5), (0, 130, 2)])          # 26, 7 and 9 pages
    by = {r["L_in"]: r for r in done}
    assert by[400]["t_start"] == by[100]["t_start"] == 0
    assert by[130]["t_start"] >= min(by[400]["t_end"], by[100]["t_end"])
    with pytest.raises(ValueError, match="pages"):
        served.Replica(pages=40, page=16, max_positions=900).serve([(0, 800, 5)])


def test_records_are_the_library_s_inputs():
    runs = [served.Replica(chunk=64, time_scale=8.0, seed=m).serve(ARRIVALS) for m in range(2)]
    rec = served.records(runs)
    window, M = 10, 2
    K = int(rec["t_end_ms"].max()) // window + 1
    diag = tre.new_diag()
    c = tre.tss_window_reduce(M, window, K, requests=rec, diag=diag)
    d = tre.read_diag(diag)
    assert d["dropped_range"] == d["dropped_model"] == d["dropped_order"] == 0
    assert c["P"].sum(0).tolist() == [sum(a[1] for a in ARRIVALS)] * M
    assert c["D"].sum(0).tolist() == [sum(a[2] for a in ARRIVALS)] * M
    lat = served.latent(rec)
    prof = {"w_p": 0.2, "w_q": 2.0, "alpha": 0.3, "theta": 10.0, "tau_crit": 0.8,
            "tau_surplus": 1.2}
    out, _, _ = tre.tre_replay(lat, M, window, K + 2000 // window, prof, 4, np.ones(M, np.int32),
                               np.ones(M, np.int32), np.ones(M, np.int32))
    assert out["served"].sum().item() == 2 * len(ARRIVALS)
