"""The generators that modules have of their own: each process's under DistributedDataParallel, and saved, loaded and moved with
the modules.  On the CPU."""
import copy
import io
import os

import pytest
import torch

from paper_2306_06098_b200.dropout import Dropout, take
from paper_2306_06098_b200.norm import RMSNorm
from test_multiprocess import json_lines, torchrun


def test_each_process_has_its_own():
    r = torchrun([os.path.join("tests", "rng_worker.py")])
    assert r.returncode == 0, r.stderr[-2000:]
    rows = sorted(json_lines(r.stdout), key=lambda x: x["rank"])
    assert [x["shared"] for x in rows] == [0.0, 0.0]  # (buffers become the first one's)
    assert rows[0]["seeds"] != rows[1]["seeds"]
    for x in rows:
        assert x["taken"] == [[s, k] for k in range(2) for s in x["seeds"]]


def model(seed):
    return torch.nn.Sequential(Dropout(0.5, seed=seed), RMSNorm(4, p=0.25, seed=seed + 1), RMSNorm(4))


def states(m):
    return [k.rng.tolist() for k in m if k.rng is not None]


@pytest.mark.parametrize("assign", [False, True])
def test_saved_and_loaded(assign):
    a, b = model(1), model(7)
    take(a[0].rng)
    assert list(a.state_dict()) == ["0.rng", "1.weight", "1.rng", "2.weight"]
    f = io.BytesIO()
    torch.save(a.state_dict(), f)
    f.seek(0)
    assert not any(b.load_state_dict(torch.load(f), assign=assign))
    assert states(b) == states(a) == [[1, 1], [2, 0]]
    take(b[1].rng)
    assert states(a)[1] == [2, 0]
    assert states(copy.deepcopy(b)) == states(b)


def test_what_does_not_fit_is_refused():
    m, full = model(1), model(2).state_dict()
    short = {k: v for k, v in full.items() if k != "1.rng"}
    with pytest.raises(RuntimeError, match="1.rng"):
        m.load_state_dict(short)
    assert m.load_state_dict(short, strict=False).missing_keys == ["1.rng"]
    with pytest.raises(RuntimeError, match="2.rng"):
        m.load_state_dict({**full, "2.rng": torch.zeros(2, dtype=torch.int64)})
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(2)):
        with pytest.raises(RuntimeError, match="seed, offset"):
            m.load_state_dict({**full, "0.rng": bad})


def test_moved():
    m = model(1)
    assert [k.rng.device.type for k in m.to("meta") if k.rng is not None] == ["meta", "meta"]
    m = model(1).half()
    assert m[0].rng.dtype == torch.int64 and states(m) == [[1, 0], [2, 0]]
