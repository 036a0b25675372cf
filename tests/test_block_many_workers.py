"""A block on more workers than a call of the layers has groups: waves and evaluations go in runs."""
import numpy as np
import pytest
import torch

from paper_1902_01064_amd import block as bl
from paper_1902_01064_amd import hop, inputs, layers


def test_runs_hold_every_worker_once():
    most = layers.HOP_MAX_INDEXED
    for n in (0, 1, most, most + 1, 3 * most + 7):
        runs = bl._runs(list(range(n)))
        assert [i for r in runs for i in r] == list(range(n)) and all(1 <= len(r) <= most for r in runs) and len(runs) == -(-n // most)


@pytest.mark.gpu
def test_300_workers():
    N, width, batch = 300, 16, 4
    block = bl.ResidualBlock(width, 24, p=0.2)
    data, held = bl.teacher_data(block, N, 8, 3)
    t = bl.Training(block, inputs.ring(N), data, 3, batch=batch, lr=2.0, seed=11, delay_kind=inputs.DELAY_NONE)
    try:
        s = t.schedule
        sizes = [int((s.kind[s.wave_order[s.wave_begin[w]:s.wave_begin[w + 1]]] == hop.HOP_STEP).sum()) for w in range(s.n_waves)]
        assert max(sizes) > layers.HOP_MAX_INDEXED
        first = t.evaluate(*held)
        assert first.shape == (N,) and torch.allclose(first, first[:1].expand(N), rtol=1e-5)       # all replicas are the same
        for w in range(s.n_waves):
            before = t.params["w1"].clone()
            index = t.versions(range(N))
            loss = t.wave(w)
            records = [e for e in s.wave_order[s.wave_begin[w]:s.wave_begin[w + 1]] if s.kind[e] == hop.HOP_STEP]
            got = t.external.clone()
            assert torch.isfinite(got).all() and bool(torch.isfinite(loss))
            if w:
                continue
            alone = []                                     # every worker by itself, from the replicas before the wave (slot 0: as they began)
            for e in records:
                i = int(s.worker[e])
                assert torch.equal(t.params["w1"][index[i]], before[index[i]])
                rows = torch.from_numpy(s.batch_rows[e].astype(np.int64)).cuda()
                out, saved = block.forward(t.params, [index[i]], t.x[i][rows], None, t.seed, draws=[(i, int(s.iter[e]), batch)])
                diff = out - t.target[i][rows]
                alone.append(float(diff.square().mean()) / 2)
                g = torch.zeros(1, block.d, device="cuda")
                block.backward(t.params, [index[i]], saved, diff / (batch * width), None, block.views(g), [0])
                assert (got[i] - g[0]).norm() <= 1e-5 * g.norm(), i
            assert abs(float(loss) - np.mean(alone)) <= 1e-5 * np.mean(alone)
        assert float(t.evaluate(*held).mean()) < float(first.mean())
    finally:
        t.close()
