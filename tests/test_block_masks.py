"""Masks of a block's dropouts are a worker's own: drawn from its number and iteration, whatever other workers share its wave."""
import numpy as np
import pytest
import torch

from oracle import layers as ol
from paper_1902_01064_amd import block as bl
from paper_1902_01064_amd import hop, inputs
from test_block import DEV, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width,hidden,counts", [(24, 40, [3, 0, 5]), (130, 77, [33, 70]), (64, 256, [1])])
@pytest.mark.parametrize("indexed", [True, False])
def test_a_block_with_masks_of_every_group(width, hidden, counts, indexed):
    p, seed = 0.25, 9
    block = bl.ResidualBlock(width, hidden, scale=0.7, p=p)
    G, T = len(counts), sum(counts)
    begin = np.concatenate([[0], np.cumsum(counts)])
    rb = torch.from_numpy(begin.astype(np.int32)).to(DEV)
    torch.manual_seed(1)
    vectors = torch.randn(2 * G if indexed else G, block.d + 8, device=DEV) * 0.3
    index = [2 * g + 1 for g in range(G)] if indexed else None
    grads = torch.full((G, block.d), 7.0, device=DEV)
    x, dout = torch.randn(T, width, device=DEV), torch.randn(T, width, device=DEV)
    params = block.views(vectors)
    draws = [(3 * g + 2, 40 - g, n) for g, n in enumerate(counts)]
    out, saved = block.forward(params, index, x, rb, seed=seed, draws=draws)
    dx = block.backward(params, index, saved, dout, rb, block.views(grads), list(range(G)) if indexed else None)
    leaves = {k: v[index or list(range(G))].double().cpu().requires_grad_(True) for k, v in params.items()}
    x64 = x.double().cpu().requires_grad_(True)
    outs = []
    for g, (worker, it, n) in enumerate(draws):
        r = slice(int(begin[g]), int(begin[g + 1]))
        masks = [torch.from_numpy(ol.mask((p, seed, worker, it, site, 0), n, cols)) for site, cols in ((1, hidden), (2, width))]
        outs.append(reference(block, {k: v[g] for k, v in leaves.items()}, x64[r], *masks))
    want = torch.cat(outs)
    want.backward(dout.double().cpu())

    def near(got, ref, what):
        # eight chained operators, each within a few hundred roundings of 2^-24 of its magnitudes
        got, ref = got.double().cpu(), ref.detach()
        assert (got - ref).norm() <= 1e-5 * ref.norm() + 1e-12, (what, float((got - ref).norm()), float(ref.norm()))
    near(out, want, "out")
    near(dx, x64.grad, "dx")
    for k, v in block.views(grads).items():
        near(v, leaves[k].grad, k)
    with pytest.raises(ValueError):
        block.forward(params, index, x, rb, draws=draws[:-1])
    with pytest.raises(ValueError):
        block.forward(params, index, x, rb, draws=draws[:-1] + [(1, 1, counts[-1] + 1)])


def test_gradients_do_not_depend_on_the_schedule():
    """With steps of length zero every replica stays where it began, so a worker's gradient at an iteration is a matter of its samples and masks
    alone; schedules with other delays put it into other waves, among other workers."""
    N, K = 5, 6
    seen, company = [], []
    for kind in (inputs.DELAY_NONE, inputs.DELAY_EXP1):
        block = bl.ResidualBlock(32, 48, p=0.3)
        data, _ = bl.teacher_data(block, N, 100, 3)
        t = bl.Training(block, inputs.ring(N), data, K, batch=20, lr=0.0, seed=11, delay_kind=kind)
        try:
            s, got, waves = t.schedule, {}, {}
            for w in range(s.n_waves):
                t.wave(w)
                records = s.wave_order[s.wave_begin[w]:s.wave_begin[w + 1]]
                for e in records:
                    if s.kind[e] == hop.HOP_STEP:
                        at = (int(s.worker[e]), int(s.iter[e]))
                        got[at] = t.external[at[0]].double().cpu()
                        waves[at] = sorted(int(s.worker[o]) for o in records if s.kind[o] == hop.HOP_STEP)
            seen.append(got)
            company.append(waves)
        finally:
            t.close()
    assert seen[0].keys() == seen[1].keys() == {(i, k) for i in range(N) for k in range(K)}
    assert any(company[0][at] != company[1][at] for at in company[0])
    for at in seen[0]:                                     # products of other sizes sum in another order: roundings, as above
        assert (seen[0][at] - seen[1][at]).norm() <= 1e-5 * seen[0][at].norm(), at
