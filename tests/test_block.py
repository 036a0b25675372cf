"""The residual block on all replicas: its gradients against torch's differentiation of the same formulas in 64 bits, and a run of
decentralized workers on them."""
import numpy as np
import pytest
import torch

from oracle import layers as ol
from paper_1902_01064_amd import block as bl
from paper_1902_01064_amd import hop, inputs, layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def reference(block, p, x, drop1, drop2):
    """Output of one replica for its rows, in 64 bits; the masks come from the oracle's generator."""
    def norm(v):
        return v / torch.sqrt(v.square().mean(1, keepdim=True) + block.eps)
    h = norm(x) * p["pre"]
    a = torch.relu(h @ p["w1"].T) * drop1
    return norm(x + block.scale * (norm(a @ p["w2"].T) * p["post"] * p["gate"]) * drop2) * p["head"]


@pytest.mark.parametrize("width,hidden,counts,p", [(24, 40, [3, 0, 5], 0.25), (130, 77, [33, 70], 0.0), (64, 256, [1], 0.5)])
def test_gradients_of_the_whole_block(width, hidden, counts, p):
    block = bl.ResidualBlock(width, hidden, scale=0.7, p=p)
    G, T = len(counts), sum(counts)
    begin = np.concatenate([[0], np.cumsum(counts)])
    rb = torch.from_numpy(begin.astype(np.int32)).to(DEV)
    torch.manual_seed(1)
    arena = torch.randn(2 * G, block.d + 8, device=DEV) * 0.3
    index = [2 * g + 1 for g in range(G)]
    grads = torch.full((G + 1, block.d), 7.0, device=DEV)
    where = list(range(1, G + 1))
    x, dout = torch.randn(T, width, device=DEV), torch.randn(T, width, device=DEV)
    params = block.views(arena)
    out, saved = block.forward(params, index, x, rb, seed=9, it=4)
    dx = block.backward(params, index, saved, dout, rb, block.views(grads), where)
    masks = [torch.from_numpy(ol.mask((p, 9, 0, 4, site, 0), T, n)) for site, n in ((1, hidden), (2, width))]
    leaves = {k: v[index].double().cpu().requires_grad_(True) for k, v in params.items()}
    x64 = x.double().cpu().requires_grad_(True)
    outs = []
    for g in range(G):
        r = slice(int(begin[g]), int(begin[g + 1]))
        outs.append(reference(block, {k: v[g] for k, v in leaves.items()}, x64[r], masks[0][r], masks[1][r]))
    want = torch.cat(outs)
    want.backward(dout.double().cpu())

    def near(got, ref, what):
        # eight chained operators, each within a few hundred roundings of 2^-24 of its magnitudes
        got, ref = got.double().cpu(), ref.detach()
        assert (got - ref).norm() <= 1e-5 * ref.norm() + 1e-12, (what, float((got - ref).norm()), float(ref.norm()))
    near(out, want, "out")
    near(dx, x64.grad, "dx")
    for k, v in block.views(grads[1:]).items():
        near(v, leaves[k].grad, k)
    assert (grads[0] == 7.0).all()


def test_workers_learn_and_every_step_is_the_schedules():
    """A ring of workers with Exp(1) delays: the held-out loss falls, and each replica is what Reduce and Apply of the recorded gradients give."""
    block = bl.ResidualBlock(32, 48, p=0.1)
    N, K = 5, 30
    data, held = bl.teacher_data(block, N, 200, 3)
    t = bl.Training(block, inputs.ring(N), data, K, batch=20, lr=8.0, seed=11)
    try:
        sched = t.schedule
        sess = t.session
        rings = np.zeros((N, sess.D, block.d))
        rings[:] = block.initial(11).numpy()
        first = float(t.evaluate(*held).mean())
        for w in range(sched.n_waves):
            t.wave(w)
            g = t.external.double().cpu().numpy()
            new = []
            for e in sched.wave_order[sched.wave_begin[w]:sched.wave_begin[w + 1]]:
                i, src = int(sched.worker[e]), range(sched.src_begin[e], sched.src_begin[e + 1])
                mean = sum(float(sched.src_weight[a]) * rings[sched.src_worker[a], sched.src_slot[a]] for a in src)
                new.append((i, int(sched.out_slot[e]), mean - (8.0 * g[i] if sched.kind[e] == hop.HOP_STEP else 0.0)))
            for i, slot, v in new:
                rings[i, slot] = v
        got = sess.ring_snapshot()
        for i in range(N):
            slot = hop.hop_params(sess.ctx, i)[1] % sess.D
            ref = rings[i, slot]
            assert np.abs(got[i, slot] - ref).max() <= 1e-4 * np.abs(ref).max()      # 30 roundings of sums of four terms, and room
        last = float(t.evaluate(*held).mean())
        assert np.isfinite(last) and last < 0.7 * first, (first, last)
    finally:
        t.close()


def test_the_command():
    first, last = bl.main(["--workers", "4", "--width", "64", "--hidden", "128", "--samples", "256", "--batch", "32", "--iterations", "20"])
    assert last < first
