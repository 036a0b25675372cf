"""A residual feed-forward block trained by decentralized workers on their own gradients.

The workers' replicas are the rings of a context; before every wave the gradients of all workers of that wave are computed at once by the calls
of `layers` - parameters read where they lie in the rings, gradients written into the buffer that HOP_GRAD_EXTERNAL reads - and
hop_step then reduces and applies them.

    h = norm(x) pre;  a = dropout(relu(w1 h));  y = x + scale dropout(gate norm(w2 a) post);  out = norm(y) head

    python -m paper_1902_01064_amd.block [--workers 16] [--width 256] [--hidden 1024] [--iterations 60]
"""
import argparse
import contextlib

import torch

from . import hop, inputs, layers
from .session import Session


class ResidualBlock:
    """Places of the block's parameters in a flat replica of `d` floats, and their gradients for many replicas at once."""

    def __init__(self, width, hidden, scale=1.0, p=0.1, eps=1e-5):
        self.width, self.hidden, self.scale, self.p, self.eps = width, hidden, scale, p, eps
        self.shapes = dict(pre=(width,), w1=(hidden, width), w2=(width, hidden), post=(width,), gate=(width,), head=(width,))
        self.places, at = {}, 0
        for name, shape in self.shapes.items():
            n = 1
            for s in shape:
                n *= s
            self.places[name] = (at, n)
            at += (n + 3) // 4 * 4                     # every tensor begins at a multiple of 16 bytes
        self.d = at

    def views(self, vectors):
        """{name: [rows, ...]} of a tensor [rows, at least d] whose rows are replicas (or gradients)."""
        return {k: vectors[:, at:at + n].unflatten(1, self.shapes[k]) for k, (at, n) in self.places.items()}

    def initial(self, seed):
        g = torch.Generator().manual_seed(seed)
        p = torch.zeros(self.d)
        for name, (at, n) in self.places.items():
            if name in ("w1", "w2"):
                p[at:at + n] = torch.randn(n, generator=g) * self.shapes[name][1] ** -0.5
            else:
                p[at:at + n] = 1.0 if name != "gate" else 0.5
        return p

    def forward(self, params, index, x, row_begin, seed=0, it=0, train=True, draws=None):
        """The block's output and what its gradient needs again.

        Masks are drawn for all rows together, from worker 0 and iteration `it`; with `draws`, [(worker, iteration, rows)] of every group
        (whose rows row_begin has to agree with), for each group from its worker and iteration, so they do not depend on which other groups there are.
        A call of the layers has one mask, so the calls that drop are then made group by group."""
        p = self.p if train else 0.0
        drops, groups = [(None, None)], [(x.shape[0], index, row_begin)]
        if p and draws is None:
            drops = [self._drops(p, seed, 0, it)]
        elif p:
            G = 1 if row_begin is None else row_begin.shape[0] - 1
            if len(draws) != G or sum(rows for _, _, rows in draws) != x.shape[0]:
                raise ValueError("draws: %d rows in %d groups are needed, got %s" % (x.shape[0], G, draws[:4]))
            drops = [self._drops(p, seed, worker, iteration) for worker, iteration, _ in draws]
            groups = [(rows, [i if index is None else index[i]], None) for i, (_, _, rows) in enumerate(draws)]
        sizes = [rows for rows, _, _ in groups]
        h = layers.norm(x, params["pre"], row_begin, index, eps=self.eps)
        u = layers.product(h, params["w1"], row_begin, index)
        a = torch.relu(u)
        if p:
            self._dropout(a, sizes, drops)
        v = layers.product(a, params["w2"], row_begin, index)
        y, out = torch.empty_like(x), torch.empty_like(x)
        how = dict(post=params["post"], gate=params["gate"], scale=self.scale, next_norm="rms", pre=params["head"], eps=self.eps)
        for (_, where, begin), (_, drop), *t in zip(groups, drops, *(m.split(sizes) for m in (x, v, y, out))):
            layers.residual(t[0], t[1], begin, where, drop=drop, out=t[2], out_next=t[3], **how)
        return out, (x, h, u, a, v, y, groups, drops)

    def _drops(self, p, seed, worker, iteration):
        return layers.Drop(p, seed, worker, iteration, 1), layers.Drop(p, seed, worker, iteration, 2)

    def _dropout(self, a, sizes, drops):
        for part, (drop, _) in zip(a.split(sizes), drops):
            layers.dropout(part, drop, out=part)

    def backward(self, params, index, saved, dout, row_begin, grads, grad_index):
        """Writes the gradients of all parameters into the rows grad_index of `grads`; returns the gradient of x."""
        x, h, u, a, v, y, groups, drops = saved
        sizes = [rows for rows, _, _ in groups]
        dy, db = torch.empty_like(x), torch.empty_like(x)
        how = dict(post=params["post"], gate=params["gate"], scale=self.scale, next_norm="rms", pre=params["head"], eps=self.eps, dpost=grads["post"],
                   dpre=grads["head"], dgate=grads["gate"])
        to = [grad_index] if len(groups) == 1 else [[i if grad_index is None else grad_index[i]] for i in range(len(groups))]
        for (_, where, begin), (_, drop), i, *t in zip(groups, drops, to, *(m.split(sizes) for m in (dout, y, v, dy, db))):
            layers.residual_grad(None, t[0], t[1], t[2], begin, where, drop=drop, grad_index=i, dx=t[3], db=t[4], **how)
        layers.product_grad(db, a, row_begin, out=grads["w2"], index=grad_index)
        da = layers.product(db, params["w2"], row_begin, index, transposed=True)
        if drops[0][0]:
            self._dropout(da, sizes, drops)
        da = da * (u > 0)
        layers.product_grad(da, h, row_begin, out=grads["w1"], index=grad_index)
        dh = layers.product(da, params["w1"], row_begin, index, transposed=True)
        dx, _ = layers.norm_grad(dh, x, params["pre"], row_begin, index, eps=self.eps, dy=dy, dpre=grads["pre"], grad_index=grad_index)
        return dx


def _runs(items):
    """Workers in runs of as many groups as a call with an index takes."""
    return [items[i:i + layers.HOP_MAX_INDEXED] for i in range(0, len(items), layers.HOP_MAX_INDEXED)]


class Training:
    """Workers on a graph that learn a block from their own samples (x, target), [samples, width] each."""

    def __init__(self, block, in_nbrs, data, K, batch=64, s=2, b=0, lr=0.5, momentum=0.0, seed=inputs.DEFAULT_SEED, delay_kind=inputs.DELAY_EXP1,
                 mult=None, device="cuda:0"):
        N = len(in_nbrs)
        self.block, self.batch, self.seed = block, batch, seed
        c = dict(in_nbrs=in_nbrs, W=inputs.uniform_weights(in_nbrs), N=N, d=block.d, s=s, b=b, max_ig=0, skip_on=False, max_skip=10, trigger=1,
                 lr=lr, lam=0.0, batch=batch, seed=seed, momentum=momentum, model="external", K=K, delay_kind=delay_kind, mult=mult)
        self.session = sess = Session(c, device)
        self.stream = torch.cuda.current_stream(sess.dev)                # the one that the session took
        self.x = torch.stack([x for x, _ in data]).to(sess.dev)
        self.target = torch.stack([t for _, t in data]).to(sess.dev)
        self.external = torch.zeros(N, block.d, device=sess.dev)
        hop.hop_set_grad_source(sess.ctx, hop.HOP_GRAD_EXTERNAL, 0.0, self.external.data_ptr())
        for i in range(N):
            hop.hop_set_rows(sess.ctx, i, self.x.shape[1])
        sess.set_params(block.initial(seed))
        self.schedule = sess.simulate(K)
        rows = N * sess.D
        self.params = block.views(sess.arena[:rows * sess.stride].view(rows, sess.stride))
        self.grads = block.views(self.external)

    def versions(self, workers):
        """Rows of the arena that hold the workers' newest parameters."""
        base = self.session.arena.data_ptr()
        return [(hop.hop_params(self.session.ctx, w)[0] - base) // (4 * self.session.stride) for w in workers]

    @contextlib.contextmanager
    def _session_stream(self):
        """Layers read the rings that hop_step writes and write the gradients that it reads, so they run where it does, on the session's stream:
        behind what the caller's stream holds now, and before what comes there next.  Yields the caller's stream."""
        caller = torch.cuda.current_stream(self.session.dev)
        if caller == self.stream:
            yield caller
            return
        self.stream.wait_stream(caller)
        try:
            with torch.cuda.stream(self.stream):
                yield caller
        finally:
            caller.wait_stream(self.stream)

    def wave(self, w):
        """One wave: gradients of its workers, then hop_step.  Returns the mean loss over its minibatches (on the GPU), or None."""
        with self._session_stream() as caller:
            loss = self._wave(w)
            if loss is not None and caller != self.stream:
                loss.record_stream(caller)
        return loss

    def _wave(self, w):
        sched = self.schedule
        records = [e for e in sched.wave_order[sched.wave_begin[w]:sched.wave_begin[w + 1]] if sched.kind[e] == hop.HOP_STEP]
        losses = [(self._gradients(run), len(run)) for run in _runs(records)]
        hop.hop_step(self.session.ctx, sched, w, w + 1)
        if len(losses) < 2:
            return losses[0][0] if losses else None
        return sum(loss * (n / len(records)) for loss, n in losses)

    def _gradients(self, records):
        """Gradients of the records' workers into their rows of `external`; mean loss."""
        sched = self.schedule
        draws = [(int(sched.worker[e]), int(sched.iter[e]), self.batch) for e in records]
        workers = [worker for worker, _, _ in draws]
        at = torch.from_numpy(sched.batch_rows[records].astype("int64")).to(self.x.device)
        who = torch.tensor(workers, device=self.x.device)[:, None]
        x, target = self.x[who, at].flatten(0, 1), self.target[who, at].flatten(0, 1)
        begin = torch.arange(0, x.shape[0] + 1, self.batch, dtype=torch.int32, device=x.device)
        index = self.versions(workers)
        out, saved = self.block.forward(self.params, index, x, begin, self.seed, draws=draws)
        diff = out - target
        self.block.backward(self.params, index, saved, diff / (self.batch * self.block.width), begin, self.grads, workers)
        return diff.square().mean() / 2

    def evaluate(self, x, target):
        """Mean loss of every worker's newest replica on the same samples, without dropout."""
        with self._session_stream() as caller:
            loss = self._evaluate(x, target)
            if caller != self.stream:
                loss.record_stream(caller)
        return loss

    def _evaluate(self, x, target):
        x, target = x.to(self.x.device), target.to(self.x.device)
        losses = []
        for run in _runs(range(len(self.external))):
            begin = torch.arange(0, (len(run) + 1) * len(x), len(x), dtype=torch.int32, device=x.device)
            out, _ = self.block.forward(self.params, self.versions(run), x.repeat(len(run), 1), begin, train=False)
            losses.append((out.view(len(run), *target.shape) - target).square().mean((1, 2)) / 2)
        return losses[0] if len(losses) == 1 else torch.cat(losses)

    def close(self):
        self.session.close()


def teacher_data(block, N, samples, seed, device="cuda:0"):
    """Samples of every worker and the outputs of a block of the same shape with other parameters, plus noise; and 256 more for all."""
    g = torch.Generator(device=device).manual_seed(seed)
    teacher = block.views(block.initial(seed + 1).to(device)[None])
    x = torch.randn(N * samples + 256, block.width, generator=g, device=device)
    out, _ = block.forward(teacher, None, x, None, train=False)
    out = out + 0.01 * torch.randn(out.shape, generator=g, device=device)
    cut = N * samples
    return [(x[i * samples:(i + 1) * samples], out[i * samples:(i + 1) * samples]) for i in range(N)], (x[cut:], out[cut:])


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--workers", type=int, default=16)
    a.add_argument("--width", type=int, default=256)
    a.add_argument("--hidden", type=int, default=1024)
    a.add_argument("--samples", type=int, default=4096)
    a.add_argument("--batch", type=int, default=128)
    a.add_argument("--iterations", type=int, default=60)
    a.add_argument("--lr", type=float, default=20.0)
    a.add_argument("--momentum", type=float, default=0.9)
    a.add_argument("--dropout", type=float, default=0.1)
    a.add_argument("--seed", type=int, default=inputs.DEFAULT_SEED)
    o = a.parse_args(argv)
    block = ResidualBlock(o.width, o.hidden, p=o.dropout)
    data, held = teacher_data(block, o.workers, o.samples, o.seed)
    t = Training(block, inputs.ring(o.workers), data, o.iterations, o.batch, lr=o.lr, momentum=o.momentum, seed=o.seed)
    try:
        first = t.evaluate(*held)
        print("%d parameters, %d workers, %d waves; mean loss %.5f" % (block.d, o.workers, t.schedule.n_waves, float(first.mean())), flush=True)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for w in range(t.schedule.n_waves):
            t.wave(w)
            if (w + 1) % max(1, t.schedule.n_waves // 8) == 0:
                print("wave %5d  mean loss %.5f" % (w + 1, float(t.evaluate(*held).mean())), flush=True)
        end.record()
        torch.cuda.synchronize()
        last = t.evaluate(*held)
        updates = int((t.schedule.kind == hop.HOP_STEP).sum())
        print("mean loss %.5f -> %.5f, worst worker %.5f; %d worker-updates in %.1f ms" % (float(first.mean()), float(last.mean()), float(last.max()), updates,
                                                                                    begin.elapsed_time(end)))
        return float(first.mean()), float(last.mean())
    finally:
        t.close()


if __name__ == "__main__":
    main()
