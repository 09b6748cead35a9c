"""Layer norm, preference loss, ghost clipping and orthogonalised updates run together, as a private step on pairs runs them:

  y = layer norm of x, logits = y W^T, the pairs' loss and its gradient G at the logits, the head's ghost norms from (y, G), the gradient
  G W at y and the norm's backward pass with its sums, one clip factor per pair for all three parameters, clipped sums, noise, the
  head's update orthogonalised,

against autograd in 64 bits.  Tolerances, with u = 2^-24: a logit is a sum of d terms and off by (d + 2) u times their magnitudes, the
normalised input and a softmax by a few u more; a pair's loss adds 2T rows of those, and its slope in h is 1 at most.  Relative to the norms of the
results that is below (2 d + 60) u * (1 + 2 T beta * the largest logit) for d = 96, T = 24, beta = 0.2 and logits below 6.
"""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as O
from paper_2609_40335_b200 import binding as dp
from paper_2609_40335_b200 import pipeline
from paper_2609_40335_b200.workloads import make_workload

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B, T, D, V, BETA, EPS, C = 6, 24, 96, 203, 0.2, 1e-5, 0.05
QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5


def f64(t):
    return t.detach().double().cpu().numpy()


def rel_norm(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


def inputs():
    g = torch.Generator().manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=g)
    x, W = 2 * n(B, 2 * T, D) + 0.3, n(V, D) / math.sqrt(D)
    gain, shift = 1 + 0.1 * n(D), 0.1 * n(D)
    targets = torch.randint(0, V, (B, 2, T), generator=g, dtype=torch.int32)
    targets[:, :, :4] = -1                                      # the prompt
    targets[1, 1, 15:] = targets[4, 0, 9:] = -1                 # padding
    targets[3] = -1                                             # a pair without tokens
    return [t.cuda() for t in (x, W, gain, shift, targets, n(B, 2) * 2 - 20 * math.log(V))]


def reference(x, W, gain, shift, targets, ref):
    """Losses, per-pair gradients of gain, shift and W, and the gradient at x, by autograd in 64 bits."""
    x, W, gain, shift, ref = (t.detach().double().cpu() for t in (x, W, gain, shift, ref))
    t = targets.cpu().long()
    losses, grads, dx = [], [], []
    for i in range(B):
        p = [v.clone().requires_grad_() for v in (gain, shift, W, x[i])]
        y = torch.nn.functional.layer_norm(p[3], (D,), p[0], p[1], EPS)
        lp = torch.log_softmax(y @ p[2].T, -1).view(2, T, V)
        l = (lp.gather(-1, t[i].clamp(min=0)[..., None])[..., 0] * (t[i] >= 0)).sum(-1)
        loss = -torch.nn.functional.logsigmoid(BETA * ((l[0] - ref[i, 0]) - (l[1] - ref[i, 1])))
        g = torch.autograd.grad(loss, p)
        losses.append(loss.item())
        grads.append([v.numpy() for v in g[:3]])
        dx.append(g[3].numpy())
    return np.array(losses), grads, np.stack(dx)


class Step:
    """The calls of the step on buffers of its own."""

    def __init__(self, x, W, gain, shift, targets, ref, sigma):
        f = lambda *s: torch.empty(*s, device="cuda")
        self.x, self.W, self.gain, self.shift, self.targets, self.ref, self.sigma = x, W, gain, shift, targets, ref, sigma
        self.y, self.mean, self.rstd = torch.empty_like(x), f(B, 2 * T), f(B, 2 * T)
        self.logits, self.G, self.dy, self.dx = f(B, 2 * T, V), f(B, 2 * T, V), torch.empty_like(x), torch.empty_like(x)
        self.loss, self.sq, self.clip, self.norms = f(B), f(B), f(B), f(B)
        self.gain_sums, self.shift_sums = f(B, D), f(B, D)
        self.outs = {"W": f(V, D), "gain": f(D), "shift": f(D)}
        self.update = f(V, D)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.head = dp.Linear(self.y, self.G, d=D, p=V)
        self.vectors = [dp.Vector(self.gain_sums.view(B, 1, D)), dp.Vector(self.shift_sums.view(B, 1, D))]
        u8 = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        self.ws = u8(max(dp.dp_ghost_norms_ws_bytes([self.head], B, 2 * T), dp.dp_clip_accumulate_grouped_ws_bytes([self.head], B, 2 * T),
                         dp.dp_clip_accumulate_vectors_ws_bytes(self.vectors, B, 1), dp.dp_preference_loss_ws_bytes(B, T),
                         dp.dp_layernorm_backward_ws_bytes(B, 2 * T, D), dp.dp_orthogonalize_ws_bytes([self.outs["W"]])))

    def run(self):
        kw = dict(ws=self.ws, dev_status=self.status)
        dp.dp_layernorm(self.x, self.gain, self.shift, EPS, Y=self.y, mean=self.mean, rstd=self.rstd)
        torch.matmul(self.y, self.W.T, out=self.logits)
        dp.dp_preference_loss(self.logits, self.targets, self.ref, BETA, loss=self.loss, G=self.G, **kw)
        torch.matmul(self.G, self.W, out=self.dy)
        self.sq.zero_()
        dp.dp_ghost_norms([self.head], B, 2 * T, self.sq, **kw)
        dp.dp_layernorm_backward(self.dy, self.x, self.gain, self.mean, self.rstd, dX=self.dx, gain_sums=self.gain_sums,
                                 shift_sums=self.shift_sums, sq=self.sq, **kw)
        dp.dp_clip_factors(self.sq, C, clip=self.clip, norms=self.norms)
        dp.dp_clip_accumulate_grouped([self.head], B, 2 * T, self.sq, C, [self.outs["W"]], **kw)
        dp.dp_clip_accumulate_vectors(self.vectors, B, 1, self.sq, C, [self.outs["gain"], self.outs["shift"]], ws=self.ws)
        if self.sigma:
            for k, n in enumerate(self.outs):
                dp.dp_add_noise(self.outs[n], self.sigma, C, 1.0, 7, k, 3)
        dp.dp_orthogonalize([self.outs["W"]], [self.update], **kw)


def test_a_private_step_on_pairs():
    args = inputs()
    losses, grads, dx = reference(*args)
    norms = np.array([math.sqrt(sum((v ** 2).sum() for v in g)) for g in grads])
    clip = np.minimum(1.0, C / np.where(norms > 0, norms, C))
    assert (clip < 1).sum() >= 3 and norms[3] == 0               # clipping is at work, and a pair without a gradient
    s = Step(*args, sigma=0.0)
    s.run()
    assert int(s.status.item()) == 0
    room = (2 * D + 60) * U * (1 + 2 * T * BETA * 6)
    assert np.abs(f64(s.loss) - losses).max() < room * 6
    assert np.abs(f64(s.norms) - norms).max() <= room * norms.max() and np.abs(f64(s.clip) - clip).max() < room
    for i in range(B):
        assert np.linalg.norm(f64(s.dx)[i] - dx[i]) <= room * np.linalg.norm(dx[i])
    for k, n in enumerate(("gain", "shift", "W")):
        want = sum(c * g[k] for c, g in zip(clip, grads))
        assert rel_norm(s.outs[n], want) < room, n


def test_a_private_step_on_pairs_with_noise_and_its_update_in_a_graph():
    args = inputs()
    plain, noisy = Step(*args, sigma=0.0), Step(*args, sigma=1.5)
    plain.run()
    noisy.run()
    for k, n in enumerate(noisy.outs):
        want = plain.outs[n].clone()
        dp.dp_add_noise(want, 1.5, C, 1.0, 7, k, 3)
        assert torch.equal(noisy.outs[n], want)
    # the update of the noised sum: products of at most V terms (see the operators' tests)
    room = 90 * (3 * 2.0 ** -22 + math.ceil(V / 16) * 2.0 ** -24) + U
    assert rel_norm(noisy.update, O.orthogonalize(f64(noisy.outs["W"]), QUINTIC)) < room
    first = {n: noisy.outs[n].clone() for n in noisy.outs}, noisy.update.clone(), noisy.loss.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        noisy.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        noisy.run()
    for _ in range(3):
        for v in (*noisy.outs.values(), noisy.update, noisy.loss, noisy.G):
            v.fill_(float("nan"))
        graph.replay()
    torch.cuda.synchronize()
    assert int(noisy.status.item()) == 0
    assert all(torch.equal(noisy.outs[n], first[0][n]) for n in first[0])
    assert torch.equal(noisy.update, first[1]) and torch.equal(noisy.loss, first[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orthogonal_updates_of_a_step(dtype):
    ds = pipeline.upload(make_workload("updates", B=3, T=16, dtype=dtype, block_shapes=[(40, 120), (40, 40), (160, 40)], n_blocks=2, d_model=40,
                                       V=97, lm_head=True))
    pipeline.allocate(ds)
    pipeline.dp_step(ds, seed=1, step=2)
    for out in (torch.float32, torch.bfloat16):
        into = {f"linear{k}": torch.empty(l.p, l.d, device="cuda", dtype=out) for k, l in enumerate(ds.linears)}
        got = pipeline.orthogonal_updates(ds, into, scale=0.5)
        for k, l in enumerate(ds.linears):
            m = f64(ds.outs[f"linear{k}"])
            want = O.orthogonalize(m, QUINTIC, 1e-7, 0.5 * max(1.0, l.p / l.d) ** 0.5)
            room = 90 * (3 * 2.0 ** -22 + math.ceil(max(l.p, l.d) / 16) * 2.0 ** -24) + torch.finfo(out).eps / 2
            assert got[f"linear{k}"] is into[f"linear{k}"] and rel_norm(got[f"linear{k}"], want) < room
    made = pipeline.orthogonal_updates(ds, scale=0.5)
    assert set(made) == {f"linear{k}" for k in range(len(ds.linears))} and int(ds.dev_status.item()) == 0
    assert all(m.dtype == torch.float32 for m in made.values())


@pytest.mark.parametrize("raw", [False, True])
def test_orthogonal_updates_on_another_stream_are_tensors_of_it(raw):
    """Updates that the call makes do not lie where the current stream still reads."""
    ds = pipeline.upload(make_workload("updates", B=3, T=16, dtype="f32", block_shapes=[(256, 512)], n_blocks=1, d_model=256, V=97, lm_head=True))
    pipeline.allocate(ds)
    pipeline.dp_step(ds, seed=1, step=2)
    want = {n: u.clone() for n, u in pipeline.orthogonal_updates(ds).items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    bait = torch.full_like(want["linear0"], 7.0)
    kept = torch.empty_like(bait)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                               # some 100 ms
    kept.copy_(bait)
    del bait
    got = pipeline.orthogonal_updates(ds, stream=side.cuda_stream if raw else side)
    side.synchronize()
    with torch.cuda.stream(side):
        assert all(torch.equal(got[n], want[n]) for n in want)
    torch.cuda.synchronize()
    assert (kept == 7.0).all()
