"""The example's step (norm and rotation, attention, loss, their gradients, then
sketch, scores, selection and update) against fp64 autograd of the same
block.  Between the inputs and a retained gradient stand at most ten bf16
roundings (q/k/v, rotated q/k, probabilities, o, y, dz, dh, do, dS, dq), each
2^-8 at most: 10 * 2^-8."""

import os
import sys

import pytest
import torch

import batch_reference as ref
from batch_reference import U_BF16, rel

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 10 * U_BF16


def autograd_pairs(w, x, lens, target):
    """Losses and the four maps' (input, output gradient), every example by itself, in fp64."""
    N, T, d = x.shape
    Hq, Hkv, D = w["Hq"], w["Hkv"], w["D"]
    W, O, V = ref.d64(w["qkv"]), ref.d64(w["o"]), ref.d64(w["head"])
    losses = torch.zeros(N, T, dtype=torch.float64)
    grads = [torch.zeros(N, T, n, dtype=torch.float64) for n in (Hq * D, Hkv * D, Hkv * D, d)]
    outs = torch.zeros(N, T, Hq * D, dtype=torch.float64)
    for i in range(N):
        n = int(lens[i])
        a, t = ref.d64(x[i, :n]), target[i, :n].cpu().long()
        pos = torch.arange(n)
        q, k, v = [u.requires_grad_() for u in (a @ W.t()).split([Hq * D, Hkv * D, Hkv * D], 1)]

        def norm(u, g):
            u = u.view(n, -1, D)
            u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-6) * ref.d64(g)
            cs = ref.d64(w["table"])[pos][:, None]
            b, c = u[..., :D // 2], u[..., D // 2:]
            return torch.cat([b * cs[..., 0] - c * cs[..., 1], b * cs[..., 1] + c * cs[..., 0]], -1)

        qh, kh = norm(q, w["wq"]), norm(k, w["wk"]).repeat_interleave(Hq // Hkv, 1)
        vh = v.view(n, Hkv, D).repeat_interleave(Hq // Hkv, 1)
        S = torch.einsum("ihd,jhd->hij", qh, kh) * D ** -0.5
        P = torch.softmax(S.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -float("inf")), -1)
        o = torch.einsum("hij,jhd->ihd", P, vh).reshape(n, Hq * D)
        m = o @ O.t()
        m.retain_grad()
        z = (m + a) @ V.t()
        live = t >= 0
        l = torch.logsumexp(z, -1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        losses[i, :n] = (l * live).detach()
        (l[live].sum() / max(1, int(live.sum()))).backward()
        outs[i, :n] = o.detach()
        for G, u in zip(grads, (q, k, v, m)):
            G[i, :n] = u.grad
    return losses, outs, grads


def test_step_matches_autograd():
    import merged_batch_step as step
    n, m, T, d, V = 5, 3, 70, 128, 333
    w = step.make_block(d, Hq=4, Hkv=2, D=64, V=V, T=T, device=DEV)
    x, lens, target = step.make_batch(n + m, T, d, V, DEV)
    for i in range(n + m):
        x[i, int(lens[i]):] = 7.0          # padding rows go through the library products, too
    loss, pairs = step.forward_backward(w, x, lens, target)
    losses, outs, grads = autograd_pairs(w, x, lens, target)
    assert rel(loss, losses) <= TOL
    assert rel(pairs[3][0], outs) <= TOL
    for (a, dy), g in zip(pairs, grads):
        live = (torch.arange(T)[None] < lens.cpu()[:, None])[..., None]
        assert rel(ref.d64(dy) * live, g) <= TOL
    s, idx, updates, info = step.select_and_update(w, pairs, lens, n, 2)
    torch.cuda.synchronize()
    assert int(info[0]) == 0 and idx.shape == (1, 2)
    # the update of the output map: the mean gradient of the selected examples
    want = sum(grads[3][i].t() @ outs[i] for i in idx[0].tolist()) / 2
    assert rel(updates[3], want) <= 2 * TOL


def test_scores_and_selection_match_autograd():
    """The scores against those of the fp64 gradients' sketches: a product of two sketches, each within TOL of its size.  The
    selected examples are the best ones but for scores that this does not tell apart."""
    import merged_batch_step as step
    import oracle
    n, m, T, d, V, k = 11, 4, 70, 128, 333, 4
    w = step.make_block(d, Hq=4, Hkv=2, D=64, V=V, T=T, device=DEV)
    x, lens, target = step.make_batch(n + m, T, d, V, DEV)
    _, outs, grads = autograd_pairs(w, x, lens, target)
    for i in range(n + m):
        x[i, int(lens[i]):] = 7.0
    _, pairs = step.forward_backward(w, x, lens, target)
    s, idx, _, info = step.select_and_update(w, pairs, lens, n, k)
    torch.cuda.synchronize()
    ins = [ref.d64(x)] * 3 + [outs]
    S = oracle.sketch_ref([dict(x=a.numpy(), dy=dy.numpy(), p_in=ref.d64(p[0]).numpy(), p_out=ref.d64(p[1]).numpy())
                           for a, dy, p in zip(ins, grads, w["p"])], lens.cpu().numpy())
    want = torch.from_numpy(oracle.gram_ref(S[:n], S[n:])[1][0])
    size = torch.from_numpy(S[:n]).norm(dim=1) * float(torch.from_numpy(S[n:]).mean(0).norm())
    err = (ref.d64(s[0]) - want).abs()
    print(f"scores within {float((err / size).max()):.2e} of the sketches' sizes, which differ from 0 by "
          f"{float((want.abs() / size).mean()):.2e} on average")
    assert bool((err <= 2 * TOL * size).all())
    got, best = sorted(idx[0].tolist()), want.topk(k).values[-1]
    assert int(info[0]) == 0 and len(set(got)) == k
    assert all(float(want[i]) >= float(best) - 4 * TOL * float(size.max()) for i in got)
    assert got == sorted(ref.d64(s[0]).topk(k).indices.tolist())
