"""One data-selection step on a small transformer block, from tokens to update.

The merged batch (n general examples, then m target examples, Sec. 4.2) goes
through one attention block and the loss over the vocabulary, forward and
backward; the linear maps' retained pairs (input, output gradient) are
sketched, the general examples scored against the mean target gradient, and
the update assembled from the best k of them:

  x -> q, k, v -> qk_norm_rope -> attention -> output map (+ x) -> cross_entropy
  cross_entropy_backward -> attention_backward -> qk_norm_rope_backward
  -> sketch -> gram -> select_topk -> assemble_update

The linear maps are plain library products; every other step is a call of
paper_2605_07063_amd.api.  Inputs and weights are random.

Usage: python examples/merged_batch_step.py [--general 12] [--target 4] [--tokens 160]
"""

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_07063_amd import api  # noqa: E402

IGNORE = -100


def rotation_table(positions, D, device, base=10000.0):
    """Cosines and sines [positions, D/2, 2], formed in fp64."""
    ang = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * torch.exp(
        torch.arange(D // 2, dtype=torch.float64, device=device) * (-2.0 / D * math.log(base)))
    return torch.stack([ang.cos(), ang.sin()], -1).float()


def make_block(d, Hq, Hkv, D, V, T, device, seed=0, sketch=16):
    """Random weights of the block and the projectors of its four maps' sketches."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def draw(o, i):
        return torch.randn(o, i, generator=g, device=device).mul_(1.0 / math.sqrt(i)).bfloat16()

    sizes = [Hq * D, Hkv * D, Hkv * D]
    w = dict(Hq=Hq, Hkv=Hkv, D=D, qkv=draw(sum(sizes), d), o=draw(d, Hq * D), head=draw(V, d),
             wq=1.0 + 0.1 * torch.randn(D, generator=g, device=device),
             wk=1.0 + 0.1 * torch.randn(D, generator=g, device=device), table=rotation_table(T, D, device))
    w["maps"] = [(d, s) for s in sizes] + [(Hq * D, d)]
    w["p"] = [tuple(torch.randn(sketch, n, generator=g, device=device).div_(math.sqrt(sketch)).bfloat16() for n in io)
              for io in w["maps"]]
    return w


def make_batch(N, T, d, V, device, seed=1):
    """Embedded tokens [N, T, d] with lengths, and targets of the answer tokens (the prompt's and the padding's are
    IGNORE)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    x = torch.randn(N, T, d, generator=g, device=device).bfloat16()
    lens = torch.randint(max(2, T // 4), T + 1, (N,), generator=g, device=device).to(torch.int32)
    t = torch.randint(0, V, (N, T), generator=g, device=device).to(torch.int32)
    at = torch.arange(T, device=device)[None]
    answer = (at >= lens[:, None] // 3) & (at < lens[:, None])
    return x, lens, torch.where(answer, t, torch.full_like(t, IGNORE))


def forward_backward(w, x, lens, target):
    """Losses [N, T] and the four maps' retained pairs [(input, output gradient)] of every example's mean loss."""
    N, T, d = x.shape
    Hq, Hkv, D = w["Hq"], w["Hkv"], w["D"]
    flat = x.view(N * T, d)
    qkv = (flat @ w["qkv"].t()).view(N, T, Hq + 2 * Hkv, D)
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)                      # views: the kernels take the row stride
    qr, kr = api.qk_norm_rope(q, k, w["table"], w["wq"], w["wk"], lengths=lens)   # positions: places in the example
    o, lse = api.attention(qr, kr, v, lengths=lens)
    y = o.view(N * T, Hq * D) @ w["o"].t() + flat
    t = target.reshape(-1)
    loss, z = api.cross_entropy(y, w["head"], t)

    live = (target != IGNORE).sum(1, keepdim=True).clamp(min=1)
    g = (1.0 / live.float()).expand(N, T).reshape(-1).contiguous()
    dy, _ = api.cross_entropy_backward(y, w["head"], t, z, g, need_dweight=False)
    do = (dy @ w["o"]).view(N, T, Hq, D)
    dqr, dkr, dv = api.attention_backward(do, qr, kr, v, o, lse, lengths=lens)
    dq, dk, _, _ = api.qk_norm_rope_backward(dqr, dkr, q, k, w["table"], w["wq"], w["wk"], lengths=lens)
    pairs = [(x, dq.view(N, T, -1)), (x, dk.view(N, T, -1)), (x, dv.view(N, T, -1)),
             (o.view(N, T, -1), dy.view(N, T, d))]
    return loss.view(N, T), pairs


def select_and_update(w, pairs, lens, n, k):
    """Scores of the n general examples, the k selected ones, and the maps' updates (means over those)."""
    layers, col = [], 0
    for (a, dy), (p_in, p_out) in zip(pairs, w["p"]):
        layers.append(dict(x=a, dy=dy, p_in=p_in, p_out=p_out, col_offset=col))
        col += p_in.shape[0] * p_out.shape[0]
    S = api.sketch(layers, lens)
    _, s, _ = api.gram(S[:n], S[n:])
    idx, weight, info = api.select_topk(s, k)
    return s, idx, api.assemble_update(layers, weight, n=n, lengths=lens), info


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--general", type=int, default=12)
    ap.add_argument("--target", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=160)
    a = ap.parse_args()
    dev, d, V = "cuda:0", 256, 1000
    N = a.general + a.target
    w = make_block(d, Hq=4, Hkv=2, D=64, V=V, T=a.tokens, device=dev)
    x, lens, target = make_batch(N, a.tokens, d, V, dev)
    loss, pairs = forward_backward(w, x, lens, target)
    s, idx, updates, info = select_and_update(w, pairs, lens, a.general, max(1, a.general // 2))
    torch.cuda.synchronize()
    assert int(info[0]) == 0
    print(f"mean loss over answer tokens {float(loss[target != IGNORE].mean()):.4f} (log V = {math.log(V):.4f})")
    print("scores  ", " ".join(f"{v:.3g}" for v in s[0].tolist()))
    print("selected", idx[0].tolist())
    print("updates ", " ".join(f"{tuple(u.shape)}: |u| {float(u.norm()):.3g}" for u in updates))


if __name__ == "__main__":
    main()
