"""Causal attention of packed and padded sequences with grouped heads, and its
gradient, against the fp64 formulas.

Tolerances (relative 2-norm): o takes two bf16 roundings, of the
probabilities and of itself, 2 * 2^-8; dv the same; dq and dk the rounding of
dS, of themselves, and that of o through delta, 3 * 2^-8.  lse is fp32
throughout: products of bf16 values are exact, so 128 + log-sized sums of
them err by at most a few 2^-24 of the scores' size, 1e-5 absolute here."""

import pytest
import torch

import batch_reference as ref
from batch_reference import U_BF16, rel
from paper_2605_07063_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL_O, TOL_DV, TOL_DQK, TOL_LSE = 2 * U_BF16, 2 * U_BF16, 3 * U_BF16, 1e-5


def make(rows, Hq, Hkv, D, fused, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(rows, (Hq + 2 * Hkv) * D, generator=g, device=DEV).mul(std).bfloat16()
    q, k, v = [p.reshape(rows, p.shape[1] // D, D) for p in x.split([Hq * D, Hkv * D, Hkv * D], 1)]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    return q, k, v, torch.randn(rows, Hq, D, generator=g, device=DEV).bfloat16()


def check(q, k, v, g, spans, where, scale=None, lse_tol=TOL_LSE):
    D = q.shape[-1]
    sc = D ** -0.5 if scale is None else scale
    o, lse = api.attention(q, k, v, scale=scale, **where)
    dq, dk, dv = api.attention_backward(g, q, k, v, o, lse, scale=scale, **where)
    flat = [t.reshape(-1, t.shape[-2], D) for t in (q, k, v)]
    want = ref.attention(*flat, spans, sc, g.reshape(-1, g.shape[-2], D))
    got = [t.reshape(-1, t.shape[-2], D) for t in (o, dq, dk, dv)]
    assert rel(got[0], want[0]) <= TOL_O
    assert float((ref.d64(lse) - want[1]).abs().max()) <= lse_tol
    assert rel(got[1], want[2]) <= TOL_DQK and rel(got[2], want[3]) <= TOL_DQK
    assert rel(got[3], want[4]) <= TOL_DV
    live = torch.zeros(flat[0].shape[0], dtype=torch.bool)
    for a, b in spans:
        live[a:b] = True
    for t in got:
        assert bool((t.cpu()[~live] == 0).all())
    assert bool((lse.cpu()[:, ~live] == 0).all())
    return o, lse, dq, dk, dv


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 200, 257]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 2), (7, 1)])
@pytest.mark.parametrize("fused", [False, True])
def test_packed_edges(D, Hq, Hkv, fused):
    """Lengths on both sides of every tile edge, empty and single-token sequences among them."""
    off = [0]
    for n in EDGES:
        off.append(off[-1] + n)
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    q, k, v, g = make(off[-1], Hq, Hkv, D, fused, 1)
    a = check(q, k, v, g, ref.spans_of(off, None, len(EDGES), 0), dict(offsets=offsets, max_len=max(EDGES)))
    b = check(q, k, v, g, ref.spans_of(off, None, len(EDGES), 0), dict(offsets=offsets, max_len=max(EDGES)))
    assert all(torch.equal(x, y) for x, y in zip(a, b))      # the same inputs, the same bits


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 17, 64, 130, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.0e38])
def test_padded_rows_are_never_read(D, T, bad):
    """[N, T] with lengths 0, 1, .., T: padding may hold any bits and comes out as zeros."""
    N = 5
    lens = [0, 1, T, max(1, T // 2), max(1, T - 1)]
    q, k, v, g = [t.view(N, T, -1, D) for t in make(N * T, 4, 2, D, False, 2)]
    for t in (q, k, v, g):
        for i, n in enumerate(lens):
            t[i, n:] = bad
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    clean = [torch.nan_to_num(t.float(), 0.0, 0.0, 0.0).bfloat16() for t in (q, k, v, g)]
    spans = ref.spans_of(None, lens, N, T)
    got = check(q, k, v, g, spans, dict(lengths=lengths))
    for t, c in zip((q, k, v, g), clean):
        for i, n in enumerate(lens):
            t[i, n:] = 0
    again = check(q, k, v, g, spans, dict(lengths=lengths))
    assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_non_finite_tokens_stay_in_their_sequence():
    q, k, v, g = make(300, 4, 2, 64, True, 3)
    offsets = torch.tensor([0, 100, 101, 300], dtype=torch.int32, device=DEV)
    where = dict(offsets=offsets, max_len=200)
    base = api.attention(q, k, v, **where)
    back = api.attention_backward(g, q, k, v, *base, **where)
    q[40, 0, 3], k[50, 1, 1], v[60, 0, 0], g[70, 1, 2] = float("nan"), float("inf"), float("-inf"), float("nan")
    o, lse = api.attention(q, k, v, **where)
    got = api.attention_backward(g, q, k, v, o, lse, **where)
    for x, y in zip((o, *got), (base[0], *back)):
        assert torch.equal(x[100:], y[100:])
    assert torch.equal(lse[:, 100:], base[1][:, 100:])


@pytest.mark.parametrize("std,scale", [(1.0, None), (6.0, None), (1.0, 1e-4), (0.0, None)])
def test_score_ranges(std, scale):
    """Flat softmax, one-hot softmax (scores in the thousands), zero scores."""
    q, k, v, g = make(190, 4, 2, 64, False, 4, std)
    if std == 0.0:
        v.normal_()
    offsets = torch.tensor([0, 190], dtype=torch.int32, device=DEV)
    check(q, k, v, g, [(0, 190)], dict(offsets=offsets, max_len=190), scale, TOL_LSE * max(1.0, std * std))


def test_rising_scores_move_the_running_maximum():
    """Keys whose scores grow along the sequence, so that every tile has a new maximum."""
    n, D = 520, 64
    q, k, v, g = make(n, 2, 1, D, False, 5)
    ramp = torch.linspace(0, 40, n, device=DEV)
    q.zero_()
    k.zero_()
    q[:, :, 0] = 8.0
    k[:, 0, 0] = ramp
    offsets = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o, lse = api.attention(q, k, v, offsets=offsets, max_len=n)
    want, lw = ref.attention(q, k, v, [(0, n)], D ** -0.5)
    assert rel(o, want) <= TOL_O and float((ref.d64(lse) - lw).abs().max()) <= 1e-4   # scores of 40


@pytest.mark.parametrize("D", [64, 128])
def test_long_sequence_and_short_ones(D):
    lens = [1500, 3, 1, 700]
    off = [0, 1500, 1503, 1504, 2204]
    q, k, v, g = make(2204, 2, 1, D, True, 6)
    check(q, k, v, g, ref.spans_of(off, None, 4, 0),
          dict(offsets=torch.tensor(off, dtype=torch.int32, device=DEV), max_len=max(lens)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,Hq,Hkv", [([700], 2, 2), ([1100, 0, 333], 3, 1), ([450, 129, 1, 64, 449], 4, 4), ([900, 70], 10, 2)])
def test_few_long_sequences(D, lens, Hq, Hkv):
    """Tiles whose steps are dealt to several workgroups, unevenly, and short ones beside them with fewer steps than parts."""
    N, T = len(lens), max(lens)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q, k, v, g = make(N * T, Hq, Hkv, D, False, 21)
    for t in (q, k, v, g):
        t.view(N, T, -1, D)[torch.arange(T, device=DEV)[None] >= lengths[:, None]] = float("nan")
    q, k, v, g = [t.view(N, T, -1, D) for t in (q, k, v, g)]
    spans = [(i * T, i * T + n) for i, n in enumerate(lens)]
    a = check(q, k, v, g, spans, dict(lengths=lengths))
    b = check(q, k, v, g, spans, dict(lengths=lengths))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("packed", [False, True])
def test_edges_in_larger_batches(D, packed):
    """The same edges where the workgroups are many, and where the sequences are few and their rows' keys are shared."""
    for copies, Hq, Hkv in ((4, 8, 4), (1, 1, 1)):
        lens = EDGES * copies
        N, T = len(lens), max(lens)
        off = [0]
        for n in lens:
            off.append(off[-1] + n)
        rows = off[-1] if packed else N * T
        q, k, v, g = make(rows, Hq, Hkv, D, packed, 22)
        if packed:
            where = dict(offsets=torch.tensor(off, dtype=torch.int32, device=DEV), max_len=T)
            spans = ref.spans_of(off, None, N, 0)
        else:
            q, k, v, g = [t.view(N, T, -1, D) for t in (q, k, v, g)]
            where = dict(lengths=torch.tensor(lens, dtype=torch.int32, device=DEV))
            spans = [(i * T, i * T + n) for i, n in enumerate(lens)]
        a = check(q, k, v, g, spans, where)
        b = check(q, k, v, g, spans, where)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_after_the_last_slot_and_lengths_with_offsets():
    q, k, v, g = make(100, 2, 2, 64, False, 7)
    off = [0, 30, 60]
    lens = [20, 30]
    for t in (q, k, v, g):
        t[20:30] = float("nan")
        t[60:] = float("nan")
    check(q, k, v, g, ref.spans_of(off, lens, 2, 0),
          dict(offsets=torch.tensor(off, dtype=torch.int32, device=DEV),
               lengths=torch.tensor(lens, dtype=torch.int32, device=DEV), max_len=30))


def test_many_sequences():
    """More short sequences than there are compute units."""
    N = 700
    lens = [(i * 37) % 9 for i in range(N)]
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    q, k, v, g = make(off[-1], 2, 1, 64, False, 8)
    check(q, k, v, g, ref.spans_of(off, None, N, 0),
          dict(offsets=torch.tensor(off, dtype=torch.int32, device=DEV), max_len=8))


@pytest.mark.parametrize("N", [3, 64, 65, 256, 257])
@pytest.mark.parametrize("where", ["first", "last", "middle"])
def test_one_long_sequence_among_short_ones(N, where):
    """Most pairs of a sequence and a tile are empty: workgroups look for their own (up to 256 sequences)."""
    lens = [(i * 5) % 4 for i in range(N)]
    lens[{"first": 0, "last": N - 1, "middle": N // 2}[where]] = 700
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    q, k, v, g = make(off[-1] + 3, 3, 1, 64, False, 13)     # and rows after the last slot
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    check(q, k, v, g, ref.spans_of(off, None, N, 0), dict(offsets=offsets, max_len=700))
    tight = api.attention(q, k, v, offsets=offsets, max_len=700)
    loose = api.attention(q, k, v, offsets=offsets, max_len=5000)
    assert all(torch.equal(a, b) for a, b in zip(tight, loose))


def test_gradient_against_differences():
    n, D = 40, 64
    q, k, v, g = make(n, 2, 1, D, False, 9)
    offsets = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o, lse = api.attention(q, k, v, offsets=offsets, max_len=n)
    grads = api.attention_backward(g, q, k, v, o, lse, offsets=offsets, max_len=n)
    x = [ref.d64(t) for t in (q, k, v)]
    gen = torch.Generator().manual_seed(1)
    dirs = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in x]
    for which in range(3):
        f = lambda s: float((ref.attention(*[t + s * d if i == which else t for i, (t, d) in enumerate(zip(x, dirs))],  # noqa: E731
                                           [(0, n)], D ** -0.5)[0] * ref.d64(g)).sum())
        want = (f(1e-5) - f(-1e-5)) / 2e-5
        got = float((ref.d64(grads[which]) * dirs[which]).sum())
        size = float(ref.d64(grads[which]).norm() * dirs[which].norm())
        assert abs(got - want) <= 3 * U_BF16 * size


def test_side_stream_and_graph():
    """The same bits on another stream, and from replays of a captured graph."""
    q, k, v, g = make(333, 4, 2, 128, True, 10)
    offsets = torch.tensor([0, 100, 333], dtype=torch.int32, device=DEV)
    where = dict(offsets=offsets, max_len=233)
    o, lse = api.attention(q, k, v, **where)
    d = api.attention_backward(g, q, k, v, o, lse, **where)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, lse2 = api.attention(q, k, v, stream=side, **where)
    d2 = api.attention_backward(g, q, k, v, o2, lse2, stream=side, **where)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(a, b) for a, b in zip(d, d2))
    o3, lse3 = torch.zeros_like(o), torch.zeros_like(lse)
    d3 = [torch.zeros_like(t) for t in d]
    ws = torch.empty(api.dr_attention_workspace_size(333, 4, 2, 128), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.dr_attention(q, k, v, offsets, None, 233, None, o3, lse3)
        api.dr_attention_backward(g, q, k, v, o3, lse3, offsets, None, 233, None, *d3, workspace=ws)
    for _ in range(3):
        o3.zero_()
        [t.fill_(7) for t in d3]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o3) and all(torch.equal(a, b) for a, b in zip(d, d3))


def test_refusals():
    q, k, v, g = make(64, 4, 2, 64, False, 11)
    off = torch.tensor([0, 64], dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        api.attention(q, k, v, offsets=off)                                  # no max_len
    with pytest.raises(ValueError):
        api.attention(q, k, v)                                               # [rows, H, D] without a layout
    with pytest.raises(ValueError):
        api.attention(q.float(), k.float(), v.float(), offsets=off, max_len=64)
    with pytest.raises(ValueError):
        api.attention(q, k, v[:, :1], offsets=off, max_len=64)
    with pytest.raises(ValueError):
        api.attention(q, k, v, offsets=off.long(), max_len=64)
    with pytest.raises(ValueError):
        api.attention(q, k, v, max_len=32, lengths=torch.ones(3, dtype=torch.int32, device=DEV))
    for bad, status in ((dict(scale=0.0), _lib.DR_ERR_ARG), (dict(scale=float("nan")), _lib.DR_ERR_ARG)):
        with pytest.raises(_lib.DrError) as e:
            api.attention(q, k, v, offsets=off, max_len=64, **bad)
        assert e.value.status == status
    q3, k2 = q[:, :3].contiguous(), k
    with pytest.raises(_lib.DrError) as e:
        api.attention(q3, k2, v, offsets=off, max_len=64)                    # 3 heads over 2
    assert e.value.status == _lib.DR_ERR_ARG
    x = torch.zeros(64, 2, 96, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(_lib.DrError) as e:
        api.attention(x, x, x, offsets=off, max_len=64)
    assert e.value.status == _lib.DR_ERR_UNSUPPORTED
    o, lse = api.attention(q, k, v, offsets=off, max_len=64)
    with pytest.raises(ValueError):
        api.dr_attention_backward(g, q, k, v, o, lse, off, None, 64, None, torch.empty_like(q), torch.empty_like(k),
                                  torch.empty_like(v), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))


def test_no_rows_and_no_sequences():
    q, k, v, g = make(0, 4, 2, 64, False, 12)
    off = torch.zeros(1, dtype=torch.int32, device=DEV)
    o, lse = api.attention(q, k, v, offsets=off, max_len=0)
    assert o.numel() == 0 and lse.numel() == 0
    assert all(t.numel() == 0 for t in api.attention_backward(g, q, k, v, o, lse, offsets=off, max_len=0))


@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (66, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_offsets_out_of_range(D, Hq, Hkv):
    """Offsets below 0 and above the rows count as 0 and as the rows, whether the launch goes over all pairs of a sequence
    and a tile (max_len 128) or workgroups look for their own (max_len 4096), with tiles of 32 rows (2 heads) and 128."""
    rows = 128
    q, k, v, g = make(rows, Hq, Hkv, D, True, 31)
    given, clamped = [-9, 64, 100, 5000, 1 << 30], [0, 64, 100, 128, 128]
    off = torch.tensor(given, dtype=torch.int32, device=DEV)
    spans = ref.spans_of(clamped, None, 4, 0)
    want = ref.attention(q, k, v, spans, D ** -0.5, g)
    for most in (128, 4096):
        o, lse = torch.full_like(q, 7.0), torch.full((Hq, rows), 7.0, device=DEV)
        grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
        ws = torch.full((api.dr_attention_workspace_size(rows, Hq, Hkv, D),), 255, dtype=torch.uint8, device=DEV)
        api.dr_attention(q, k, v, off, None, most, None, o, lse)
        api.dr_attention_backward(g, q, k, v, o, lse, off, None, most, None, *grads, workspace=ws)
        assert rel(o, want[0]) <= TOL_O and float((ref.d64(lse) - want[1]).abs().max()) <= TOL_LSE
        assert rel(grads[0], want[2]) <= TOL_DQK and rel(grads[1], want[3]) <= TOL_DQK and rel(grads[2], want[4]) <= TOL_DV


@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (32, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_reaches_the_statistics_it_belongs_to(D, Hq, Hkv):
    """A NaN in a key makes o and lse NaN in that key's row and every later one of its sequence, a NaN in a query in its
    own row, with tiles of 32 rows (2 heads) and 128; lse keeps its bits elsewhere."""
    lens, at = [200, 129, 65, 200, 33, 1], [0, 32, 64, 96, 31, 0]
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    rows = off[-1]
    where = dict(offsets=torch.tensor(off, dtype=torch.int32, device=DEV), max_len=max(lens))
    q, k, v, _ = make(rows, Hq, Hkv, D, False, 32)
    _, base = api.attention(q, k, v, **where)
    for which in (k, q):
        bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
        x = which.clone()
        for a, b, i in zip(off, off[1:], at):
            x[a + i, :, 5] = float("nan")
            bad[a + i:b if which is k else a + i + 1] = True
        o, lse = api.attention(x if which is q else q, x if which is k else k, v, **where)
        assert bool(torch.isnan(lse[:, bad]).all()) and bool(torch.isnan(o[bad].float()).all())
        assert torch.equal(lse[:, ~bad], base[:, ~bad])


def bounds(q, k, v, g, spans, scale):
    """What each row of o, dq, dk, dv of each head may be off by, in norm, given the roundings to bf16 (2^-8 of a value each):
    P, with sums of P and dS in fp32, dS, o in delta, and the outputs.  5 % more for fp32 arithmetic."""
    q, k, v, g = (ref.d64(t) for t in (q, k, v, g))
    rows, Hq, D = q.shape
    G = Hq // k.shape[1]
    out = [torch.zeros(rows, n, dtype=torch.float64) for n in (Hq, Hq, k.shape[1], k.shape[1])]
    for a, b in spans:
        hide = torch.ones(b - a, b - a, dtype=torch.bool).triu(1)
        for h in range(Hq if b > a else 0):
            Q, K, V, dO = q[a:b, h], k[a:b, h // G], v[a:b, h // G], g[a:b, h]
            P = torch.softmax((scale * Q @ K.t()).masked_fill(hide, -float("inf")), -1)
            O = P @ V
            weight = P @ V.norm(dim=1) + O.norm(dim=1)           # what o's error may be 2^-8 of
            off = dO.norm(dim=1) * weight                        # delta's
            dS = (P * (dO @ V.t() - (dO * O).sum(-1, keepdim=True))).abs()
            out[0][a:b, h] = weight
            out[1][a:b, h] = scale * (dS @ K.norm(dim=1) + off * (P @ K).norm(dim=1))
            out[2][a:b, h // G] += scale * (dS.t() @ Q.norm(dim=1) + P.t() @ (off * Q.norm(dim=1)))
            out[3][a:b, h // G] += P.t() @ dO.norm(dim=1)
    o, lse, dq, dk, dv = ref.attention(q, k, v, spans, scale, g)
    for x, t in zip(out[1:], (dq, dk, dv)):
        x += t.norm(dim=-1)
    return [1.05 * U_BF16 * x for x in out], (o, dq, dk, dv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,Hq,Hkv", [(EDGES, 4, 2), ([700, 650, 300, 5], 8, 8), ([700, 650, 300, 5], 8, 2), ([900, 70], 10, 2),
                                         ([1100], 2, 1)])
def test_rows_one_by_one(D, lens, Hq, Hkv):
    """Every row of every head by itself, so that a few wrong values of a tile's edge show: tiles of 32 rows and 128, dk and
    dv whole and in parts."""
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    q, k, v, g = make(off[-1], Hq, Hkv, D, True, 33)
    where = dict(offsets=offsets, max_len=max(lens))
    spans = ref.spans_of(off, None, len(lens), 0)
    o, lse = api.attention(q, k, v, **where)
    got = (o, *api.attention_backward(g, q, k, v, o, lse, **where))
    limit, want = bounds(q, k, v, g, spans, D ** -0.5)
    for x, y, m in zip(got, want, limit):
        worst = ((ref.d64(x) - y).norm(dim=-1) / m).max()
        print(f"{float(worst):.2f} of the bound")
        assert float(worst) <= 1.0
