"""Per-head norm and rotation of queries and keys, and its gradient, against
the fp64 formulas.  Tolerances: fp32 arithmetic takes about ten roundings per
value (sums of up to 128 squares among them), 16 * 2^-24; a bf16 output adds
its own rounding, 2^-8.  Weight gradients are fp32 sums in a fixed order of
fp32 terms: 64 * 2^-24 covers the sizes here."""

import math

import pytest
import torch

import batch_reference as ref
from batch_reference import U_BF16, U_F32, rel
from paper_2605_07063_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = {torch.float32: 16 * U_F32, torch.bfloat16: U_BF16 + 16 * U_F32}
TOL_DW = 64 * U_F32


def table_of(n, D):
    ang = torch.arange(n, dtype=torch.float64)[:, None] * torch.exp(
        torch.arange(D // 2, dtype=torch.float64) * (-2.0 / D * math.log(10000.0)))
    return torch.stack([ang.cos(), ang.sin()], -1).float().to(DEV)


def inputs(rows, Hq, Hkv, D, dtype, fused, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(rows, (Hq + 2 * Hkv) * D, generator=g, device=DEV).mul(2).to(dtype)
    q, k, _ = [p.reshape(rows, -1, D) for p in x.split([Hq * D, Hkv * D, Hkv * D], 1)]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    gq = torch.randn(rows, Hq, D, generator=g, device=DEV).to(dtype)
    gk = torch.randn(rows, Hkv, D, generator=g, device=DEV).to(dtype)
    w = 1 + 0.3 * torch.randn(2, D, generator=g, device=DEV)
    pos = torch.randint(0, 300, (rows,), generator=g, device=DEV).to(torch.int32)
    return q, k, gq, gk, w[0].contiguous(), w[1].contiguous(), pos


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("norm,pairs", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("rows,Hq,Hkv,fused", [(1, 1, 1, False), (5, 7, 1, True), (33, 8, 2, True), (257, 21, 3, False),
                                               (4099, 4, 4, True)])
def test_forward_and_gradient(dtype, D, norm, pairs, rows, Hq, Hkv, fused):
    q, k, gq, gk, wq, wk, pos = inputs(rows, Hq, Hkv, D, dtype, fused, 11 + rows)
    if not norm:
        wq = wk = None
    tab = table_of(300, D)
    qo, ko = api.qk_norm_rope(q, k, tab, wq, wk, eps=1e-5, pos=pos, pairs=pairs)
    dq, dk, dwq, dwk = api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, eps=1e-5, pos=pos, pairs=pairs)
    for x, w, out, g, dx, dw in ((q, wq, qo, gq, dq, dwq), (k, wk, ko, gk, dk, dwk)):
        assert rel(out, ref.norm_rope(x, w, 1e-5, tab, pos, pairs)) <= TOL[dtype]
        dx_ref, dw_ref = ref.norm_rope_back(g, x, w, 1e-5, tab, pos, pairs)
        assert rel(dx, dx_ref) <= 2 * TOL[dtype]
        if norm:
            assert rel(dw, dw_ref) <= TOL_DW
        else:
            assert dw is None
    again = api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, eps=1e-5, pos=pos, pairs=pairs)
    assert all(a is b or torch.equal(a, b) for a, b in zip((dq, dk, dwq, dwk), again))


def test_gradient_against_differences():
    """<gradient, direction> equals the central difference of the fp64 forward."""
    q, k, gq, gk, wq, wk, pos = inputs(9, 4, 2, 64, torch.float32, False, 3)
    tab = table_of(300, 64)
    dq, dk, dwq, dwk = api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, eps=1e-5, pos=pos)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        gen = torch.Generator().manual_seed(1)
        vx, vw = torch.randn(x.shape, generator=gen, dtype=torch.float64), torch.randn(w.shape, generator=gen, dtype=torch.float64)
        e = 1e-5
        f = lambda s: float((ref.norm_rope(ref.d64(x) + s * vx, ref.d64(w) + s * vw, 1e-5, tab, pos, False)  # noqa: E731
                             * ref.d64(g)).sum())
        want = (f(e) - f(-e)) / (2 * e)
        got = float((ref.d64(dx) * vx).sum() + (ref.d64(dw) * vw).sum())
        size = float(ref.d64(dx).norm() * vx.norm() + ref.d64(dw).norm() * vw.norm())
        assert abs(got - want) <= 64 * U_F32 * size + 1e-8 * size


def test_default_positions_and_clamping():
    """Without pos a row's position is its place in its example; positions outside the table take its ends."""
    q, k, *_ = inputs(30, 2, 1, 64, torch.float32, False, 5)
    tab = table_of(10, 64)
    a = api.qk_norm_rope(q.view(3, 10, 2, 64), k.view(3, 10, 1, 64), tab)
    pos = torch.arange(10, dtype=torch.int32, device=DEV).repeat(3)
    b = api.qk_norm_rope(q, k, tab, pos=pos)
    assert torch.equal(a[0].view(30, 2, 64), b[0]) and torch.equal(a[1].view(30, 1, 64), b[1])
    c = api.qk_norm_rope(q, k, tab, pos=torch.where(pos == 9, torch.full_like(pos, 1 << 30), torch.where(
        pos == 0, torch.full_like(pos, -5), pos)))
    assert torch.equal(c[0], b[0]) and torch.equal(c[1], b[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extremes(dtype):
    """A zero head, large and tiny values; a NaN stays in its head; no rows."""
    q, k, gq, gk, wq, wk, pos = inputs(4, 4, 1, 64, dtype, False, 6)
    q[0, 0] = 0
    q[1, 1] *= 1e15
    q[2, 2] *= 1e-15
    tab = table_of(300, 64)
    want = ref.norm_rope(q, wq, 1e-5, tab, pos, False)
    got, _ = api.qk_norm_rope(q, k, tab, wq, wk, eps=1e-5, pos=pos)
    assert rel(got, want) <= TOL[dtype]
    q[3, 1, 7] = float("nan")
    got, gk_ = api.qk_norm_rope(q, k, tab, wq, wk, eps=1e-5, pos=pos)
    bad = torch.isnan(got.float()).any(-1)
    assert bool(bad[3, 1]) and int(bad.sum()) == 1 and not torch.isnan(gk_.float()).any()
    e = q[:0]
    dq, dk, dwq, dwk = api.qk_norm_rope_backward(e, k[:0], e, k[:0], tab, wq, wk, pos=pos[:0])
    assert dq.numel() == 0 and float(dwq.abs().sum()) == 0 and float(dwk.abs().sum()) == 0


def test_refusals():
    q, k, gq, gk, wq, wk, pos = inputs(4, 4, 2, 64, torch.bfloat16, False, 7)
    tab = table_of(300, 64)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q.half(), k.half(), tab, pos=pos)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, k.float(), tab, pos=pos)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, k[:3], tab, pos=pos)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, k, tab, wq, None, pos=pos)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, k, tab.double(), pos=pos)
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, k, tab, pos=pos.long())
    with pytest.raises(ValueError):
        api.qk_norm_rope(q.transpose(1, 2), k, tab, pos=pos)
    x = torch.randn(4, 4, 96, device=DEV)
    with pytest.raises(_lib.DrError) as e:
        api.qk_norm_rope(x, x, table_of(4, 96), pos=pos.clamp(max=3))
    assert e.value.status == _lib.DR_ERR_UNSUPPORTED
    off = torch.randn(4 * 4 * 64 + 1, device=DEV).to(torch.bfloat16)[1:].view(4, 4, 64)   # not 16-byte aligned
    with pytest.raises(_lib.DrError) as e:
        api.qk_norm_rope(off, k, tab, pos=pos)
    assert e.value.status == _lib.DR_ERR_ARG


def check_batch(dtype, D, norm, spans, rows, where, given_pos, bad, seed):
    """Rows outside the spans are padding of bits `bad`: zeros come out there, nothing of them enters dwq and dwk, and the
    tokens get what they get without any."""
    q, k, gq, gk, wq, wk, pos = inputs(rows, 6, 2, D, dtype, False, seed)
    if not norm:
        wq = wk = None
    tab = table_of(300, D)
    live = torch.zeros(rows, dtype=torch.bool)
    place = torch.zeros(rows, dtype=torch.int64)
    for a, b in spans:
        live[a:b] = True
        place[a:b] = torch.arange(b - a)
    if not given_pos:
        pos = place.to(torch.int32).to(DEV)
    whole = api.qk_norm_rope(q, k, tab, wq, wk, eps=1e-5, pos=pos)
    for t in (q, k, gq, gk):
        t[~live.to(DEV)] = bad
    if where.get("shape"):
        q, k, gq, gk = [t.view(*where["shape"], *t.shape[1:]) for t in (q, k, gq, gk)]
    kw = dict(offsets=where.get("offsets"), lengths=where.get("lengths"), max_len=where.get("max_len"))
    out = api.qk_norm_rope(q, k, tab, wq, wk, eps=1e-5, pos=pos if given_pos else None, **kw)
    grads = api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, eps=1e-5, pos=pos if given_pos else None, **kw)
    flat = lambda t: t.reshape(rows, -1, D).cpu()     # noqa: E731
    for x, w, o, plain, g, dx, dw in ((q, wq, out[0], whole[0], gq, grads[0], grads[2]),
                                      (k, wk, out[1], whole[1], gk, grads[1], grads[3])):
        assert torch.equal(flat(o)[live], flat(plain)[live])
        assert bool((flat(o)[~live] == 0).all()) and bool((flat(dx)[~live] == 0).all())
        dx_ref, dw_ref = ref.norm_rope_back(flat(g)[live], flat(x)[live], w, 1e-5, tab, pos.cpu()[live], False)
        assert rel(flat(dx)[live], dx_ref) <= 2 * TOL[dtype]
        if norm:
            assert rel(dw, dw_ref) <= TOL_DW
    again = api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, eps=1e-5, pos=pos if given_pos else None, **kw)
    assert all(a is b or torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("norm,given_pos", [(True, False), (True, True), (False, False)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 7.0])
def test_padded_batch(dtype, D, norm, given_pos, bad):
    for N, T in ((5, 33), (1, 1), (900, 7), (4, 1)):
        lens = [(0, 1, T, T // 2, T - 1)[i % 5] for i in range(N)]
        lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
        check_batch(dtype, D, norm, ref.spans_of(None, lens, N, T), N * T, dict(shape=(N, T), lengths=lengths), given_pos, bad, 21)
    lens = [-3, 1 << 30]                             # out of range: none, all
    check_batch(dtype, D, norm, [(9, 18)], 18, dict(shape=(2, 9), lengths=torch.tensor(lens, dtype=torch.int32, device=DEV)),
                given_pos, bad, 22)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 130, 5000])
@pytest.mark.parametrize("given_pos", [False, True])
def test_packed_batch(dtype, N, given_pos):
    """Slots of 0 to 12 rows, lengths inside them, the most tokens of one below the longest slot, rows after the last."""
    slots = [(i * 7 + 3) % 13 for i in range(N)]
    off = [0]
    for n in slots:
        off.append(off[-1] + n)
    lens, most, rows = [(i * 5) % 14 for i in range(N)], 11, off[-1] + 6
    offsets, lengths = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (off, lens))
    spans = [(a, min(b, a + n, a + most)) for a, b, n in zip(off, off[1:], lens)]
    check_batch(dtype, 64, True, spans, rows, dict(offsets=offsets, lengths=lengths, max_len=most), given_pos, float("nan"), 23)
    spans = [(a, min(b, a + most)) for a, b in zip(off, off[1:])]
    check_batch(dtype, 64, True, spans, rows, dict(offsets=offsets, max_len=most), given_pos, float("nan"), 24)
    wild = offsets.clone()
    wild[0], wild[-1] = -5, 1 << 30                  # out of range: the first row, the last
    spans[-1] = (off[-2], min(rows, off[-2] + most))
    check_batch(dtype, 64, True, spans, rows, dict(offsets=wild, max_len=most), given_pos, float("nan"), 25)


def test_batch_without_tokens_and_refusals():
    q, k, gq, gk, wq, wk, pos = inputs(6, 2, 1, 64, torch.bfloat16, False, 26)
    tab = table_of(300, 64)
    none = torch.zeros(2, dtype=torch.int32, device=DEV)
    four = [t.view(2, 3, -1, 64) for t in (q, k, gq, gk)]
    out = (*api.qk_norm_rope(*four[:2], tab, wq, wk, lengths=none),
           *api.qk_norm_rope_backward(*four[2:], *four[:2], tab, wq, wk, lengths=none))
    assert all(float(t.float().abs().max()) == 0 for t in out)
    e = q[:0], k[:0]
    assert all(t.numel() == 0 for t in api.qk_norm_rope(*e, tab, wq, wk, offsets=none[:1], max_len=0))
    for kw in (dict(offsets=none), dict(offsets=none.long(), max_len=3), dict(lengths=none), dict(lengths=none, max_len=4),
               dict(lengths=none.float(), max_len=3), dict(lengths=none[:1], max_len=3)):
        with pytest.raises(ValueError):
            api.qk_norm_rope(q, k, tab, wq, wk, **kw)
        with pytest.raises(ValueError):
            api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, **kw)


def test_side_stream_and_graph():
    """The same bits on another stream, and from replays of a captured graph, with lengths and without."""
    q, k, gq, gk, wq, wk, pos = inputs(260, 4, 2, 64, torch.bfloat16, True, 27)
    tab = table_of(300, 64)
    lengths = torch.tensor([0, 64, 65, 20], dtype=torch.int32, device=DEV)
    for kw in (dict(), dict(lengths=lengths, max_len=65)):
        want = (*api.qk_norm_rope(q, k, tab, wq, wk, pos=pos, **kw), *api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, pos=pos, **kw))
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = (*api.qk_norm_rope(q, k, tab, wq, wk, pos=pos, stream=side, **kw),
               *api.qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, pos=pos, stream=side, **kw))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        out = [torch.empty_like(t) for t in want]
        ws = torch.empty(api.dr_qk_norm_rope_workspace_size(260, 64), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            api.dr_qk_norm_rope(q, k, tab, wq, wk, 1e-6, pos, False, *out[:2], **kw)
            api.dr_qk_norm_rope_backward(gq, gk, q, k, tab, wq, wk, 1e-6, pos, False, *out[2:], workspace=ws, **kw)
        for _ in range(3):
            [t.fill_(7) for t in out]
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, out))
