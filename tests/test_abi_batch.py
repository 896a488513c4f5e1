"""The merged batch's operators refuse invalid arguments before any HIP call."""

import os

import pytest

from paper_2605_07063_amd import _lib
from paper_2605_07063_amd._lib import (DR_BF16, DR_ERR_ARG, DR_ERR_DTYPE, DR_ERR_UNSUPPORTED, DR_ERR_WORKSPACE, DR_F32,
                                       DR_OK)

FAKE = 0x1000_0000   # 16-byte aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2605_07063_amd import build
        build.build()
    return _lib.load()


def rope(lib, back=False, **kw):
    d = dict(q=FAKE, ldq=256, k=FAKE, ldk=128, rows=10, T=10, Hq=4, Hkv=2, D=64, dtype=DR_BF16, wq=FAKE, wk=FAKE, eps=1e-6,
             table=FAKE, table_rows=16, pos=None, pairing=0, oq=FAKE, ldoq=256, ok=FAKE, ldok=128, gq=FAKE, gk=FAKE,
             dwq=FAKE, dwk=FAKE, ws=FAKE, wsb=1 << 30)
    d.update(kw)
    mid = [d[n] for n in ("q", "ldq", "k", "ldk", "rows", "T", "Hq", "Hkv", "D", "dtype", "wq", "wk", "eps", "table",
                          "table_rows", "pos", "pairing", "oq", "ldoq", "ok", "ldok")]
    if back:
        return lib.dr_qk_norm_rope_backward(d["gq"], 256, d["gk"], 128, *mid, d["dwq"], d["dwk"], d["ws"], d["wsb"], None)
    return lib.dr_qk_norm_rope(*mid, None)


@pytest.mark.parametrize("back", [False, True])
def test_rope(lib, back):
    for kw, want in [(dict(rows=-1), DR_ERR_ARG), (dict(Hq=0), DR_ERR_ARG), (dict(Hkv=-1), DR_ERR_ARG),
                     (dict(dtype=5), DR_ERR_DTYPE), (dict(D=96), DR_ERR_UNSUPPORTED), (dict(ldq=248), DR_ERR_ARG),
                     (dict(ldq=260), DR_ERR_ARG), (dict(q=FAKE + 8), DR_ERR_ARG), (dict(table=None), DR_ERR_ARG),
                     (dict(table_rows=0), DR_ERR_ARG), (dict(T=0), DR_ERR_ARG), (dict(wk=None), DR_ERR_ARG),
                     (dict(eps=-1.0), DR_ERR_ARG), (dict(eps=float("nan")), DR_ERR_ARG), (dict(pairing=2), DR_ERR_ARG),
                     (dict(oq=None), DR_ERR_ARG), (dict(ldok=64), DR_ERR_ARG)]:
        assert rope(lib, back, **kw) == want, kw
    if back:
        assert rope(lib, True, ws=None) == DR_ERR_WORKSPACE
        assert rope(lib, True, wsb=8) == DR_ERR_WORKSPACE
        assert rope(lib, True, dwq=None) == DR_ERR_ARG
        assert rope(lib, True, wq=None, wk=None, q=None, k=None, rows=0) == DR_OK
    else:
        assert rope(lib, rows=0) == DR_OK
    assert lib.dr_qk_norm_rope_workspace_size(0, 64) == 0 and lib.dr_qk_norm_rope_workspace_size(100, 64) > 0


def attn(lib, back=False, **kw):
    d = dict(q=FAKE, ldq=256, k=FAKE, ldk=128, v=FAKE, ldv=128, o=FAKE, ldo=256, lse=FAKE, rows=64, N=2, T=32, off=None,
             len=None, Hq=4, Hkv=2, D=64, dtype=DR_BF16, scale=0.125, g=FAKE, dq=FAKE, lddq=256, dk=FAKE, dv=FAKE, ws=FAKE,
             wsb=1 << 30)
    d.update(kw)
    qkv = [d[n] for n in ("q", "ldq", "k", "ldk", "v", "ldv")]
    shape = [d[n] for n in ("rows", "N", "T", "off", "len", "Hq", "Hkv", "D", "dtype", "scale")]
    if back:
        return lib.dr_attention_backward(d["g"], 256, *qkv, d["o"], d["ldo"], d["lse"], *shape, d["dq"], d["lddq"], d["dk"],
                                         128, d["dv"], 128, d["ws"], d["wsb"], None)
    return lib.dr_attention(*qkv, *shape, d["o"], d["ldo"], d["lse"], None)


@pytest.mark.parametrize("back", [False, True])
def test_attention(lib, back):
    for kw, want in [(dict(rows=-1), DR_ERR_ARG), (dict(rows=63), DR_ERR_ARG), (dict(N=-1), DR_ERR_ARG),
                     (dict(Hq=3), DR_ERR_ARG), (dict(Hkv=0), DR_ERR_ARG), (dict(D=80, ldq=320, ldk=160), DR_ERR_UNSUPPORTED),
                     (dict(dtype=DR_F32), DR_ERR_UNSUPPORTED), (dict(dtype=9), DR_ERR_DTYPE), (dict(scale=0.0), DR_ERR_ARG),
                     (dict(scale=-1.0), DR_ERR_ARG), (dict(scale=float("inf")), DR_ERR_ARG), (dict(ldk=120), DR_ERR_ARG),
                     (dict(ldv=132), DR_ERR_ARG), (dict(q=None), DR_ERR_ARG), (dict(v=FAKE + 2), DR_ERR_ARG),
                     (dict(o=None), DR_ERR_ARG), (dict(lse=None), DR_ERR_ARG), (dict(off=FAKE, N=0), DR_ERR_ARG),
                     (dict(rows=1 << 31, N=1, T=1 << 31), DR_ERR_UNSUPPORTED),
                     (dict(off=FAKE, N=1 << 22, T=1 << 20), DR_ERR_UNSUPPORTED)]:
        assert attn(lib, back, **kw) == want, kw
    assert attn(lib, back, rows=0, N=0) == DR_OK
    if back:
        assert attn(lib, True, ws=None) == DR_ERR_WORKSPACE
        assert attn(lib, True, wsb=64) == DR_ERR_WORKSPACE
        assert attn(lib, True, dq=None) == DR_ERR_ARG and attn(lib, True, g=None) == DR_ERR_ARG
    assert lib.dr_attention_workspace_size(0, 4, 2, 64) == 0 and lib.dr_attention_workspace_size(64, 4, 2, 64) >= 64 * 4 * 4


def xent(lib, back=False, **kw):
    d = dict(h=FAKE, ldh=64, W=FAKE, ldw=64, t=FAKE, M=10, V=100, D=64, dtype=DR_BF16, loss=FAKE, lse=FAKE, g=FAKE, dh=FAKE,
             lddh=64, dW=FAKE, lddw=64, ws=FAKE, wsb=1 << 40)
    d.update(kw)
    head = [d[n] for n in ("h", "ldh", "W", "ldw", "t")]
    if back:
        return lib.dr_cross_entropy_backward(*head, d["lse"], d["g"], d["M"], d["V"], d["D"], d["dtype"], d["dh"], d["lddh"],
                                             d["dW"], d["lddw"], d["ws"], d["wsb"], None)
    return lib.dr_cross_entropy(*head, d["M"], d["V"], d["D"], d["dtype"], d["loss"], d["lse"], d["ws"], d["wsb"], None)


@pytest.mark.parametrize("back", [False, True])
def test_cross_entropy(lib, back):
    for kw, want in [(dict(M=-1), DR_ERR_ARG), (dict(V=0), DR_ERR_ARG), (dict(D=60), DR_ERR_ARG), (dict(D=0), DR_ERR_ARG),
                     (dict(dtype=DR_F32), DR_ERR_UNSUPPORTED), (dict(dtype=4), DR_ERR_DTYPE), (dict(ldh=56), DR_ERR_ARG),
                     (dict(ldw=68), DR_ERR_ARG), (dict(h=FAKE + 4), DR_ERR_ARG), (dict(W=None), DR_ERR_ARG),
                     (dict(t=None), DR_ERR_ARG), (dict(lse=None), DR_ERR_ARG), (dict(M=1 << 31), DR_ERR_UNSUPPORTED),
                     (dict(ws=None), DR_ERR_WORKSPACE), (dict(wsb=100), DR_ERR_WORKSPACE), (dict(ws=FAKE + 4), DR_ERR_ARG)]:
        assert xent(lib, back, **kw) == want, kw
    if back:
        assert xent(lib, True, g=None) == DR_ERR_ARG and xent(lib, True, lddh=32) == DR_ERR_ARG
        assert xent(lib, True, dh=None, dW=None) == DR_OK
        assert xent(lib, True, M=0, dW=None) == DR_OK
    else:
        assert xent(lib, loss=None) == DR_ERR_ARG
        assert xent(lib, M=0) == DR_OK
    for b in (0, 1):
        assert lib.dr_cross_entropy_workspace_size(0, 100, 64, b) == 0
        assert lib.dr_cross_entropy_workspace_size(64, 1000, 64, b) > 0


@pytest.mark.parametrize("back", [False, True])
def test_rope_grid(lib, back):
    # a workgroup of 256 threads takes 4 rows, and a launch fewer than 2^32 threads
    rows = 4 * ((1 << 24) - 1)
    assert rope(lib, back, rows=rows + 1) == DR_ERR_UNSUPPORTED
    if back:
        assert rope(lib, True, rows=rows, ws=None) == DR_ERR_WORKSPACE


@pytest.mark.parametrize("back", [False, True])
def test_cross_entropy_grid(lib, back):
    # a launch takes fewer than 2^24 workgroups of 256 threads: one a token, 256 x 256 logits, or 64 x 256 with D < 256
    for M, V, D, ok in [(1 << 24, 8, 8, False), ((1 << 24) - 1, 8, 8, True),
                        (1 << 23, 1 << 17, 256, False), (1 << 22, 1 << 17, 256, True),
                        (1 << 21, 1 << 17, 64, False), (1 << 20, 1 << 17, 64, True),
                        (64, 1 << 30, 64, False), (64, 1 << 29, 64, True)]:
        d = dict(ldh=D, ldw=D, lddh=D, lddw=D, M=M, V=V, D=D)
        assert (xent(lib, back, ws=None, **d) == (DR_ERR_WORKSPACE if ok else DR_ERR_UNSUPPORTED)), d
        assert (lib.dr_cross_entropy_workspace_size(M, V, D, int(back)) > 0) == ok, d


@pytest.mark.parametrize("back", [False, True])
def test_cross_entropy_leading_dimensions(lib, back):
    # h, dh and dW may have any (one token of every long example: T D between rows); W's rows, of which a tile spans 256
    # at 32-bit offsets, are at most 2^22 apart
    for ld, ok in [(1 << 22, True), ((1 << 22) + 8, False)]:
        assert xent(lib, back, ldw=ld, ws=None) == (DR_ERR_WORKSPACE if ok else DR_ERR_ARG)
    for ld, ok in [(1 << 24, True), (1 << 32, True), ((1 << 32) + 8, False)]:
        for name in ("ldh", "lddh", "lddw") if back else ("ldh",):
            assert xent(lib, back, ws=None, **{name: ld}) == (DR_ERR_WORKSPACE if ok else DR_ERR_ARG), (name, ld)


@pytest.mark.parametrize("back", [False, True])
def test_rope_batch(lib, back):
    def call(**kw):
        d = dict(rows=64, N=2, T=32, off=None, len=FAKE, pos=None, D=64, ldq=256, table=FAKE, ws=FAKE, wsb=1 << 30)
        d.update(kw)
        head = [FAKE, d["ldq"], FAKE, 128, d["rows"], d["N"], d["T"], d["off"], d["len"], 4, 2, d["D"], DR_BF16, FAKE, FAKE,
                1e-6, d["table"], 16, d["pos"], 0, FAKE, 256, FAKE, 128]
        if back:
            return lib.dr_qk_norm_rope_batch_backward(FAKE, 256, FAKE, 128, *head, FAKE, FAKE, d["ws"], d["wsb"], None)
        return lib.dr_qk_norm_rope_batch(*head, None)
    for kw, want in [(dict(N=-1), DR_ERR_ARG), (dict(T=-1, pos=FAKE), DR_ERR_ARG), (dict(rows=63), DR_ERR_ARG),
                     (dict(off=FAKE, N=0), DR_ERR_ARG), (dict(D=96), DR_ERR_UNSUPPORTED), (dict(ldq=248), DR_ERR_ARG),
                     (dict(table=None), DR_ERR_ARG), (dict(off=FAKE, T=1 << 31), DR_ERR_UNSUPPORTED),
                     (dict(off=FAKE, N=1 << 31), DR_ERR_UNSUPPORTED)]:
        assert call(**kw) == want, kw
    if back:
        assert call(ws=None) == DR_ERR_WORKSPACE and call(wsb=8) == DR_ERR_WORKSPACE
    else:
        assert call(rows=0, N=0) == DR_OK and call(rows=0, N=2, T=0) == DR_OK
