"""Calls of the graph-transformer operators that are refused on the host, before
anything is launched (no GPU needed)."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2101_11552_amd as tfg
    return tfg.load()


FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call fails its checks first
TOP = 2 ** 31 - 2 ** 20
INVALID, TOO_LARGE, WORKSPACE = 1, 4, 5


def embedding(lib, **kw):
    a = {**dict(table=FAKE, ft=0, V=10, F=8, ldt=8, ids=FAKE, it=0, N=5, scale=1.0, pad=-1, out=FAKE,
                validate=1, ws=FAKE, n=1 << 20), **kw}
    return lib.tfg_embedding(a["table"], a["ft"], a["V"], a["F"], a["ldt"], a["ids"], a["it"], a["N"],
                             a["scale"], a["pad"], a["out"], a["validate"], a["ws"], a["n"], None)


def embedding_backward(lib, **kw):
    a = {**dict(dout=FAKE, ft=0, F=8, ids=FAKE, it=0, N=5, V=10, scale=1.0, pad=-1, dt=FAKE,
                validate=1, ws=FAKE, n=1 << 20), **kw}
    return lib.tfg_embedding_backward(a["dout"], a["ft"], a["F"], a["ids"], a["it"], a["N"], a["V"],
                                      a["scale"], a["pad"], a["dt"], a["validate"], a["ws"], a["n"], None)


@pytest.mark.parametrize("call", [embedding, embedding_backward])
def test_embedding_refusals(lib, call):
    for kw, rc in ((dict(ft=2), INVALID), (dict(it=5), INVALID), (dict(V=-1), INVALID),
                   (dict(N=-1), INVALID), (dict(F=-1), INVALID), (dict(N=TOP), TOO_LARGE),
                   (dict(V=TOP), TOO_LARGE), (dict(pad=10), INVALID), (dict(pad=-2), INVALID),
                   (dict(V=0), INVALID), (dict(ids=None), INVALID), (dict(n=8), WORKSPACE),
                   (dict(ws=None), WORKSPACE), (dict(ws=ctypes.c_void_p(0x1004)), WORKSPACE)):
        assert call(lib, **kw) == rc, kw
    assert embedding(lib, ldt=7) == INVALID
    assert embedding(lib, table=None) == INVALID and embedding(lib, out=None) == INVALID
    assert embedding_backward(lib, dout=None) == INVALID and embedding_backward(lib, dt=None) == INVALID


def norm(lib, **kw):
    a = {**dict(x=FAKE, ft=0, Nb=10, F=8, ldx=8, gi=FAKE, it=0, G=2, K=4, eps=1e-5, act=0, out=FAKE,
                mean=FAKE, rstd=FAKE, ws=FAKE, n=1 << 20), **kw}
    return lib.tfg_group_norm(a["x"], a["ft"], a["Nb"], a["F"], a["ldx"], a["gi"], a["it"], a["G"],
                              a["K"], None, None, a["eps"], a["act"], a["out"], a["mean"], a["rstd"], 1,
                              a["ws"], a["n"], None)


def norm_backward(lib, **kw):
    a = {**dict(x=FAKE, ft=0, Nb=10, F=8, ldx=8, gi=FAKE, it=0, G=2, K=4, act=0, out=FAKE,
                mean=FAKE, rstd=FAKE, ws=FAKE, n=1 << 20), **kw}
    return lib.tfg_group_norm_backward(FAKE, a["x"], a["ft"], a["Nb"], a["F"], a["ldx"], a["gi"],
                                       a["it"], a["G"], a["K"], a["mean"], a["rstd"], None, None,
                                       a["act"], a["out"], FAKE, FAKE, 1, a["ws"], a["n"], None)


@pytest.mark.parametrize("call", [norm, norm_backward])
def test_group_norm_refusals(lib, call):
    for kw, rc in ((dict(ft=-1), INVALID), (dict(it=2), INVALID), (dict(Nb=-1), INVALID),
                   (dict(Nb=TOP), TOO_LARGE), (dict(G=-1), INVALID), (dict(ldx=7), INVALID),
                   (dict(K=0), INVALID), (dict(K=3), INVALID), (dict(act=4), INVALID),
                   (dict(act=-1), INVALID), (dict(G=TOP - 1, K=8), TOO_LARGE), (dict(x=None), INVALID),
                   (dict(out=None), INVALID), (dict(gi=None), INVALID), (dict(mean=None), INVALID),
                   (dict(rstd=None), INVALID), (dict(n=64), WORKSPACE),
                   (dict(ws=ctypes.c_void_p(0x1010)), WORKSPACE)):
        assert call(lib, **kw) == rc, kw
    assert norm(lib, eps=-1.0) == INVALID and norm(lib, eps=float("nan")) == INVALID


def attention(lib, **kw):
    a = {**ATT, **kw}
    return lib.tfg_graph_attention(a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["ft"], a["Nq"],
                                   a["Nk"], a["qo"], a["ko"], a["G"], a["H"], a["Hk"], a["D"], 0.25,
                                   a["cap"], a["bias"], a["B"], a["dist"], a["nd"], a["doff"], a["out"],
                                   FAKE, 1, a["ws"], a["n"], None)


def attention_backward(lib, **kw):
    a = {**ATT, **kw}
    return lib.tfg_graph_attention_backward(
        FAKE, a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["out"], FAKE, a["ft"], a["Nq"],
        a["Nk"], a["qo"], a["ko"], a["G"], a["H"], a["Hk"], a["D"], 0.25, a["cap"], a["bias"], a["B"],
        a["dist"], a["nd"], a["doff"], FAKE, FAKE, FAKE, a.get("dbias"), 1, a["ws"], a["n"], None)


ATT = dict(q=FAKE, ldq=64, k=FAKE, ldk=32, v=FAKE, ldv=32, ft=1, Nq=10, Nk=12, qo=FAKE, ko=FAKE, G=2,
           H=4, Hk=2, D=16, cap=0.0, bias=FAKE, B=5, dist=FAKE, nd=120, doff=FAKE, out=FAKE, ws=FAKE,
           n=1 << 24)


@pytest.mark.parametrize("call", [attention, attention_backward])
def test_attention_refusals(lib, call):
    for kw, rc in ((dict(ft=2), INVALID), (dict(Nq=-1), INVALID), (dict(Nk=TOP), TOO_LARGE),
                   (dict(G=-1), INVALID), (dict(H=0), INVALID), (dict(Hk=3), INVALID),
                   (dict(Hk=0), INVALID), (dict(H=2048, Hk=2048, ldq=1 << 20, ldk=1 << 20, ldv=1 << 20), INVALID),
                   (dict(D=0), INVALID), (dict(D=129, ldq=1024, ldk=1024, ldv=1024), INVALID),
                   (dict(ldq=63), INVALID), (dict(ldk=31), INVALID), (dict(ldv=31), INVALID),
                   (dict(cap=-1.0), INVALID), (dict(cap=float("nan")), INVALID),
                   (dict(cap=float("inf")), INVALID), (dict(B=256), INVALID), (dict(B=-1), INVALID),
                   (dict(H=64, Hk=1, B=65, ldq=1024), INVALID), (dict(bias=None), INVALID),
                   (dict(dist=None), INVALID), (dict(doff=None), INVALID), (dict(nd=-1), INVALID),
                   (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(q=None), INVALID),
                   (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
                   (dict(n=8), WORKSPACE), (dict(ws=None), WORKSPACE),
                   (dict(ws=ctypes.c_void_p(0x1080)), WORKSPACE)):
        assert call(lib, **kw) == rc, kw
    assert attention_backward(lib, B=0, bias=None, dbias=FAKE) == INVALID


def test_size_queries(lib):
    assert lib.tfg_embedding_ws_bytes() >= 4
    assert lib.tfg_embedding_backward_ws_bytes(1000, 50, 64) >= 3 * 4 * 1000
    assert lib.tfg_embedding_backward_ws_bytes(-1, 50, 64) == 0
    assert lib.tfg_group_norm_ws_bytes(100, 64, 7, 4) >= 8 * 4
    assert lib.tfg_group_norm_backward_ws_bytes(100, 64, 7, 4) > lib.tfg_group_norm_ws_bytes(100, 64, 7, 4)
    assert lib.tfg_group_norm_ws_bytes(100, 64, 7, 0) == 0
    few = lib.tfg_graph_attention_ws_bytes(4, 400000, 4, 8, 8, 64)
    assert few > lib.tfg_graph_attention_ws_bytes(400000, 400000, 4, 8, 8, 64)  # keys are split
    assert lib.tfg_graph_attention_backward_ws_bytes(1000, 1000, 4, 8, 8, 64, 0) >= 4 * 8 * 1000
    assert lib.tfg_graph_attention_ws_bytes(10, 10, 1, 3, 2, 16) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch
    import paper_2101_11552_amd as tfg
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    off = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        tfg.tfg_embedding(x, ids)
    with pytest.raises(ValueError):
        tfg.tfg_embedding_backward(x, ids, 4)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x, ids, 1, 2)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm_backward(x, x, ids, 1, 2, x, x)
    with pytest.raises(ValueError):
        tfg.tfg_graph_attention(x, x, x, off, 2)
    with pytest.raises(ValueError):
        tfg.tfg_graph_attention_backward(x, x, x, x, x, x, off, 2)


@pytest.mark.parametrize("call", [attention, attention_backward])
def test_attention_cap_refusals(lib, call):
    """A cap whose tanh bfloat16's form would not resolve, and one that scale / cap overflows."""
    assert call(lib, ft=1, cap=4097.0) == INVALID
    assert call(lib, cap=1e-38) == INVALID and call(lib, ft=1, cap=1e-39) == INVALID
    # (with a workspace too small: the next check is reached)
    assert call(lib, ft=1, cap=4096.0, n=8) == WORKSPACE
    assert call(lib, ft=0, cap=1e30, n=8) == WORKSPACE
    assert call(lib, cap=1e-30, n=8) == WORKSPACE
