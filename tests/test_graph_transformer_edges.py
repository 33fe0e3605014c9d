"""The graph-transformer operators where their kernels change form: biases of the type's
lowest value in the gradients, scales that are negative or zero, queries split over
blocks, empty inputs, matrices and distances past 2^31 elements, workspaces. References
and bounds as in test_graph_transformer.py (u = 2^-24)."""

import math

import numpy as np
import pytest

from test_graph_transformer import SIZES, Case, U, ints, layer, layer_state, normal, tfg, within  # noqa: F401

pytestmark = pytest.mark.gpu


def lowest_reference(c):
    """Outputs and gradients in double of a case whose bucket 0 has the type's lowest value:
    in a row with other unmasked buckets it has no weight, alone it shares the row evenly
    (a score is rounded to the bias). With sums of the terms' sizes for the bounds."""
    import torch
    f64 = dict(dtype=torch.float64, device="cuda")
    H, Hk, D = c.H, c.Hk, c.D
    r = {k: torch.zeros(n, h * D, **f64) for k, n, h in (
        ("out", c.Nq, H), ("dq", c.Nq, H), ("dk", c.Nk, Hk), ("dv", c.Nk, Hk))}
    r["dbias"] = torch.zeros(H, c.B, **f64)
    size = {k: torch.zeros_like(v) for k, v in r.items()}
    for g, (nq, nk) in enumerate(c.sizes):
        if nq == 0 or nk == 0:
            continue
        q0, k0, o = int(c.qo[g]), int(c.ko[g]), int(c.doff[g])
        dist = c.dist[o:o + nq * nk].view(nq, nk).long()
        for h in range(H):
            hk = h // (H // Hk)
            qs, ks = slice(h * D, (h + 1) * D), slice(hk * D, (hk + 1) * D)
            q, do = c.q[q0:q0 + nq, qs].double(), c.dout[q0:q0 + nq, qs].double()
            k, v = c.k[k0:k0 + nk, ks].double(), c.v[k0:k0 + nk, ks].double()
            s = q @ k.t() * c.scale
            live = dist < c.B
            plain = live & (dist > 0)
            some = plain.any(1, keepdim=True)
            u = torch.where(some, s + c.bias[h].double()[dist.clamp(max=c.B - 1)], 0.0)
            u = torch.where(torch.where(some, plain, live), u, -math.inf)
            p = torch.nan_to_num(torch.softmax(u, 1), nan=0.0)  # (rows without any key)
            out, dp = p @ v, do @ v.t()
            delta = (p * dp).sum(1, keepdim=True)
            du = p * (dp - delta)
            sd = p * (do.abs() @ v.abs().t() + (do.abs() * (p @ v.abs())).sum(1, keepdim=True))
            flat = dist.clamp(max=c.B).view(-1)
            sums = lambda x: torch.zeros(c.B + 1, **f64).index_add_(0, flat, x.view(-1))[:c.B]  # noqa: E731
            for key, at, a, b in (
                    ("out", (slice(q0, q0 + nq), qs), out, p @ v.abs()),
                    ("dq", (slice(q0, q0 + nq), qs), du @ k * c.scale, sd @ k.abs() * abs(c.scale)),
                    ("dk", (slice(k0, k0 + nk), ks), du.t() @ q * c.scale, sd.t() @ q.abs() * abs(c.scale)),
                    ("dv", (slice(k0, k0 + nk), ks), p.t() @ do, p.t() @ do.abs()),
                    ("dbias", h, sums(du), sums(sd))):
                r[key][at] += a
                size[key][at] += b
    return r, size


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,H,Hk,D", [("batch", 2, 1, 16), ("middle", 2, 2, 24), ("many", 8, 4, 16),
                                          ("many", 4, 4, 32), ("split", 2, 1, 64)])
def test_gradient_lowest_value_bias(tfg, name, sizes, H, Hk, D):
    """Rows with nothing but such a bucket, and rows with others beside it."""
    import torch
    c = Case(name, SIZES[sizes], H, Hk, D, 0.0, 5, seed=80)
    c.bias[:, 0] = torch.finfo(c.bias.dtype).min
    rng = np.random.default_rng(81)
    for g, (nq, nk) in enumerate(c.sizes):
        d = c.dist[int(c.doff[g]):int(c.doff[g]) + nq * nk].view(nq, nk)
        rows = torch.from_numpy(rng.random(nq) < 0.4).cuda()
        d[rows] = torch.where(d[rows] < 5, 0, d[rows]).to(d.dtype)
    out, lse = c.forward(tfg)
    got = dict(zip(("dq", "dk", "dv", "dbias"), c.backward(tfg, out, lse)), out=out)
    ref, size = lowest_reference(c)
    w = 2.0 ** -8 if name == "bf16" else U
    # bf16: weights and du are operands of the type, delta of long rows comes from the rounded
    # output, the result is rounded: 4 half steps of the terms' sizes. float32: the scores are at
    # most 12 (products of D unit normals over sqrt(D)) with D + 8 roundings, the weight's sum
    # has nk terms, a gradient's sum max(nq H / Hk, nk), and 32 for the factors.
    n = max(max(nk, nq * H // Hk) for nq, nk in c.sizes)
    rel = 4 * w + (12 * 2 * (D + 8) + 2 * n + 32) * U
    for key in ref:
        within(got[key], ref[key], rel * size[key] + 1e-37, key)
    again = c.backward(tfg, out, lse, validate=False)
    assert all(torch.equal(a, got[k]) for a, k in zip(again, ("dq", "dk", "dv", "dbias")))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("sizes,H,Hk,D,cap,B", [
    ("batch", 4, 2, 16, 2.0, 0), ("middle", 2, 1, 64, 0.0, 6), ("split", 2, 2, 32, 0.0, 0),
    ("many", 4, 4, 16, 0.0, 0), ("many", 4, 4, 16, 3.0, 7)])
def test_attention_scales(tfg, name, scale, sizes, H, Hk, D, cap, B):
    Case(name, SIZES[sizes], H, Hk, D, cap, B, seed=90, scale=scale).check(tfg)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,H,Hk,D,cap,B", [
    ([(1500, 300)], 8, 2, 64, 0.0, 6), ([(1200, 40), (0, 7), (1111, 90)], 6, 2, 16, 4.0, 0),
    ([(700, 129)], 4, 1, 128, 0.0, 9), ([(900, 70)], 3, 1, 21, 0.0, 0)])
def test_gradient_queries_in_parts(tfg, name, sizes, H, Hk, D, cap, B):
    """Few keys, many rows: a key tile's queries are several blocks'."""
    Case(name, sizes, H, Hk, D, cap, B, seed=100).check(tfg)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[], [(0, 0)], [(0, 5)], [(5, 0)], [(0, 0)] * 700])
def test_attention_nothing(tfg, name, sizes):
    """No graphs, no queries, no keys."""
    import torch
    c = Case(name, sizes, 2, 2, 16, 0.0, 3, seed=110)
    out, lse = c.forward(tfg)
    assert out.shape == (c.Nq, 32) and bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv, dbias = c.backward(tfg, out, lse)
    for x, like in ((dq, c.q), (dk, c.k), (dv, c.v), (dbias, c.bias)):
        assert x.shape == like.shape and bool((x == 0).all())
    torch.cuda.synchronize()


def test_attention_large_bias_tables(tfg):
    """Many small graphs whose heads' bias tables leave no room for a wavefront a graph."""
    c = Case("f32", SIZES["many"], 64, 4, 128, 0.0, 255, seed=115)
    out, lse = c.forward(tfg)
    ref = c.reference()
    within(out, ref["out"], ref["t_out"] + 1e-37, "out")
    dq, dk, dv, dbias = c.backward(tfg, out, lse)
    for x, key in ((dq, "dq"), (dk, "dk"), (dv, "dv"), (dbias, "dbias")):
        within(x, ref[key], ref["t_" + key] + 1e-37, key)


def test_group_norm_nothing(tfg):
    import torch
    x = normal(120, 0, 16)
    gi = ints([], "int64")
    for G in (0, 3):
        out, mean, rstd = tfg.tfg_group_norm(x, gi, G, 4)
        assert out.shape == (0, 16) and mean.shape == rstd.shape == (G, 4)
        dx, dg, db = tfg.tfg_group_norm_backward(x, x, gi, G, 4, mean, rstd,
                                                 torch.ones(16, device="cuda"), torch.ones(16, device="cuda"))
        assert dx.shape == (0, 16) and bool((dg == 0).all()) and bool((db == 0).all())


def test_caller_workspaces(tfg):
    """A workspace of the caller's, larger than asked for, with anything in it: the same bits."""
    import torch
    ws = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN as floats)
    for sizes in ("split", "many", "middle"):
        c = Case("bf16", SIZES[sizes], 4, 4, 16, 0.0, 6, seed=130)
        out, lse = c.forward(tfg)
        grads = c.backward(tfg, out, lse)
        ws.fill_(0xFF)
        again = c.forward(tfg, ws=ws)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
        ws.fill_(0xFF)
        assert all(torch.equal(a, b) for a, b in zip(grads, c.backward(tfg, out, lse, ws=ws)))
    ids = ints(np.random.default_rng(131).integers(0, 50, 3000), "int64")
    d = normal(132, 3000, 24)
    a = tfg.tfg_embedding_backward(d, ids, 50)
    ws.fill_(0xFF)
    assert torch.equal(a, tfg.tfg_embedding_backward(d, ids, 50, ws=ws))
    gi = ints(np.sort(np.random.default_rng(133).integers(0, 9, 3000)), "int64")
    a = tfg.tfg_group_norm(d, gi, 9, 4)
    b = tfg.tfg_group_norm_backward(d, d, gi, 9, 4, *a[1:])
    ws.fill_(0xFF)
    assert all(torch.equal(s, t) for s, t in zip(a, tfg.tfg_group_norm(d, gi, 9, 4, ws=ws)))
    ws.fill_(0xFF)
    again = tfg.tfg_group_norm_backward(d, d, gi, 9, 4, *a[1:], ws=ws)
    assert all(torch.equal(s, t) for s, t in zip(b, again))
    small = torch.full((8,), 9, dtype=torch.uint8, device="cuda")  # too small: not used
    assert torch.equal(tfg.tfg_group_norm(d, gi, 9, 4, ws=small)[0], a[0])
    assert bool((small == 9).all())


def test_two_captured_graphs(tfg):
    """Two captured steps, replayed in turn and again after eager work: the eager bits."""
    import torch
    states = [layer_state(tfg, "bf16", (300, 40, 700), seed=s) for s in (140, 150)]
    eager = [layer(tfg, st, "bf16") for st in states]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for st in states:
            layer(tfg, st, "bf16")
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for st in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = layer(tfg, st, "bf16")
        graphs.append((graph, outs))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, outs), ref in zip(graphs, eager):
            assert all(torch.equal(a, b) for a, b in zip(outs, ref))
        layer(tfg, states[0], "bf16")


def test_embedding_past_2_31_elements(tfg):
    import torch
    V, F = (1 << 31) // 128 + 1000, 128
    table = torch.zeros(V, F, dtype=torch.bfloat16, device="cuda")
    rows = normal(160, 500, F, name="bf16")
    table[-500:] = rows
    ids = ints(np.arange(V - 500, V), "int64")
    assert torch.equal(tfg.tfg_embedding(table, ids), rows)
    del table
    grad = tfg.tfg_embedding_backward(rows, ids, V)
    assert torch.equal(grad[-500:], rows) and bool((grad[-1500:-500] == 0).all())


def test_group_norm_past_2_31_elements(tfg):
    import torch
    N, F = (1 << 31) // 128 + 1000, 128
    x = torch.zeros(N, F, dtype=torch.bfloat16, device="cuda")
    rows = normal(170, 400, F, name="bf16")
    x[-400:] = rows
    gi = torch.zeros(N, dtype=torch.int32, device="cuda")
    gi[-400:] = 1
    out, mean, rstd = tfg.tfg_group_norm(x, gi, 2, 8)
    one = ints(np.zeros(400))
    ref, m1, r1 = tfg.tfg_group_norm(rows, one, 1, 8)
    # (other orders of the same double sums: a rounding of mean and rstd more, then bf16's step)
    within(mean[1], m1[0].double(), 4 * U * m1[0].double().abs() + 1e-9, "mean")
    within(rstd[1], r1[0].double(), 4 * U * r1[0].double().abs(), "rstd")
    within(out[-400:], ref.double(), 2.0 ** -7 * ref.double().abs() + 1e-6, "out")
    dx = tfg.tfg_group_norm_backward(x, x, gi, 2, 8, mean, rstd, want_params=False)[0]
    d1 = tfg.tfg_group_norm_backward(rows, rows, one, 1, 8, m1, r1, want_params=False)[0]
    within(dx[-400:], d1.double(), 2.0 ** -7 * d1.double().abs() + 1e-5, "dx")


def test_attention_past_2_31(tfg):
    """Distances and keys that lie past 2^31 bytes and elements: the last rows of a graph of
    50,000 nodes, and a graph at the end of 2^31 elements, as in a call of their own."""
    import torch
    n, last = 50000, 64
    q, k, v = (normal(180 + i, n, 16, name="bf16") for i in range(3))
    dist = torch.zeros(n * n, dtype=torch.uint8, device="cuda")
    tail = torch.from_numpy(np.random.default_rng(183).integers(0, 5, last * n).astype(np.uint8)).cuda()
    dist[-last * n:] = tail
    bias = normal(184, 1, 4, name="bf16")
    a = dict(bias=bias, want_lse=True)
    out, lse = tfg.tfg_graph_attention(q, k, v, ints([0, n]), 1, distance=dist,
                                       distance_offsets=ints([0], "int64"), **a)
    ref, rl = tfg.tfg_graph_attention(q[-last:], k, v, ints([0, last]), 1, k_offsets=ints([0, n]),
                                      distance=tail, distance_offsets=ints([0], "int64"), **a)
    # both sum n terms of weights rounded to bf16, in other orders: a step of the output and
    # n u of the values' sizes apart
    within(out[-last:], ref.double(), 2.0 ** -7 * ref.double().abs() + n * U * 4.0, "out")
    within(lse[-last:], rl.double(), (n + 64) * U + 0 * rl.double(), "lse")
    del a["want_lse"]
    dout = torch.zeros(n, 16, dtype=torch.bfloat16, device="cuda")
    dout[-last:] = normal(185, last, 16, name="bf16")
    got = tfg.tfg_graph_attention_backward(dout, q, k, v, out, lse, ints([0, n]), 1, distance=dist,
                                           distance_offsets=ints([0], "int64"), **a)
    one = tfg.tfg_graph_attention_backward(dout[-last:], q[-last:], k, v, ref, rl, ints([0, last]), 1,
                                           k_offsets=ints([0, n]), distance=tail,
                                           distance_offsets=ints([0], "int64"), **a)
    for x, y, what in zip((got[0][-last:],) + got[1:3], one[:3], ("dq", "dk", "dv")):
        # outputs a bf16 step apart change delta, and so every du of the row, by as much of sizes
        assert float((x.double() - y.double()).norm()) <= 2.0 ** -6 * float(y.double().norm()), what
    del dist, q, k, v, out, got
    rows = (1 << 31) // 128 + 300
    wide = torch.zeros(rows, 128, dtype=torch.bfloat16, device="cuda")
    wide[-200:] = normal(186, 200, 128, name="bf16")
    x = wide[-200:]
    at = rows - 200
    big = tfg.tfg_graph_attention(wide, wide, wide, ints([at, rows]), 2)
    assert torch.equal(big[-200:], tfg.tfg_graph_attention(x, x, x, ints([0, 200]), 2))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_the_same_tensor_for_all(tfg, name):
    """q, k and v may be one tensor; the last graph's rows may be one node."""
    import torch
    x = normal(190, 77, 32, name=name)
    off = ints([0, 40, 76, 77])
    out, lse = tfg.tfg_graph_attention(x, x, x, off, 2, want_lse=True)
    parts = [t.clone() for t in (x, x, x)]
    ref, rl = tfg.tfg_graph_attention(*parts, off, 2, want_lse=True)
    assert torch.equal(out, ref) and torch.equal(lse, rl)
    assert torch.equal(out[-1], x[-1])  # a single key has all the weight
