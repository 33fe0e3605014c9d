"""The operators of a graph-transformer layer over a BatchGraph, as a user's program calls them.

Each case names an operator, its sizes and its options:

* ``embed``      rows of a table by node type or token id, scaled
* ``embed_train``  the same, and the table's gradient by sorted ids
* ``norm``       group norm per graph with an activation, channels last
* ``norm_train``   the same, and its gradients
* ``attn``       attention inside each graph: scores capped by a tanh, a bias by hop distance,
                 shared key/value heads, a readout of one query per graph
* ``attn_train``   the same, and its gradients

Graphs are contiguous runs of nodes (a BatchGraph). Their sizes come from the case alone, the
values of features, ids, distances and gradients from the seed. With ``own`` the calls are the
framework's, otherwise elementary torch operations in 32 bits (long sums in 64).
"""

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # a handful of atom types looked up for one small molecule: launches and latency
        {"name": "embed_one", "kind": "embed", "type": "f32", "N": 7, "V": 119, "F": 64,
         "ids": "uniform", "index": "int64", "scale": 1.0, "pad": -1},
        # the atom types of a mini-batch of 4,096 graphs: few rows, every one of them hot
        {"name": "embed_batch_train", "kind": "embed_train", "type": "f32", "N": 143360, "V": 119,
         "F": 128, "ids": "uniform", "index": "int64", "scale": 1.0, "pad": 0},
        # words of a text-attributed graph: a large table read by Zipf's law, an odd width
        {"name": "embed_zipf_train", "kind": "embed_train", "type": "bf16", "N": 500000,
         "V": 100003, "F": 300, "ids": "zipf", "index": "int32", "scale": 17.32, "pad": -1},
        # instance norm of a small mini-batch at inference
        {"name": "norm_small", "kind": "norm", "type": "f32", "G": 128, "lo": 10, "hi": 60,
         "F": 64, "groups": 64, "act": "relu"},
        # the training step's norm over a mini-batch of 4,096 graphs
        {"name": "norm_batch_train", "kind": "norm_train", "type": "bf16", "G": 4096, "lo": 10,
         "hi": 60, "F": 128, "groups": 8, "act": "gelu"},
        # one citation graph as a single sample
        {"name": "norm_large_train", "kind": "norm_train", "type": "f32", "G": 1, "lo": 169343,
         "hi": 169343, "F": 128, "groups": 32, "act": "silu"},
        # the readout of eight small graphs, one query each: launches and latency
        {"name": "attn_readout_small", "kind": "attn", "type": "f32", "G": 8, "lo": 40, "hi": 200,
         "queries": 1, "H": 4, "Hk": 4, "D": 16, "cap": 0.0, "B": 0},
        # the training step's attention over a mini-batch of 4,096 graphs
        {"name": "attn_batch_train", "kind": "attn_train", "type": "bf16", "G": 4096, "lo": 10,
         "hi": 60, "queries": 0, "H": 8, "Hk": 8, "D": 16, "cap": 0.0, "B": 16},
        # graphs of hundreds of nodes in float32, capped scores and hop distances
        {"name": "attn_mid_train", "kind": "attn_train", "type": "f32", "G": 96, "lo": 100,
         "hi": 500, "queries": 0, "H": 8, "Hk": 8, "D": 16, "cap": 20.0, "B": 20},
        # inference over three large graphs, capped scores
        {"name": "attn_large", "kind": "attn", "type": "bf16", "G": 3, "lo": 4000, "hi": 9000,
         "queries": 0, "H": 8, "Hk": 8, "D": 64, "cap": 30.0, "B": 0},
        # the readout of a few very large graphs, one query each, shared key/value heads
        {"name": "attn_readout_long", "kind": "attn", "type": "bf16", "G": 6, "lo": 20000,
         "hi": 60000, "queries": 1, "H": 16, "Hk": 4, "D": 64, "cap": 0.0, "B": 0},
        # training on two citation graphs, wide heads that share keys, hop distances
        {"name": "attn_large_train", "kind": "attn_train", "type": "bf16", "G": 2, "lo": 2708,
         "hi": 3327, "queries": 0, "H": 8, "Hk": 2, "D": 128, "cap": 50.0, "B": 32},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_train", "norm", "norm_train", "attn", "attn_train"])
    c = {"kind": kind, "type": rng.choice(["f32", "bf16"])}
    if kind.startswith("embed"):
        V = _log(rng, 20, 100000)
        return {**c, "N": _log(rng, 5, 400000), "V": V, "F": _log(rng, 16, 320),
                "ids": rng.choice(["uniform", "zipf"]), "index": rng.choice(["int32", "int64"]),
                "scale": rng.choice([1.0, round(rng.uniform(0.5, 16.0), 2)]),
                "pad": rng.choice([-1, 0, rng.randrange(V)])}
    if kind.startswith("norm"):
        lo = _log(rng, 10, 4000)
        hi = _log(rng, lo, 4 * lo)
        groups = rng.choice([1, 4, 8, 16, 32])
        return {**c, "G": max(1, _log(rng, 8000, 200000) // hi), "lo": lo, "hi": hi,
                "F": groups * _log(rng, 4, 320 // groups if groups < 32 else 10),
                "groups": groups, "act": rng.choice(["none", "relu", "silu", "gelu"])}
    Hk = rng.choice([1, 2, 4, 8])
    H = Hk * rng.choice([1, 1, 2, 4])
    D = rng.choice([8, 16, 20, 32, 48, 64, 80, 128])
    B = rng.choice([0, rng.randrange(4, 40)])
    if kind == "attn" and rng.random() < 0.4:
        lo = _log(rng, 50, 20000)
        return {**c, "G": rng.randrange(1, 33), "lo": lo, "hi": 2 * lo, "queries": rng.choice([1, 3]),
                "H": H, "Hk": Hk, "D": D, "cap": rng.choice([0.0, 30.0]), "B": B}
    lo = _log(rng, 10, 1500)
    hi = _log(rng, lo, 2 * lo)
    G = max(1, min(2000, int(rng.uniform(0.1, 1.0) * 2.0e7 / (hi * hi * max(H, 8) / 8))))
    return {**c, "G": G, "lo": lo, "hi": hi, "queries": 0, "H": H, "Hk": Hk, "D": D,
            "cap": rng.choice([0.0, 20.0, 50.0]), "B": B}


def _sizes(case):
    """Nodes of each graph, by the case alone."""
    if case["kind"].startswith("embed"):
        return [case["N"]]
    rng = random.Random("%d %d %d" % (case["G"], case["lo"], case["hi"]))
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["G"])]


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, dtype=np.int64))])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = TYPES[case["type"]]

    def randn(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device=DEV) * scale + shift).to(dt)

    st = {"case": case}
    kind = case["kind"]
    if kind.startswith("embed"):
        N, V, F = case["N"], case["V"], case["F"]
        u = torch.rand(N, generator=gen, device=DEV, dtype=torch.float64)
        ids = u * V if case["ids"] == "uniform" else torch.exp(u * math.log(V + 1.0)) - 1.0
        it = torch.int32 if case["index"] == "int32" else torch.int64
        st["ids"] = ids.to(torch.int64).clamp_(0, V - 1).to(it)
        st["table"] = randn(V, F, scale=0.5)
        if kind == "embed_train":
            st["dout"] = randn(N, F)
        return st
    counts = _sizes(case)
    off = _offsets(counts)
    N, G = int(off[-1]), case["G"]
    st["counts"], st["nmax"] = counts, max(counts)
    st["offsets"] = torch.from_numpy(off.astype(np.int32)).to(DEV)
    if kind.startswith("norm"):
        F = case["F"]
        st["graph_index"] = torch.repeat_interleave(
            torch.arange(G, device=DEV), torch.tensor(counts, device=DEV))
        st["x"] = randn(N, F, scale=1.5, shift=0.7)
        st["gamma"] = randn(F, scale=0.3, shift=1.0)
        st["beta"] = randn(F, scale=0.3)
        if kind == "norm_train":
            st["dout"] = randn(N, F)
        return st
    H, Hk, D, B = case["H"], case["Hk"], case["D"], case["B"]
    st["scale"] = 1.0 / math.sqrt(D)
    if case["queries"]:  # a readout: a few queries per graph over its nodes
        qc = [case["queries"]] * G
        st["q"] = randn(sum(qc), H * D)
        kv = randn(N, 2 * Hk * D)
        st["k"], st["v"] = kv[:, :Hk * D], kv[:, Hk * D:]
    else:  # one projection of the nodes: q, k and v are columns of it
        qc = counts
        qkv = randn(N, (H + 2 * Hk) * D)
        st["q"], st["k"] = qkv[:, :H * D], qkv[:, H * D:(H + Hk) * D]
        st["v"] = qkv[:, (H + Hk) * D:]
    qoff = _offsets(qc)
    st["q_offsets"] = torch.from_numpy(qoff.astype(np.int32)).to(DEV)
    st["k_offsets"] = st["offsets"]
    st["qmax"], st["kmax"] = max(qc), max(counts)
    st["bias"] = st["dist"] = st["dist_offsets"] = None
    if B:
        pairs = _offsets([a * b for a, b in zip(qc, counts)])
        st["dist_offsets"] = torch.from_numpy(pairs).to(DEV)
        # hops 0 .. B-1, and now and then an unreachable node (B: masked)
        st["dist"] = torch.randint(0, 20 * B + 1, (int(pairs[-1]),), generator=gen, device=DEV,
                                   dtype=torch.int32).div_(20, rounding_mode="floor").to(torch.uint8)
        st["bias"] = randn(H, B, scale=0.7)
    if kind == "attn_train":
        st["dout"] = randn(int(qoff[-1]), H * D)
    return st


# ---- plain forms -----------------------------------------------------------------------


def _padded(off, nmax):
    """Node of (graph, place) in a batch padded to nmax places, and whether there is one."""
    off = off.long()
    at = off[:-1, None] + torch.arange(nmax, device=off.device)
    return torch.minimum(at, off[-1] - 1), at < off[1:, None]


def _act(z, name):
    """activation(z) and its derivative."""
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).to(z.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        c = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * c, c + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return z, torch.ones_like(z)


def _plain_embed(st):
    c = st["case"]
    ids = st["ids"].long()
    live = (ids != c["pad"])[:, None]
    out = torch.where(live, st["table"].float()[ids] * c["scale"], 0.0).to(st["table"].dtype)
    if c["kind"] == "embed":
        return {"out": out}
    d = torch.where(live, st["dout"].double(), 0.0)
    grad = torch.zeros(c["V"], c["F"], dtype=torch.float64, device=d.device).index_add_(0, ids, d)
    return {"out": out, "dtable": (grad * c["scale"]).to(st["table"].dtype)}


def _plain_norm(st):
    c = st["case"]
    F, K = c["F"], c["groups"]
    at, live = _padded(st["offsets"], st["nmax"])
    G, n = at.shape
    gi = st["graph_index"]
    x = st["x"].float()
    cnt = (live.sum(1) * (F // K)).double()[:, None]
    xp = torch.where(live[:, :, None], x[at], 0.0).view(G, n, K, F // K)
    mean = xp.double().sum((1, 3)) / cnt
    dev = torch.where(live[:, :, None, None], xp.double() - mean[:, None, :, None], 0.0)
    rstd = 1.0 / torch.sqrt((dev * dev).sum((1, 3)) / cnt + EPS)
    mean, rstd = mean.float(), rstd.float()
    xh = ((x.view(-1, K, F // K) - mean[gi][:, :, None]) * rstd[gi][:, :, None])
    z = xh.view(-1, F) * st["gamma"].float() + st["beta"].float()
    y, dz = _act(z, c["act"])
    res = {"out": y.to(st["x"].dtype), "mean": mean, "rstd": rstd}
    if c["kind"] == "norm":
        return res
    dz = dz * st["dout"].float()
    res["dgamma"] = (dz * xh.view(-1, F)).double().sum(0).to(st["x"].dtype)
    res["dbeta"] = dz.double().sum(0).to(st["x"].dtype)
    dh = (dz * st["gamma"].float()).view(-1, K, F // K)
    dhp = torch.where(live[:, :, None, None], dh[at], 0.0).double()
    xhp = torch.where(live[:, :, None, None], xh[at], 0.0).double()
    a = (dhp.sum((1, 3)) / cnt).float()
    b = ((dhp * xhp).sum((1, 3)) / cnt).float()
    dx = (dh - a[gi][:, :, None] - xh * b[gi][:, :, None]) * rstd[gi][:, :, None]
    res["dx"] = dx.view(-1, F).to(st["x"].dtype)
    return res


def _heads(x, at, live, heads):
    """[N, heads * D] as [G, heads, places, D] in 32 bits, zeros where there is no node."""
    p = torch.where(live[:, :, None], x.float()[at], 0.0)
    return p.view(*at.shape, heads, -1).permute(0, 2, 1, 3).contiguous()


def _plain_attn(st):
    c = st["case"]
    H, Hk, D, B, cap = c["H"], c["Hk"], c["D"], c["B"], c["cap"]
    dt = st["q"].dtype
    qa, ql = _padded(st["q_offsets"], st["qmax"])
    ka, kl = _padded(st["k_offsets"], st["kmax"])
    q = _heads(st["q"], qa, ql, H)
    k = _heads(st["k"], ka, kl, Hk).repeat_interleave(H // Hk, 1)
    v = _heads(st["v"], ka, kl, Hk).repeat_interleave(H // Hk, 1)
    s = (q @ k.transpose(2, 3).contiguous()) * st["scale"]
    tanh = None
    if cap:
        tanh = torch.tanh(s / cap)
        s = tanh * cap
    live = ql[:, :, None] & kl[:, None, :]
    if B:
        nk = (st["k_offsets"][1:] - st["k_offsets"][:-1]).long()
        iq, ik = (torch.arange(n, device=s.device) for n in (st["qmax"], st["kmax"]))
        pair = st["dist_offsets"][:-1, None, None] + iq[:, None] * nk[:, None, None] + ik
        bucket = st["dist"][torch.where(live, pair, 0)].long()
        live = live & (bucket < B)
        bucket = bucket.clamp(max=B - 1)
        s = s + st["bias"].float()[:, bucket].transpose(0, 1)
    s = torch.where(live[:, None], s, -math.inf)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    del s
    p = p / p.sum(3, keepdim=True).clamp(min=1e-30)
    out = p @ v
    rows = (torch.arange(qa.shape[0], device=qa.device)[:, None].expand_as(qa)[ql],
            torch.arange(qa.shape[1], device=qa.device).expand_as(qa)[ql])
    res = {"out": out.permute(0, 2, 1, 3)[rows].reshape(-1, H * D).to(dt)}
    if c["kind"] == "attn":
        return res
    do = _heads(st["dout"], qa, ql, H)
    dv = p.transpose(2, 3).contiguous() @ do
    ds = do @ v.transpose(2, 3).contiguous()
    ds = p * (ds - (p * ds).sum(3, keepdim=True))
    if B:
        hot = (bucket[..., None] == torch.arange(B, device=ds.device)) & live[..., None]
        by = ds.permute(0, 2, 1, 3).contiguous() @ hot.float()  # [G, queries, H, B]
        res["dbias"] = by.double().sum((0, 1)).to(dt)
        del hot
    if cap:
        ds = ds * (1.0 - tanh * tanh)
    ds = ds * st["scale"]
    dq = ds @ k
    dk = ds.transpose(2, 3).contiguous() @ q
    krows = (torch.arange(ka.shape[0], device=ka.device)[:, None].expand_as(ka)[kl],
             torch.arange(ka.shape[1], device=ka.device).expand_as(ka)[kl])

    def shared(x):  # the heads that share a key/value head add up
        x = x.view(x.shape[0], Hk, H // Hk, *x.shape[2:]).sum(2)
        return x.permute(0, 2, 1, 3)[krows].reshape(-1, Hk * D).to(dt)

    res["dq"] = dq.permute(0, 2, 1, 3)[rows].reshape(-1, H * D).to(dt)
    res["dk"], res["dv"] = shared(dk), shared(dv)
    return res


# ---- the framework's calls ----------------------------------------------------------------


def _own(st):
    import paper_2101_11552_amd as tfg
    c = st["case"]
    kind = c["kind"]
    if kind.startswith("embed"):
        pad = None if c["pad"] < 0 else c["pad"]
        res = {"out": tfg.tfg_embedding(st["table"], st["ids"], scale=c["scale"], padding_id=pad,
                                        validate=False)}
        if kind == "embed_train":
            res["dtable"] = tfg.tfg_embedding_backward(st["dout"], st["ids"], c["V"],
                                                       scale=c["scale"], padding_id=pad,
                                                       validate=False)
        return res
    if kind.startswith("norm"):
        out, mean, rstd = tfg.tfg_group_norm(st["x"], st["graph_index"], c["G"], c["groups"],
                                             st["gamma"], st["beta"], EPS, c["act"],
                                             validate=False)
        res = {"out": out, "mean": mean, "rstd": rstd}
        if kind == "norm_train":
            res["dx"], res["dgamma"], res["dbeta"] = tfg.tfg_group_norm_backward(
                st["dout"], st["x"], st["graph_index"], c["G"], c["groups"], mean, rstd,
                st["gamma"], st["beta"], c["act"], validate=False)
        return res
    args = dict(k_offsets=st["k_offsets"], kv_heads=c["Hk"], scale=st["scale"], cap=c["cap"],
                bias=st["bias"], distance=st["dist"], distance_offsets=st["dist_offsets"],
                validate=False)
    if kind == "attn":
        return {"out": tfg.tfg_graph_attention(st["q"], st["k"], st["v"], st["q_offsets"], c["H"],
                                               **args)}
    out, lse = tfg.tfg_graph_attention(st["q"], st["k"], st["v"], st["q_offsets"], c["H"],
                                       want_lse=True, **args)
    dq, dk, dv, dbias = tfg.tfg_graph_attention_backward(
        st["dout"], st["q"], st["k"], st["v"], out, lse, st["q_offsets"], c["H"], **args)
    res = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if c["B"]:
        res["dbias"] = dbias
    return res


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind.startswith("embed"):
        return _plain_embed(state)
    if kind.startswith("norm"):
        return _plain_norm(state)
    return _plain_attn(state)


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    sz = 4 if case["type"] == "f32" else 2
    kind = case["kind"]
    train = kind.endswith("_train")
    if kind.startswith("embed"):
        N, V, F = case["N"], case["V"], case["F"]
        idx = 4 if case["index"] == "int32" else 8
        b = N * idx + min(N, V) * F * sz + N * F * sz
        fl = N * F
        if train:
            b += N * F * sz + N * idx + V * F * sz
            fl += N * F
        return {"bytes": b, "flops": fl}
    counts = _sizes(case)
    N = sum(counts)
    if kind.startswith("norm"):
        F, K, G = case["F"], case["groups"], case["G"]
        b = 2 * N * F * sz + 8 * N + 8 * G * K + 2 * F * sz
        fl = 10 * N * F
        if train:
            b += 3 * N * F * sz + 8 * N + 8 * G * K + 4 * F * sz
            fl += 20 * N * F
        return {"bytes": b, "flops": fl}
    H, Hk, D = case["H"], case["Hk"], case["D"]
    qc = [case["queries"]] * case["G"] if case["queries"] else counts
    pairs = sum(a * b for a, b in zip(qc, counts))
    M = sum(qc)
    b = 2 * M * H * D * sz + 2 * N * Hk * D * sz + 8 * (case["G"] + 1)
    fl = 4 * pairs * H * D
    dist = pairs + H * case["B"] * sz + 8 * (case["G"] + 1) if case["B"] else 0
    b += dist
    if train:
        b += 4 * M * H * D * sz + 4 * N * Hk * D * sz + dist + H * case["B"] * sz
        fl += 10 * pairs * H * D
    return {"bytes": b, "flops": fl}


# ---- the definition in 64 bits ----------------------------------------------------------------


def _exact_embed(st):
    c = st["case"]
    ids = st["ids"].cpu().numpy().astype(np.int64)
    table = st["table"].double().cpu().numpy()
    keep = ids != c["pad"]
    out = table[ids] * c["scale"]
    out[~keep] = 0.0
    res = {"out": torch.from_numpy(out)}
    if c["kind"] == "embed_train":
        d = st["dout"].double().cpu().numpy()
        order = np.argsort(ids[keep], kind="stable")
        rows, first = np.unique(ids[keep][order], return_index=True)
        grad = np.zeros((c["V"], c["F"]))
        if len(rows):
            grad[rows] = np.add.reduceat(d[keep][order], first, axis=0) * c["scale"]
        res["dtable"] = torch.from_numpy(grad)
    return res


def _exact_norm(st):
    c = st["case"]
    F, K, train = c["F"], c["groups"], c["kind"] == "norm_train"
    gamma, beta = st["gamma"].double(), st["beta"].double()
    acc = {n: [] for n in ("out", "mean", "rstd", "dx")}
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(gamma)
    first = 0
    for n in st["counts"]:
        x = st["x"][first:first + n].double().reshape(n, K, F // K)
        mean = x.mean((0, 2))
        var = x.var((0, 2), unbiased=False)
        rstd = (var + EPS).rsqrt()
        xh = (x - mean[None, :, None]) * rstd[None, :, None]
        z = (xh.reshape(n, F) * gamma + beta)
        if c["act"] == "relu":
            y, slope = z.clamp(min=0.0), (z > 0).double()
        elif c["act"] == "silu":
            sg = torch.sigmoid(z)
            y, slope = z * sg, sg + z * sg * (1 - sg)
        elif c["act"] == "gelu":
            phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
            y, slope = z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            y, slope = z, torch.ones_like(z)
        acc["out"].append(y)
        acc["mean"].append(mean[None])
        acc["rstd"].append(rstd[None])
        if train:
            dz = slope * st["dout"][first:first + n].double()
            dgamma += (dz * xh.reshape(n, F)).sum(0)
            dbeta += dz.sum(0)
            dh = (dz * gamma).reshape(n, K, F // K)
            mid = dh.mean((0, 2))[None, :, None]
            cor = (dh * xh).mean((0, 2))[None, :, None]
            acc["dx"].append(((dh - mid - xh * cor) * rstd[None, :, None]).reshape(n, F))
        first += n
    res = {n: torch.cat(t) for n, t in acc.items() if t}
    if train:
        res["dgamma"], res["dbeta"] = dgamma, dbeta
    return res


def _exact_attn(st):
    c = st["case"]
    H, Hk, D, B, cap = c["H"], c["Hk"], c["D"], c["B"], c["cap"]
    train = c["kind"] == "attn_train"
    qo, ko = st["q_offsets"].tolist(), st["k_offsets"].tolist()
    po = st["dist_offsets"].tolist() if B else None
    new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=x.device)  # noqa: E731
    out = new(st["q"])
    if train:
        dq, dk, dv = new(st["q"]), new(st["k"]), new(st["v"])
    dbias = torch.zeros(H, max(B, 1), dtype=torch.float64, device=out.device)
    step = H if max(st["counts"]) <= 512 else 1  # heads at a time
    for g in range(c["G"]):
        qs, ks = slice(qo[g], qo[g + 1]), slice(ko[g], ko[g + 1])
        nq, nk = qo[g + 1] - qo[g], ko[g + 1] - ko[g]
        dist = st["dist"][po[g]:po[g + 1]].view(nq, nk).long() if B else None
        for h0 in range(0, H, step):
            hs = torch.arange(h0, h0 + step, device=out.device)
            kh = torch.div(hs, H // Hk, rounding_mode="floor")
            q = st["q"][qs].double().view(nq, H, D)[:, hs]
            k = st["k"][ks].double().view(nk, Hk, D)[:, kh]
            v = st["v"][ks].double().view(nk, Hk, D)[:, kh]
            s = torch.einsum("ihd,jhd->hij", q, k) * st["scale"]
            t = torch.tanh(s / cap) if cap else None
            if cap:
                s = cap * t
            if B:
                full = torch.cat([st["bias"].double(), torch.full((H, 1), -math.inf, device=s.device,
                                                                   dtype=torch.float64)], 1)
                s = s + full[hs][:, dist.clamp(max=B)]
            lse = torch.logsumexp(s, 2, keepdim=True)
            p = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse))
            o = torch.einsum("hij,jhd->ihd", p, v)
            out.view(-1, H, D)[qs, h0:h0 + step] = o
            if not train:
                continue
            do = st["dout"][qs].double().view(nq, H, D)[:, hs]
            dp = torch.einsum("ihd,jhd->hij", do, v)
            ds = p * (dp - (do * o).sum(2).t()[:, :, None])
            if B:
                flat = torch.nn.functional.one_hot(dist.clamp(max=B).view(-1), B + 1)[:, :B]
                dbias[hs] += ds.reshape(step, -1) @ flat.double() if nq * nk < 1 << 19 else torch.stack(
                    [(ds * (dist == b)).sum((1, 2)) for b in range(B)], 1)
                del flat
            if cap:
                ds = ds * (1 - t * t)
            ds = ds * st["scale"]
            dq.view(-1, H, D)[qs, h0:h0 + step] = torch.einsum("hij,jhd->ihd", ds, k)
            dk.view(-1, Hk, D)[ks].index_add_(1, kh, torch.einsum("hij,ihd->jhd", ds, q))
            dv.view(-1, Hk, D)[ks].index_add_(1, kh, torch.einsum("hij,ihd->jhd", p, do))
    res = {"out": out}
    if train:
        res.update(dq=dq, dk=dk, dv=dv)
        if B:
            res["dbias"] = dbias
    return res


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("embed"):
        return _exact_embed(st)
    if kind.startswith("norm"):
        return _exact_norm(st)
    return _exact_attn(st)
