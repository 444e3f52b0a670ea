"""Timed cases of the operators around the layer: LayerNorm with its gradients, dropout, the grouping
of tokens by leaf, and the leaf experts' products with their gradients.

A case is a dict of plain values; "op" names the operator and the other keys its sizes and types:

  layer_norm  "direction" forward or backward; tokens, hidden; x, s, y: types of the branch, of the
              residual stream and of the normalised rows; "residual": the branch is added to a stream
              first; "p": dropout of the branch; "stats": whether mean and 1/std are wanted (training)
  dropout     tokens, hidden; x: type of input, residual and output; "residual"; "p"
  group_rows  tokens, trees, ids (leaves per tree), "depth": the leaf level they come from
  products    "op" grouped_matmul or grouped_weight_grad; entries, groups, "empty": groups without a
              row; k, n; x: type of all operands; "gather": rows are read through the grouping's
              order; "act"; "keep_z": the pre-activation is stored (training); "gradient": the data
              gradient (weights read transposed, times the activation's derivative)

`own` chooses between the plain forms below and the framework's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5


def _norm(direction, tokens, hidden, x, s, y, residual, p, stats=True):
    return {"op": "layer_norm", "direction": direction, "tokens": tokens, "hidden": hidden, "x": x, "s": s, "y": y,
            "residual": residual, "p": p, "stats": stats}


def _dropout(tokens, hidden, x, residual, p):
    return {"op": "dropout", "tokens": tokens, "hidden": hidden, "x": x, "residual": residual, "p": p}


def _group(tokens, trees, depth):
    return {"op": "group_rows", "tokens": tokens, "trees": trees, "depth": depth}


def _product(op, entries, groups, empty, k, n, x, gather=False, act="identity", keep_z=False, gradient=False):
    return {"op": op, "entries": entries, "groups": groups, "empty": empty, "k": k, "n": n, "x": x, "gather": gather,
            "act": act, "keep_z": keep_z, "gradient": gradient}


def listed():
    cases = {
        # one token before a layer of LLM width: a serving step, latency alone
        "norm_token_4096_bf16": _norm("forward", 1, 4096, "bf16", "bf16", "bf16", False, 0.0, stats=False),
        # between two blocks of a training step at the throughput batch: the layer's output through
        # dropout onto the stream, and the next block's normalised rows, in one pass
        "norm_residual_dropout_65536x768_bf16": _norm("forward", 65536, 768, "bf16", "bf16", "bf16", True, 0.1),
        # the same step's gradients at BERT-large's width, the residual stream in single precision
        "norm_backward_65536x1024_mixed": _norm("backward", 65536, 1024, "bf16", "f32", "bf16", True, 0.1),
        # a small ragged finetuning batch of an odd width
        "dropout_333x101_f32": _dropout(333, 101, "f32", False, 0.1),
        # the end of a block at the throughput batch
        "dropout_residual_65536x768_bf16": _dropout(65536, 768, "bf16", True, 0.1),
        # a batch of the paper's speed test over the 64 leaves of a depth-6 routing tree
        "group_16384_depth6": _group(16384, 1, 6),
        # the throughput batch through eight trees of 512 leaves: half a million entries, 4096 groups
        "group_65536x8_depth9": _group(65536, 8, 9),
        # decoding eight tokens over 64 leaf experts of LLM width: the weights of the leaves in use are the work
        "experts_decode_8_bf16": _product("grouped_matmul", 8, 64, 8, 4096, 1024, "bf16", gather=True, act="gelu"),
        # first product of 32 leaf experts in training: gathered rows, GELU, the pre-activation kept
        "experts_up_65536_bf16": _product("grouped_matmul", 65536, 32, 1, 1024, 4096, "bf16", gather=True, act="gelu",
                                          keep_z=True),
        # data gradient through the second product and the GELU, single precision, ragged sizes
        "experts_gradient_9001_f32": _product("grouped_matmul", 9001, 16, 2, 768, 1000, "f32", act="gelu", gradient=True),
        # weight gradients of the first product: few groups, long sums
        "experts_weight_grad_65536_bf16": _product("grouped_weight_grad", 65536, 32, 1, 1024, 4096, "bf16", gather=True),
        # weight gradients of many small single-precision experts of an odd width
        "experts_weight_grad_5003_f32": _product("grouped_weight_grad", 5003, 64, 5, 300, 203, "f32", gather=True),
    }
    return [dict(name=n, **c) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width of lo..hi: as often a multiple of 64 or of 8 as any number."""
    w = _log_int(rng, lo, hi)
    step = rng.choice((1, 8, 64, 64))
    return max(step, w // step * step)


def draw(rng):
    op = rng.choice(("layer_norm", "layer_norm", "dropout", "group_rows", "grouped_matmul", "grouped_matmul",
                     "grouped_weight_grad"))
    types = ("f32", "bf16")
    if op in ("layer_norm", "dropout"):
        hidden = _width(rng, 16, 8192)
        tokens = _log_int(rng, 1, min(65536, 65536 * 1024 // hidden))
        residual, p = rng.random() < 0.6, rng.choice((0.0, 0.1, rng.uniform(0.01, 0.9)))
        if op == "dropout":
            return _dropout(tokens, hidden, rng.choice(types), residual, p or 0.1)
        s = rng.choice(types)
        x, y = rng.choice(types) if residual or p else s, rng.choice(types)
        return _norm(rng.choice(("forward", "backward")), tokens, hidden, x, s, y, residual, p,
                     stats=rng.random() < 0.7)
    if op == "group_rows":
        trees = rng.choice((1, 1, 2, 4, 8))
        return _group(_log_int(rng, 1, 65536), trees, rng.randint(0, 12 - trees.bit_length()))
    x = rng.choice(("bf16", "bf16", "f32"))
    groups = _log_int(rng, 1, 256)
    k, n = _width(rng, 16, 4096), _width(rng, 16, 4096)
    while groups * k * n > 32 * 1024 * 4096:
        groups = max(1, groups // 2)
        k = k if groups > 1 else k // 2
    # at most the listed cases' products: 2 x 65536 x 1024 x 4096 operations in bf16, a tenth in single precision
    most = 65536 * 1024 * 4096 // (1 if x == "bf16" else 10)
    entries = _log_int(rng, 1, max(1, min(65536, most // (k * n))))
    empty = min(groups - 1, rng.choice((0, 0, groups // 8, groups // 2)))
    if op == "grouped_weight_grad":
        return _product(op, entries, groups, empty, k, n, x, gather=rng.random() < 0.5)
    act = rng.choice(("identity", "gelu", "gelu_tanh"))
    if rng.random() < 0.4:
        return _product(op, entries, groups, empty, k, n, x, gather=rng.random() < 0.3, act=act, gradient=True)
    return _product(op, entries, groups, empty, k, n, x, gather=rng.random() < 0.6, act=act, keep_z=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs


def _stream(gen, tokens, hidden, dtype):
    """Rows of a residual stream: a few channels are large and a mean is left, as in trained models."""
    v = torch.randn((tokens, hidden), generator=gen, device="cuda")
    scale = torch.exp(0.5 * torch.randn(hidden, generator=gen, device="cuda"))
    return (v * scale + 0.3).to(dtype)


def _gains(gen, hidden):
    return (1 + 0.2 * torch.randn(hidden, generator=gen, device="cuda"),
            0.1 * torch.randn(hidden, generator=gen, device="cuda"))


def _leaves(gen, entries, groups, empty):
    """A group for every entry: uneven shares, `empty` groups without any, each other one with at least
    one while there are entries."""
    used = torch.randperm(groups, generator=gen, device="cuda")[:groups - empty]
    share = torch.exp(0.5 * torch.randn(used.numel(), generator=gen, device="cuda"))
    g = used[torch.multinomial(share, entries, replacement=True, generator=gen)]
    first = min(entries, used.numel())
    g[:first] = used[:first]
    return g[torch.randperm(entries, generator=gen, device="cuda")]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    st = {"case": case, "seed": 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 63), "offset": (1 << 32) + 5 * seed + 1}
    op = case["op"]
    if op == "layer_norm":
        B, H, s = case["tokens"], case["hidden"], DT[case["s"]]
        st["gamma"], st["beta"] = _gains(gen, H)
        if case["direction"] == "forward":
            st["x"] = randn(B, H, dtype=DT[case["x"]]) if case["residual"] else _stream(gen, B, H, DT[case["x"]])
            st["residual"] = _stream(gen, B, H, s) if case["residual"] else None
        else:
            st["s"] = _stream(gen, B, H, s)
            wide = st["s"].float()
            st["mean"] = wide.mean(1)
            st["rstd"] = 1 / torch.sqrt((wide - st["mean"][:, None]).square().mean(1) + EPS)
            st["dy"] = randn(B, H, dtype=DT[case["y"]])
            st["ds_in"] = randn(B, H, dtype=s) if case["residual"] else None
    elif op == "dropout":
        B, H, t = case["tokens"], case["hidden"], DT[case["x"]]
        st["x"] = randn(B, H, dtype=t)
        st["residual"] = _stream(gen, B, H, t) if case["residual"] else None
    elif op == "group_rows":
        leaves = 1 << case["depth"]
        pick = _leaves(gen, case["tokens"] * case["trees"], leaves, leaves // 16)
        st["ids"] = (pick + (leaves - 1)).to(torch.int32).view(case["tokens"], case["trees"])
    else:
        E, G, K, N, t = case["entries"], case["groups"], case["k"], case["n"], DT[case["x"]]
        ids = _leaves(gen, E, G, case["empty"])
        order = torch.sort(ids, stable=True).indices
        sizes = torch.bincount(ids, minlength=G)
        st["offsets"] = torch.cat((sizes.new_zeros(1), sizes.cumsum(0))).to(torch.int32)
        st["order"] = order.to(torch.int32)
        st["used"], st["longest"] = sizes.nonzero().flatten(), int(sizes.max())
        st["x"] = randn(E, K, dtype=t)
        if op == "grouped_weight_grad":
            st["dy"] = randn(E, N, dtype=t)
        elif case["gradient"]:
            st["w"] = randn(G, K, N, dtype=t, scale=K ** -0.5)
            st["z"] = randn(E, N, dtype=t)
        else:
            st["w"] = randn(G, N, K, dtype=t, scale=K ** -0.5)
    return st


# -------------------------------------------------------------------------------------- plain forms


def _philox(c0, c1, seed, offset):
    """Philox4x32-10 (Salmon et al., Parallel random numbers: as easy as 1, 2, 3): the four words for
    counter (c0, c1, offset) and key `seed`, in int64 tensors."""
    low = 0xFFFFFFFF
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        h0 = ((c0 >> 16) * 0xD2511F53 + ((c0 & 0xFFFF) * 0xD2511F53 >> 16)) >> 16
        h1 = ((c2 >> 16) * 0xCD9E8D57 + ((c2 & 0xFFFF) * 0xCD9E8D57 >> 16)) >> 16
        l0, l1 = c0 * 0xD2511F53 & low, c2 * 0xCD9E8D57 & low
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), -1)


def _drop(x, p, seed, offset):
    """x / (1 - p) where the generator keeps the element, 0 elsewhere."""
    if p == 0:
        return x
    B, H = x.shape
    blocks = torch.arange((H + 3) // 4, device=x.device).expand(B, -1)
    rows = torch.arange(B, device=x.device)[:, None].expand_as(blocks)
    words = _philox(blocks, rows, seed, offset).reshape(B, -1)[:, :H]
    return torch.where(words >= int(p * 2.0 ** 32), x * (1 / (1 - p)), torch.zeros_like(x))


_ROOT_HALF = math.sqrt(0.5)
_ROOT_2_PI = math.sqrt(2 / math.pi)


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * _ROOT_HALF)
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * _ROOT_2_PI * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "gelu":
        return 0.5 * torch.erfc(-z * _ROOT_HALF) + z * torch.exp(-0.5 * z * z) * (0.5 * _ROOT_2_PI)
    if act == "gelu_tanh":
        u = _ROOT_2_PI * (z + 0.044715 * z * z * z)
        up, down = 1 / (1 + torch.exp(-2 * u)), 1 / (1 + torch.exp(2 * u))
        return up + 2 * z * up * down * _ROOT_2_PI * (1 + 0.134145 * z * z)
    return torch.ones_like(z)


def _places(st):
    """Where entry i of the grouped order stands in a batch [used groups, longest group]."""
    E = st["order"].numel()
    at = torch.arange(E, device="cuda")
    group = torch.searchsorted(st["offsets"][1:].long(), at, right=True)
    return torch.searchsorted(st["used"], group), at - st["offsets"].long()[group]


def _batch(st, rows, places):
    out = rows.new_zeros((st["used"].numel(), st["longest"], rows.shape[1]))
    out[places] = rows
    return out


def _plain(st):
    c = st["case"]
    op = c["op"]
    if op == "layer_norm" and c["direction"] == "forward":
        s = _drop(st["x"].float(), c["p"], st["seed"], st["offset"])
        if c["residual"]:
            s = s + st["residual"].float()
        mean = s.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((s - mean).square().mean(1, keepdim=True) + EPS)
        out = [((s - mean) * rstd * st["gamma"] + st["beta"]).to(DT[c["y"]])]
        if c["residual"] or c["p"]:
            out.append(s.to(DT[c["s"]]))
        return out + [mean[:, 0], rstd[:, 0]] if c["stats"] else out
    if op == "layer_norm":
        dy, rstd = st["dy"].float(), st["rstd"][:, None]
        xh = (st["s"].float() - st["mean"][:, None]) * rstd
        g = dy * st["gamma"]
        ds = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if c["residual"]:
            ds = ds + st["ds_in"].float()
        out = [ds.to(DT[c["s"]]), (dy * xh).sum(0), dy.sum(0)]
        return out + [_drop(ds, c["p"], st["seed"], st["offset"]).to(DT[c["x"]])] if c["p"] else out
    if op == "dropout":
        y = _drop(st["x"].float(), c["p"], st["seed"], st["offset"])
        return [(y + st["residual"].float() if c["residual"] else y).to(DT[c["x"]])]
    if op == "group_rows":
        leaves = 1 << c["depth"]
        tree = torch.arange(c["trees"], device="cuda", dtype=torch.int32)
        key = (st["ids"] - (leaves - 1) + tree * leaves).flatten()
        ordered, order = torch.sort(key, stable=True)
        bounds = torch.arange(c["trees"] * leaves + 1, device="cuda", dtype=torch.int32)
        return [order.to(torch.int32), torch.searchsorted(ordered, bounds).to(torch.int32)]
    x = st["x"].float()
    x = x[st["order"].long()] if c["gather"] else x
    places = _places(st)
    x = _batch(st, x, places)
    if op == "grouped_weight_grad":
        dy = _batch(st, st["dy"].float(), places)
        dw = torch.zeros((c["groups"], c["n"], c["k"]), device="cuda")
        dw[st["used"]] = torch.matmul(dy.transpose(1, 2).contiguous(), x)
        return [dw]
    w = st["w"][st["used"]].float()
    z = torch.matmul(x, w if c["gradient"] else w.transpose(1, 2))[places]
    if c["gradient"]:
        return [(z * _act_grad(st["z"].float(), c["act"])).to(DT[c["x"]])]
    y = _act(z, c["act"]).to(DT[c["x"]])
    return [y, z.to(DT[c["x"]])] if c["keep_z"] else [y]


# ------------------------------------------------------------------------------ the framework's calls


def _framework(st):
    import paper_2311_10770_amd as fff

    c = st["case"]
    op = c["op"]
    drop = {"p": c["p"], "seed": st["seed"], "offset": st["offset"]} if c.get("p") else {}
    if op == "layer_norm" and c["direction"] == "forward":
        y, s, mean, rstd = fff.layer_norm(st["x"], st["gamma"], st["beta"], eps=EPS, residual=st["residual"],
                                          y_dtype=DT[c["y"]], s_dtype=DT[c["s"]], stats=c["stats"], **drop)
        out = [y, s] if c["residual"] or c["p"] else [y]
        return out + [mean, rstd] if c["stats"] else out
    if op == "layer_norm":
        ds, dx, dgamma, dbeta = fff.layer_norm_backward(st["dy"], st["s"], st["mean"], st["rstd"], st["gamma"],
                                                        ds_in=st["ds_in"], dx_dtype=DT[c["x"]], **drop)
        return [ds, dgamma, dbeta, dx] if c["p"] else [ds, dgamma, dbeta]
    if op == "dropout":
        return [fff.dropout(st["x"], residual=st["residual"], **drop)]
    if op == "group_rows":
        leaves = 1 << c["depth"]
        return list(fff.group_rows(st["ids"], leaves, first=leaves - 1, n_trees=c["trees"]))
    index = st["order"] if c["gather"] else None
    if op == "grouped_weight_grad":
        return [fff.grouped_weight_grad(st["dy"], st["x"], st["offsets"], x_index=index)]
    if c["gradient"]:
        return [fff.grouped_matmul(st["x"], st["w"], st["offsets"], x_index=index, transpose_w=True, act=c["act"],
                                   z_in=st["z"])]
    got = fff.grouped_matmul(st["x"], st["w"], st["offsets"], x_index=index, act=c["act"], keep_z=c["keep_z"])
    return list(got) if c["keep_z"] else [got]


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------ the bill


def work(case):
    op = case["op"]
    if op in ("layer_norm", "dropout"):
        B, H = case["tokens"], case["hidden"]
        x = BYTES[case["x"]]
        random = 30 if case["p"] else 0  # operations of the generator an element
        if op == "dropout":
            return {"bytes": B * H * x * (3 if case["residual"] else 2), "flops": B * H * (2 + random)}
        s, y = BYTES[case["s"]], BYTES[case["y"]]
        if case["direction"] == "forward":
            a = x + y + (s if case["residual"] else 0) + (s if case["residual"] or case["p"] else 0)
            return {"bytes": B * H * a + 8 * H + (8 * B if case["stats"] else 0), "flops": B * H * (8 + random)}
        a = y + 2 * s + (s if case["residual"] else 0) + (x if case["p"] else 0)
        return {"bytes": B * H * a + 8 * B + 12 * H, "flops": B * H * (16 + random)}
    if op == "group_rows":
        e = case["tokens"] * case["trees"]
        return {"bytes": 8 * e + 4 * (case["trees"] * (1 << case["depth"]) + 1), "flops": 2 * e}
    E, G, K, N, b = case["entries"], case["groups"], case["k"], case["n"], BYTES[case["x"]]
    used = min(E, G - case["empty"])
    lists = 4 * (G + 1) + (4 * E if case["gather"] else 0)
    if op == "grouped_weight_grad":
        return {"bytes": b * E * (K + N) + 4 * G * N * K + lists, "flops": 2 * E * N * K}
    rows = E * (K + N * (2 if case["keep_z"] or case["gradient"] else 1))
    return {"bytes": b * (rows + used * N * K) + lists, "flops": 2 * E * N * K}


# --------------------------------------------------------------------------- the definitions in 64 bits


def _kept(B, H, p, seed, offset):
    """Which elements dropout keeps: the generator in numpy's unsigned 64-bit products."""
    u = np.uint64
    low, s32 = u(0xFFFFFFFF), u(32)
    cols = (H + 3) // 4
    a = np.tile(np.arange(cols, dtype=u), B)
    b = np.repeat(np.arange(B, dtype=u), cols)
    c, d = np.full(B * cols, offset & 0xFFFFFFFF, u), np.full(B * cols, offset >> 32, u)
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        pa, pc = a * u(0xD2511F53), c * u(0xCD9E8D57)
        a, b, c, d = (pc >> s32) ^ b ^ u(key[0]), pc & low, (pa >> s32) ^ d ^ u(key[1]), pa & low
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.stack((a, b, c, d), 1).reshape(B, 4 * cols)[:, :H]
    return torch.from_numpy(bits >= u(math.floor(p * 4294967296.0))).cuda()


def exact(case, seed):
    st = prepare(case, seed)
    f8 = torch.float64
    op = case["op"]
    if op == "group_rows":
        leaves = 1 << case["depth"]
        key = st["ids"].cpu().numpy().astype(np.int64) - (leaves - 1) + leaves * np.arange(case["trees"])
        key = key.ravel()
        counts = np.bincount(key, minlength=case["trees"] * leaves)
        return [np.argsort(key, kind="stable").astype(np.int32),
                np.concatenate(([0], np.cumsum(counts))).astype(np.int32)]
    if op in ("layer_norm", "dropout"):
        B, H, p = case["tokens"], case["hidden"], case["p"]
        kept = _kept(B, H, p, st["seed"], st["offset"]) if p else None

        def dropped(v):
            return v if kept is None else (v / (1.0 - p)).masked_fill(~kept, 0.0)

        if op == "dropout":
            y = dropped(st["x"].to(f8))
            return [y + st["residual"].to(f8)] if case["residual"] else [y]
        if case["direction"] == "forward":
            s = dropped(st["x"].to(f8))
            s = s + st["residual"].to(f8) if case["residual"] else s
            var, mean = torch.var_mean(s, 1, correction=0)
            rstd = (var + EPS) ** -0.5
            y = torch.addcmul(st["beta"].to(f8), (s - mean[:, None]) * rstd[:, None], st["gamma"].to(f8))
            out = [y, s] if case["residual"] or p else [y]
            return out + [mean, rstd] if case["stats"] else out
        # the gradient as products with the projection that LayerNorm's derivative is
        rstd, dy = st["rstd"].to(f8), st["dy"].to(f8)
        hat = (st["s"].to(f8) - st["mean"].to(f8)[:, None]) * rstd[:, None]
        g = dy * st["gamma"].to(f8)
        along = torch.linalg.vecdot(g, hat) / H
        ds = (g - g.sum(1, keepdim=True) / H - hat * along[:, None]) * rstd[:, None]
        ds = ds + st["ds_in"].to(f8) if case["residual"] else ds
        out = [ds, torch.linalg.vecdot(dy, hat, dim=0), dy.sum(0)]
        return out + [dropped(ds)] if p else out
    bounds = st["offsets"].tolist()
    src = st["order"].long() if case["gather"] else torch.arange(case["entries"], device="cuda")
    groups = [(g, slice(a, b)) for g, (a, b) in enumerate(zip(bounds, bounds[1:])) if b > a]
    if op == "grouped_weight_grad":
        dw = torch.zeros((case["groups"], case["n"], case["k"]), dtype=f8, device="cuda")
        for g, r in groups:
            dw[g] = st["dy"][r].to(f8).T @ st["x"][src[r]].to(f8)
        return [dw]
    z = torch.empty((case["entries"], case["n"]), dtype=f8, device="cuda")
    for g, r in groups:
        w = st["w"][g].to(f8)
        z[r] = st["x"][src[r]].to(f8) @ (w if case["gradient"] else w.T)
    v = (st["z"].to(f8) if case["gradient"] else z).requires_grad_(case["gradient"])
    if case["act"] == "gelu":
        a = v * torch.special.ndtr(v)
    elif case["act"] == "gelu_tanh":
        a = 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    else:
        a = v * 1
    if case["gradient"]:
        return [z * torch.autograd.grad(a.sum(), v)[0]]
    return [a, z] if case["keep_z"] else [a]
