"""Performance cases of the operators around a transformer's linear layers, on one party's replicated shares over Z_{2^64}:
embedding lookup and its gradient, norms of the heads with the position rotation, and the gradient norm with clipping.

Shares are uniform 64-bit words whatever the plaintext, held as int64 tensors whose bits are the ring elements; sums and
products of int64 tensors wrap mod 2^64, so every result is exact and has to be equal, bit for bit.  Token ids, positions,
angles and the clip factor are public.  Layer sets of the gradient norm are those of paper_2104_10949_amd/workloads.py,
written out here; the other sizes are generic.

With `own` false the operators are computed from elementary torch operations, with `own` true by the package's calls.
"""
import math

import numpy as np
import torch

own = False

FRAC_BITS = 16     # fractional bits of the fixed-point encodings
ANGLE_BITS = 14    # fractional bits of the public cosines and sines
FACTOR_BITS = 16   # fractional bits of the clip factor


def _embed(name, n, V, D, ids, idx64, scaled):
    return {"name": name, "kind": "embed", "n": n, "V": V, "D": D, "ids": ids, "idx64": idx64, "scaled": scaled}


def _embed_grad(name, n, V, D, ids, idx64, pad, batches):
    return {"name": name, "kind": "embed_grad", "n": n, "V": V, "D": D, "ids": ids, "idx64": idx64, "pad": pad, "batches": batches}


def _heads(name, kind, T, q, k, v, dim, rot, interleaved):
    return {"name": name, "kind": kind, "T": T, "q": q, "k": k, "v": v, "dim": dim, "rot": rot, "interleaved": interleaved}


def listed():
    return [
        # the next token of a generation: launch latency
        _embed("embed_1_of_32000x512", 1, 32000, 512, "token", True, False),
        # a batch of sequences, embeddings scaled by the root of their width
        _embed("embed_8192_of_32000x768", 8192, 32000, 768, "token", False, True),
        # rows of odd length (8-byte aligned only), gradients of two micro-batches summed in one buffer
        _embed_grad("embed_grad_777_of_1531x515", 777, 1531, 515, "token", True, 0.0, 2),
        # one micro-batch, a tenth of it padding: most of the time goes into rows without a token
        _embed_grad("embed_grad_4096_of_32000x768", 4096, 32000, 768, "token", True, 0.1, 1),
        # a large batch: the most frequent tokens occur thousands of times
        _embed_grad("embed_grad_65536_of_32000x1024", 65536, 32000, 1024, "token", False, 0.0, 1),
        # gradient clipping of the three fully connected layers 784-128-128-10: launch latency
        {"name": "clip_fc_784_128_128_10", "kind": "clip", "net": "fc"},
        # ... and of the VGG16-shaped network
        {"name": "clip_vgg16", "kind": "clip", "net": "vgg16"},
        # gradient norm of the ResNet-50-shaped network (monitored without clipping): 108 tensors, half of them short
        {"name": "norm_resnet50", "kind": "norm", "net": "resnet50"},
        # queries and keys of the next token: launch latency
        _heads("heads_1x12+4x64", "heads", 1, 12, 4, 4, 64, 64, False),
        # queries and keys of a long prompt, read in place from the packed output of their projection
        _heads("heads_4096x20+5x128", "heads", 4096, 20, 5, 5, 128, 128, False),
        # training: half of each head rotated, neighbouring elements paired, sizes that are multiples of little
        _heads("heads_grad_333x6+1x80", "heads_grad", 333, 6, 1, 0, 80, 40, True),
        # training on long sequences
        _heads("heads_grad_2048x20+5x128", "heads_grad", 2048, 20, 5, 5, 128, 128, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed", "embed_grad", "embed_grad", "embed_grad", "norm", "clip", "heads", "heads", "heads_grad"])
    if kind in ("embed", "embed_grad"):
        while True:
            ids = rng.choice(["token", "token", "position"])
            n, D = _log_int(rng, 1, 65536), _log_int(rng, 16, 2048)
            V = _log_int(rng, 100, 128000) if ids == "token" else _log_int(rng, 64, 8192)
            D = D if rng.random() < 0.25 else (D + 15) // 16 * 16
            if n * D <= 1 << 25 and V * D <= 1 << 25:
                break
        case = {"kind": kind, "n": n, "V": V, "D": D, "ids": ids, "idx64": rng.random() < 0.5}
        if kind == "embed":
            return {**case, "scaled": rng.random() < 0.5}
        return {**case, "pad": rng.choice([0.0, 0.0, 0.1, 0.5]), "batches": rng.choice([1, 1, 2])}
    if kind in ("norm", "clip"):
        return {"kind": kind, "net": "random", "tensors": _log_int(rng, 1, 200), "largest": _log_int(rng, 1000, 1 << 20), "sizes": rng.randrange(1 << 20)}
    while True:
        q, T = _log_int(rng, 1, 64), _log_int(rng, 1, 8192)
        k = rng.choice([q, max(1, q // 4), 1])
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        if T * (q + k) * dim <= 1 << 23:
            rot = rng.choice([dim, dim, dim // 2])
            case = _heads("", kind, T, q, k, rng.choice([0, k]), dim, rot, rng.random() < 0.3)
            del case["name"]
            return case


def _sizes(case):
    """Numbers of elements of the tensors whose gradients are taken: weights, and a bias each."""
    if case["net"] == "fc":
        layers = [(128, 784), (128, 128), (10, 128)]
    elif case["net"] == "vgg16":
        layers = [(64, 27), (64, 576), (128, 576), (128, 1152), (256, 1152), (256, 2304), (256, 2304), (512, 2304), (512, 4608), (512, 4608),
                  (512, 4608), (512, 4608), (512, 4608), (512, 8192), (512, 512), (200, 512)]
    elif case["net"] == "resnet50":
        layers, cin = [(64, 147)], 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                layers += [(width, cin), (width, 9 * width), (4 * width, width)] + ([(4 * width, cin)] if b == 0 else [])
                cin = 4 * width
        layers.append((1000, 2048))
    else:   # sizes over their logarithm, odd ones among them
        rng = np.random.default_rng(case["sizes"])
        return [int(v) for v in np.exp(rng.uniform(0.0, math.log(case["largest"]), case["tensors"])).round()]
    return [v for out, k in layers for v in (out * k, out)]


def _ring(shape, gen):
    return torch.randint(-2 ** 63, 2 ** 63 - 1, tuple(shape), dtype=torch.int64, device="cuda", generator=gen)


def _pair(shape, gen):
    return _ring(shape, gen), _ring(shape, gen)


def _ids(case, gen):
    n, V = case["n"], case["V"]
    if case["ids"] == "position":   # sequences one after the other
        ids = torch.arange(n, device="cuda") % V
    else:                           # the k-th most frequent token with a probability of about 1 / k
        ids = torch.rand(n, dtype=torch.float64, device="cuda", generator=gen).mul(math.log(V + 1)).exp().long().sub(1).clamp(0, V - 1)
    if case.get("pad"):
        ids[torch.rand(n, device="cuda", generator=gen) < case["pad"]] = -1
    return ids if case["idx64"] else ids.int()


def _open_norm(x, y):
    return (x * (x + 2 * y)).sum()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "embed":
        n, V, D = case["n"], case["V"], case["D"]
        s["table"], s["ids"] = _pair((V, D), gen), _ids(case, gen)
        s["alpha"] = round(math.sqrt(D) * 2 ** FRAC_BITS) if case["scaled"] else 1
        s["z"] = torch.empty((2, n, D), dtype=torch.int64, device="cuda")
    elif kind == "embed_grad":
        n, V, D = case["n"], case["V"], case["D"]
        s["g"] = [_pair((n, D), gen) for _ in range(case["batches"])]
        s["ids"] = [_ids(case, gen) for _ in range(case["batches"])]
        s["alpha"] = round(math.sqrt(D) * 2 ** FRAC_BITS)
        s["d"] = torch.empty((2, V, D), dtype=torch.int64, device="cuda")
    elif kind in ("norm", "clip"):
        # all gradients of a step, one after the other in a buffer for each component, as a training program keeps them
        sizes = _sizes(case)
        N = sum(sizes)
        g = (torch.randn(N, dtype=torch.float32, device="cuda", generator=gen) * (8.0 / math.sqrt(N)) * 2 ** FRAC_BITS).round().long()
        s0, s1 = _pair((N,), gen)
        s2 = g - s0 - s1
        s["flat"], s["out"] = (s0, s1), torch.empty((2, N), dtype=torch.int64, device="cuda")
        # what the other two parties send when the norm is opened
        s["z1"], s["z2"] = _open_norm(s1, s2).reshape(1), _open_norm(s2, s0).reshape(1)
        s["max_norm"] = int(torch.randint(1, 16, (1,), device="cuda", generator=gen)) * 2 ** FRAC_BITS
        if own:   # the lists of tensors, made once
            from paper_2104_10949_amd import binding as cg
            s["x"] = cg.ShareList(s0.split(sizes), s1.split(sizes))
            s["y"] = cg.ShareList(s["out"][0].split(sizes), s["out"][1].split(sizes))
    else:
        T, heads, dim, rot = case["T"], case["q"] + case["k"], case["dim"], case["rot"]
        packed = _pair((T, heads + case["v"], dim), gen)
        s["x"] = tuple(t[:, :heads] for t in packed)
        s["r"] = _pair((T, heads), gen)
        # public angles of the positions, sequences of 2048 after some that are already there
        P = 4096
        angle = torch.arange(P, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") / (rot // 2))
        s["cos"], s["sin"] = ((f(angle) * 2 ** ANGLE_BITS).round().long() for f in (torch.cos, torch.sin))
        s["pos"] = torch.arange(T, device="cuda") % 2048 + int(torch.randint(0, 2048, (1,), device="cuda", generator=gen))
        if kind == "heads_grad":
            s["g"] = _pair((T, heads, dim), gen)
    return s


def _three(x, y):
    """One party's local step of a product: x_i y_i + x_{i+1} y_i + x_i y_{i+1}."""
    return x[0] * y[0] + x[1] * y[0] + x[0] * y[1]


def _rotate(u, c, sn, rot, interleaved):
    first, second = (u[..., 0:rot:2], u[..., 1:rot:2]) if interleaved else (u[..., :rot // 2], u[..., rot // 2:rot])
    a, b = first * c - second * sn, first * sn + second * c
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, u[..., rot:] << ANGLE_BITS), -1)


def _plain_embed_grad(s, k):
    V = s["case"]["V"]
    ids = s["ids"][k].long()
    at = torch.where((ids >= 0) & (ids < V), ids, V)
    sums = [torch.zeros((V + 1, s["case"]["D"]), dtype=torch.int64, device="cuda").index_add_(0, at, t * s["alpha"]) for t in s["g"][k]]
    return [t[:V] for t in sums]


def _plain_factor(S, max_norm):
    root = S.double().sqrt().long()
    root = root - (root * root > S).long()
    root = root + ((root + 1) * (root + 1) <= S).long()
    return torch.where(root <= max_norm, torch.full_like(S, 1 << FACTOR_BITS), (max_norm << FACTOR_BITS) // root.clamp(min=1))


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        ids = s["ids"].long()
        there = (ids >= 0) & (ids < case["V"])
        row = torch.where(there, ids, 0)
        return [t[row] * (there.long() * s["alpha"])[:, None] for t in s["table"]]
    if kind == "embed_grad":
        d = _plain_embed_grad(s, 0)
        return d if case["batches"] == 1 else [a + b for a, b in zip(d, _plain_embed_grad(s, 1))]
    if kind in ("norm", "clip"):
        x, y = s["flat"]
        z = (x * (x + 2 * y)).sum().reshape(1)
        if kind == "norm":
            return [z]
        c = _plain_factor(z + s["z1"] + s["z2"], s["max_norm"])
        return [z, c, x * c, y * c]
    c, sn, rot = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None], case["rot"]
    r = tuple(t[..., None] for t in s["r"])
    if kind == "heads":
        x, y = s["x"]
        return [(x * (x + 2 * y)).sum(-1), _rotate(_three(s["x"], r), c, sn, rot, case["interleaved"])]
    v = tuple(_rotate(t, c, -sn, rot, case["interleaved"]) for t in s["g"])
    return [_three(v, r), _three(s["x"], v).sum(-1)]


def _calls(s):
    from paper_2104_10949_amd import binding as cg
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        return list(cg.cg_share_embedding(*s["table"], s["ids"], s["alpha"], za=s["z"][0], zb=s["z"][1]))
    if kind == "embed_grad":
        d = cg.cg_share_embedding_grad(*s["g"][0], s["ids"][0], case["V"], s["alpha"], da=s["d"][0], db=s["d"][1])
        if case["batches"] == 2:
            d = cg.cg_share_embedding_grad(*s["g"][1], s["ids"][1], case["V"], s["alpha"], da=s["d"][0], db=s["d"][1], accumulate=True)
        return list(d)
    if kind in ("norm", "clip"):
        z = cg.cg_share_sq_norm(s["x"])
        if kind == "norm":
            return [z]
        c = cg.cg_clip_factor(z, s["z1"], s["z2"], s["max_norm"], FACTOR_BITS)
        cg.cg_share_clip(s["x"], c, s["y"])
        return [z, c, s["out"][0], s["out"][1]]
    angles = {"cos": s["cos"], "sin": s["sin"], "pos": s["pos"], "frac_bits": ANGLE_BITS, "interleaved": case["interleaved"]}
    if kind == "heads":
        return [cg.cg_share_head_sq_sum(*s["x"]), cg.cg_share_head_norm_rotate(*s["x"], *s["r"], **angles)]
    return list(cg.cg_share_head_norm_rotate_grad(*s["g"], *s["x"], *s["r"], **angles))


def run(s):
    return _calls(s) if own else _plain(s)


def _distinct(case):
    """How many rows of the table a call touches, as expected from the ids' distribution."""
    n, V = case["n"] * (1 - case.get("pad", 0.0)), case["V"]
    if case["ids"] == "position":
        return min(n, V)
    k = np.arange(1, V + 1)
    p = np.log((k + 1) / k) / math.log(V + 1)
    return float((1 - np.exp(n * np.log1p(-p))).sum())


def work(case):
    """Bytes: every operand read once (of a table the rows that are asked for, of the gradients those of no padding), every
    result written once.  Operations: a product of 64-bit words and its addition count as two, a sum as one."""
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        n, V, D, idb = case["n"], case["V"], case["D"], 8 if case["idx64"] else 4
        if kind == "embed":
            return {"bytes": 16 * D * (_distinct(case) + n) + idb * n, "flops": 2 * n * D * (1 if case["scaled"] else 0)}
        n *= case["batches"]
        return {"bytes": 16 * D * (V + n * (1 - case["pad"])) + idb * n, "flops": 2 * D * (n + V)}
    if kind in ("norm", "clip"):
        N = sum(_sizes(case))
        # clipping needs the whole norm before the first element: the gradients are read twice
        return {"bytes": N * 16 * (1 if kind == "norm" else 3), "flops": N * (3 if kind == "norm" else 7)}
    T, heads = case["T"], case["q"] + case["k"]
    n = T * heads * case["dim"]
    angles = min(T, 2048) * case["rot"] * 8 + 8 * T
    if kind == "heads":   # the norm is opened up in between: the heads are read twice
        return {"bytes": n * (16 + 16 + 8) + T * heads * (16 + 8) + angles, "flops": n * (3 + 4 + 4)}
    return {"bytes": n * (32 + 8) + T * heads * (16 + 8) + angles, "flops": n * (8 + 4 + 4)}


def _host(t):
    return t.contiguous().cpu().numpy().view(np.uint64)


def _exact_rotate(u, c, sn, rot, interleaved):
    out = u << np.uint64(ANGLE_BITS)
    at = np.arange(rot // 2)
    first, second = (2 * at, 2 * at + 1) if interleaved else (at, at + rot // 2)
    out[..., first] = u[..., first] * c - u[..., second] * sn
    out[..., second] = u[..., first] * sn + u[..., second] * c
    return out


def exact(case, seed):
    """The definitions on the host, on numpy's unsigned 64-bit integers."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        alpha, V, D = np.uint64(s["alpha"]), case["V"], case["D"]
        if kind == "embed":
            ids = s["ids"].cpu().numpy()
            out = [np.zeros((case["n"], D), np.uint64) for _ in range(2)]
            there = np.nonzero((ids >= 0) & (ids < V))[0]
            for z, t in zip(out, s["table"]):
                z[there] = _host(t)[ids[there]] * alpha
        else:
            out = [np.zeros((V, D), np.uint64) for _ in range(2)]
            for ids, pair in zip(s["ids"], s["g"]):
                ids = ids.cpu().numpy()
                there = np.nonzero((ids >= 0) & (ids < V))[0]
                order = there[np.argsort(ids[there], kind="stable")]
                rows, first = np.unique(ids[order], return_index=True)
                for d, g in zip(out, pair):
                    d[rows] += np.add.reduceat(_host(g)[order], first, axis=0) * alpha if len(rows) else np.uint64(0)
        return [t.view(np.int64) for t in out]
    if kind in ("norm", "clip"):
        x, y = (_host(t) for t in s["flat"])
        z = (x * x + x * y + y * x).sum(dtype=np.uint64).reshape(1)
        if kind == "norm":
            return [z.view(np.int64)]
        S = (int(z[0]) + int(_host(s["z1"])[0]) + int(_host(s["z2"])[0])) % (1 << 64)
        root = math.isqrt(S)
        c = np.uint64(1 << FACTOR_BITS if root <= s["max_norm"] else (s["max_norm"] << FACTOR_BITS) // root)
        return [z.view(np.int64), np.array([c]).view(np.int64), (x * c).view(np.int64), (y * c).view(np.int64)]
    pos = s["pos"].cpu().numpy()
    c, sn = (_host(s[k])[pos][:, None] for k in ("cos", "sin"))
    x, r = [_host(t) for t in s["x"]], [_host(t)[..., None] for t in s["r"]]
    if kind == "heads":
        u = x[0] * r[0] + x[1] * r[0] + x[0] * r[1]
        sq = (x[0] * x[0] + x[1] * x[0] + x[0] * x[1]).sum(-1, dtype=np.uint64)
        return [sq.view(np.int64), _exact_rotate(u, c, sn, case["rot"], case["interleaved"]).view(np.int64)]
    v = [_exact_rotate(_host(t), c, np.uint64(0) - sn, case["rot"], case["interleaved"]) for t in s["g"]]
    dx = v[0] * r[0] + v[1] * r[0] + v[0] * r[1]
    dr = (x[0] * v[0] + x[1] * v[0] + x[0] * v[1]).sum(-1, dtype=np.uint64)
    return [dx.view(np.int64), dr.view(np.int64)]
