"""Optimizer operators on whole weight matrices, as cases that can be timed: in their plain form and as the framework computes them.

``ortho``   orthogonalise a set of matrices: O = p^5(X / ||X||_F) with p(X) = a X + (b X X^T + c (X X^T)^2) X (Newton-Schulz)
``muon``    the optimizer step around it: m <- mu m + g; u = g + mu m; x <- x - lr (s O(u) + wd x), s = 0.2 sqrt(max(rows, cols))
``decode``  the receiving side of compressed momenta: R = IDCT(sum of the workers' records); matrices x <- x - lr (s O(R) + wd x),
            vectors x <- x - lr (sign(R) + wd x)
``adamw``   the step of the tensors that are not orthogonalised: embeddings, heads, norm vectors

Tensor sets, chunk sizes, k, worker counts and value distributions are those of the benchmark configurations and tests of this
repository.  A set's tensors are views of one flat buffer per kind (gradients, momenta, parameters), as in a training program that
keeps them in arenas; what is returned are these buffers.
"""
from __future__ import annotations

import math

import torch

own = False

MU, LR, WD = 0.95, 1e-3, 0.1
A, B, C, STEPS, EPS = 3.4445, -4.7750, 2.0315, 5, 1e-7
BETA1, BETA2, ADAM_EPS = 0.9, 0.95, 1e-8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(op, tensors, **kw):
    c = {"op": op, "tensors": tensors, "grad": "bf16", "values": "normal"}
    if op == "decode":
        c.update(chunk=64, topk=32, workers=1)
    c.update(kw)
    return c


def listed():
    return [
        # One small weight (the "tiny" configuration's): latency, nothing else.
        _case("ortho", "matrix", name="ortho_tiny", rows=256, cols=512, grad="f32"),
        # Convolution weights as matrices, a 7 x 7 stem and a table with an odd number of rows: ragged, tall and wide.
        _case("ortho", "conv", name="ortho_conv_ragged", layers=4, out_ch=512, in_ch=512, kernel=3, stem=7, table_rows=7511,
              table_cols=512),
        # The large single matrix with row-wise scaled values (the single-matrix configuration).
        _case("ortho", "matrix", name="ortho_8192", rows=8192, cols=8192, grad="f32", values="rows"),
        # A scaled-down decoder, as in quick runs: fourteen small matrices in one step.
        _case("muon", "decoder", name="muon_small_decoder", d_model=256, layers=2, d_ff=1024, grad="f32"),
        # The 300M-class decoder's layers; gradients of a few strong directions over noise.
        _case("muon", "decoder", name="muon_300m", d_model=1024, layers=24, d_ff=4096, values="spiked"),
        # The 1B-class decoder's layers: the largest step.
        _case("muon", "decoder", name="muon_1b", d_model=2048, layers=16, d_ff=8192),
        # The "tiny" configuration received from two workers: one matrix, one bias.
        _case("decode", "matrix", name="decode_tiny", rows=256, cols=512, bias=512, chunk=8, topk=4, workers=2),
        # One decoder layer of the 1B class from eight workers, two norm vectors with it.
        _case("decode", "decoder", name="decode_layer_1b", d_model=2048, layers=1, d_ff=8192, norms=2, workers=8),
        # The stress matrix from 64 workers.
        _case("decode", "matrix", name="decode_fan_in_64", rows=4096, cols=4096, bias=0, workers=64),
        # The norm vectors of the scaled-down decoder: latency.
        _case("adamw", "vectors", name="adamw_vectors", n=256, count=5, rows=0, tables=0, grad="f32"),
        # Tied embedding and norm vectors of the 300M class.
        _case("adamw", "vectors", name="adamw_300m", n=1024, count=48, rows=50304, tables=1),
        # Embedding, untied head and norm vectors of the 1B class.
        _case("adamw", "vectors", name="adamw_1b", n=2048, count=32, rows=50304, tables=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Matrices from one row to 4096, square, wide and tall, of any size; decoder layers of odd and even widths from 64 to 1024; records
    in every chunk size from one to 64 workers; vectors from one element and tables of up to 50304 rows."""
    op = rng.choice(["ortho"] * 3 + ["muon"] * 3 + ["decode"] * 2 + ["adamw"] * 2)
    grad = rng.choice(["bf16", "bf16", "f32"])
    values = rng.choice(["normal", "rows", "heavy", "spiked"])
    if op == "ortho":
        if rng.random() < 0.25:
            return _case(op, "conv", layers=rng.randint(1, 4), out_ch=_log_int(rng, 16, 512), in_ch=_log_int(rng, 16, 512),
                         kernel=rng.choice([1, 3, 5]), stem=rng.choice([0, 7]), table_rows=_log_int(rng, 16, 8192),
                         table_cols=_log_int(rng, 16, 512), grad=grad, values=values)
        return _case(op, "matrix", rows=_log_int(rng, 1, 4096), cols=_log_int(rng, 1, 4096), copies=rng.choice([1, 1, 2, 5]),
                     grad=grad, values=values)
    if op == "muon":
        d = _log_int(rng, 64, 1024)
        return _case(op, "decoder", d_model=d, layers=_log_int(rng, 1, 12), d_ff=rng.choice([4 * d, 4 * d, 2 * d + 7]), grad=grad,
                     values=values)
    if op == "decode":
        s = rng.choice([64, 64, 64, 32, 128, 16])
        side = 4096 if s >= 32 else 1024
        rows, cols = (max(1, round(_log_int(rng, 2 * s, side) / s)) * s for _ in range(2))
        return _case(op, "matrix", rows=rows, cols=cols, bias=rng.choice([0, cols]), chunk=s,
                     topk=min(_log_int(rng, 4, 128), s * s), workers=_log_int(rng, 1, 64))
    return _case(op, "vectors", n=_log_int(rng, 1, 4096), count=rng.randint(1, 60), rows=rng.choice([0, _log_int(rng, 1, 50304)]),
                 tables=rng.choice([1, 2]), grad=grad, values=rng.choice(["normal", "heavy"]))


def _shapes(case):
    t = case["tensors"]
    if t == "matrix":
        return [(case["rows"], case["cols"])] * case.get("copies", 1) + ([(case["bias"],)] if case.get("bias") else [])
    if t == "conv":
        s = [(case["out_ch"], case["in_ch"] * case["kernel"] ** 2)] * case["layers"]
        s += [(case["out_ch"], 3 * case["stem"] ** 2)] if case["stem"] else []
        return s + [(case["table_rows"], case["table_cols"])]
    if t == "decoder":
        d, f = case["d_model"], case["d_ff"]
        return ([(d, d)] * 4 + [(d, f)] * 2 + [(f, d)] + [(d,)] * case.get("norms", 0)) * case["layers"]
    tables = [(case["rows"], case["n"])] * case["tables"] if case["rows"] else []
    return tables + [(case["n"],)] * case["count"]


def work(case):
    shapes = _shapes(case)
    n = sum(math.prod(s) for s in shapes)
    g = 4 if case["grad"] == "f32" else 2
    if case["op"] == "adamw":  # gradient read; two moments and the parameter read and written
        return {"bytes": n * (g + 24), "flops": 15 * n}
    # X X^T and (X X^T)^2 are symmetric: half their products
    flops = sum(STEPS * (min(s) ** 2 * max(s) * 3 + min(s) ** 3) for s in shapes if len(s) == 2)
    if case["op"] == "ortho":
        return {"bytes": n * (g + 2), "flops": flops}
    if case["op"] == "muon":
        return {"bytes": n * (g + 16), "flops": flops}
    records = sum(math.prod(s) // case["chunk"] ** len(s) * min(case["topk"], case["chunk"] ** len(s)) for s in shapes)
    flops += sum(2 * math.prod(s) * case["chunk"] * len(s) for s in shapes)
    return {"bytes": n * 8 + records * 8 * case["workers"], "flops": flops}


# --- inputs ------------------------------------------------------------------------------------------------------------------


def _arena(shapes, dtype):
    """A flat buffer of zeros and one view of it for each tensor, each at a multiple of 16 elements."""
    at, places = 0, []
    for s in shapes:
        places.append(at)
        at += -(-math.prod(s) // 16) * 16
    flat = torch.zeros(at, dtype=dtype, device="cuda")
    return flat, [flat[p:p + math.prod(s)].view(s) for p, s in zip(places, shapes)]


def _values(shape, kind, gen):
    x = torch.randn(shape, generator=gen, device="cuda")
    if kind == "rows":  # rows of very different sizes
        x *= torch.exp(torch.randn((shape[0],) + (1,) * (len(shape) - 1), generator=gen, device="cuda"))
    elif kind == "heavy":  # Student-t with three degrees of freedom
        chi = sum(torch.randn(shape, generator=gen, device="cuda").square_() for _ in range(3))
        x *= (chi / 3).rsqrt_().clamp_(max=1e3)
    elif kind == "spiked" and len(shape) == 2:  # sixteen strong directions over noise
        u = torch.randn((shape[0], 16), generator=gen, device="cuda")
        x = x * 0.3 + 0.75 * u @ torch.randn((16, shape[1]), generator=gen, device="cuda")
    return x


def _payload(case, shapes, gen):
    """One worker's records (index and value side by side, as bytes): the largest DCT coefficients of every chunk, by index."""
    parts = []
    for s in shapes:
        m = case["chunk"] ** len(s)
        k, n_chunks = min(case["topk"], m), math.prod(s) // m
        q = torch.randn((n_chunks, m), generator=gen, device="cuda") * 1e-3
        idx = q.abs().topk(k, dim=1).indices.sort(dim=1).values
        val = torch.gather(q, 1, idx)
        parts.append(torch.stack([idx.to(torch.int32), val.view(torch.int32)], dim=2).flatten())
    return torch.cat(parts).view(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    shapes, op = _shapes(case), case["op"]
    scales = (10 ** (2 * torch.rand(len(shapes), generator=gen, device="cuda") - 1) * 1e-3).tolist()
    s = {"case": case, "shapes": shapes}
    if op != "decode":
        s["g"], s["gs"] = _arena(shapes, TYPES[case["grad"]])
        for t, f in zip(s["gs"], scales):
            t.copy_(_values(tuple(t.shape), case["values"], gen) * f)
    else:
        s["payloads"] = [_payload(case, shapes, gen) for _ in range(case["workers"])]
    if op in ("muon", "adamw"):
        s["m"], s["ms"] = _arena(shapes, torch.float32)
        for t, f in zip(s["ms"], scales):
            t.copy_(_values(tuple(t.shape), case["values"], gen) * (3 * f if op == "muon" else 0.3 * f))
    if op == "adamw":
        s["v"], s["vs"] = _arena(shapes, torch.float32)
        for t, f in zip(s["vs"], scales):
            t.copy_((0.5 + torch.rand(tuple(t.shape), generator=gen, device="cuda")) * f * f)
        s["step"] = torch.tensor([100], dtype=torch.int64, device="cuda")
    if op == "ortho":
        s["out"], s["outs"] = _arena(shapes, torch.bfloat16)
    else:
        s["x"], s["xs"] = _arena(shapes, torch.float32)
        for t in s["xs"]:
            t.copy_(torch.randn(tuple(t.shape), generator=gen, device="cuda") * 0.02)
    if own:
        import paper_2411_19870_b200 as demo

        dtype = demo.DEMO_F32 if case["grad"] == "f32" else demo.DEMO_BF16
        matrices = [x for x in shapes if len(x) == 2]
        if op == "adamw":
            s["adamw"] = demo.AdamwTransform(shapes, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, lr=LR, weight_decay=WD, grad_dtype=dtype)
        else:
            s["muon"] = demo.MuonTransform(matrices, momentum=MU, nesterov=True, steps=STEPS, coefficients=(A, B, C), eps=EPS, lr=LR,
                                           weight_decay=WD, scale=demo.DEMO_SCALE_RMS, grad_dtype=dtype)
        if op == "decode":
            s["demo"] = demo.DemoTransform(shapes, chunk=case["chunk"], topk=case["topk"], beta=0.999, lr=LR, weight_decay=WD,
                                           num_workers=case["workers"])
    return s


# --- the plain forms ---------------------------------------------------------------------------------------------------------


def _alike(tensors):
    """The tensors' places by shape: matrices of one shape are orthogonalised as one batch."""
    return {s: [i for i, t in enumerate(tensors) if t.shape == s] for s in dict.fromkeys(t.shape for t in tensors)}


def _orthogonal(u):
    """u: matrices of one shape, [count, rows, cols], fp32."""
    x = u / (u.square().sum(dim=(1, 2), dtype=torch.float64).sqrt() + EPS).float()[:, None, None]
    tall = x.shape[1] > x.shape[2]
    x = x.mT.contiguous() if tall else x
    for _ in range(STEPS):
        a = x @ x.mT
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.mT if tall else x


def _update(x, o):
    """x <- x - lr (s o + wd x)"""
    x.copy_(x - LR * (0.2 * math.sqrt(max(x.shape)) * o + WD * x))


def _plain_ortho(s):
    for at in _alike(s["gs"]).values():
        for i, o in zip(at, _orthogonal(torch.stack([s["gs"][i] for i in at]).float()).bfloat16()):
            s["outs"][i].copy_(o)
    return s["out"]


def _plain_muon(s):
    g = s["g"].float()
    s["m"].mul_(MU).add_(g)
    u = g + MU * s["m"]
    us = [u[m.storage_offset():m.storage_offset() + m.numel()].view(m.shape) for m in s["ms"]]
    for at in _alike(us).values():
        for i, o in zip(at, _orthogonal(torch.stack([us[i] for i in at]))):
            _update(s["xs"][i], o)
    return {"m": s["m"], "x": s["x"]}


def _basis(n):
    """Orthonormal DCT-II: row u is the u-th basis vector."""
    at = torch.arange(n, dtype=torch.float64, device="cuda")
    c = torch.cos(math.pi * (2 * at + 1) * at[:, None] / (2 * n)) * math.sqrt(2.0 / n)
    c[0] /= math.sqrt(2.0)
    return c.float()


def _received(s):
    """R of every tensor: the workers' records summed into coefficient chunks, transformed back, the chunks put in their places."""
    case = s["case"]
    chunk, c, at, got = case["chunk"], _basis(case["chunk"]), 0, []
    for shape in s["shapes"]:
        m = chunk ** len(shape)
        k, n_chunks = min(case["topk"], m), math.prod(shape) // m
        rec = torch.stack([p.view(torch.int32).view(-1, 2)[at:at + n_chunks * k] for p in s["payloads"]]).view(-1, n_chunks, k, 2)
        at += n_chunks * k
        idx = rec[..., 0].permute(1, 0, 2).reshape(n_chunks, -1).long()
        val = rec[..., 1].permute(1, 0, 2).reshape(n_chunks, -1).contiguous().view(torch.float32)
        q = torch.zeros((n_chunks, m), device="cuda").scatter_add_(1, idx, val)
        if len(shape) == 1:
            got.append((q @ c).flatten())
        else:
            r = c.T @ q.view(n_chunks, chunk, chunk) @ c
            got.append(r.view(shape[0] // chunk, shape[1] // chunk, chunk, chunk).permute(0, 2, 1, 3).reshape(shape))
    return got


def _plain_decode(s):
    for x, r in zip(s["xs"], _received(s)):
        if x.dim() == 2:
            _update(x, _orthogonal(r[None])[0])
        else:
            x.copy_(x - LR * (torch.sign(r) + WD * x))
    return s["x"]


def _plain_adamw(s):
    s["step"].add_(1)
    t = s["step"].double()
    c1, c2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).float()
    g = s["g"].float()
    m = s["m"].mul_(BETA1).add_((1 - BETA1) * g)
    v = s["v"].mul_(BETA2).add_((1 - BETA2) * g.square())
    s["x"].mul_(1 - LR * WD).sub_(LR * (m / c1) / ((v / c2).sqrt() + ADAM_EPS))
    return {"m": m, "v": v, "x": s["x"], "step": s["step"]}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"ortho": _plain_ortho, "muon": _plain_muon, "decode": _plain_decode, "adamw": _plain_adamw}[op](s)
    if op == "ortho":
        s["muon"].orthogonalize(s["gs"], s["outs"])
        return s["out"]
    if op == "muon":
        s["muon"].step(s["gs"], s["ms"], s["xs"])
        return {"m": s["m"], "x": s["x"]}
    if op == "decode":
        s["muon"].decode_apply(s["demo"], s["payloads"], s["xs"])
        return s["x"]
    s["adamw"].step(s["gs"], s["ms"], s["vs"], s["xs"], s["step"])
    return {"m": s["m"], "v": s["v"], "x": s["x"], "step": s["step"]}


# --- the definitions in 64 bits ----------------------------------------------------------------------------------------------


def _exact_polar(u):
    u = u.double()
    y = u / (torch.linalg.norm(u) + EPS)
    for _ in range(STEPS):
        # the Gram matrix of the shorter side: X (b G + c G G) from the right, or (b G + c G G) X from the left
        if y.shape[0] > y.shape[1]:
            gram = y.T.mm(y)
            y = y.mul(A).addmm(y, gram.mul(B).addmm(gram, gram, alpha=C))
        else:
            gram = y.mm(y.T)
            y = y.mul(A).addmm(gram.mul(B).addmm(gram, gram, alpha=C), y)
    return y


def _exact_received(s):
    case, at = s["case"], 0
    n = case["chunk"]
    i = torch.arange(n, dtype=torch.float64, device="cuda")
    rows = [torch.full_like(i, n ** -0.5)] + [torch.cos((i + 0.5) * (math.pi * f / n)) * (2.0 / n) ** 0.5 for f in range(1, n)]
    basis = torch.stack(rows)
    for shape in s["shapes"]:
        m = n ** len(shape)
        k, count = min(case["topk"], m), math.prod(shape) // m
        q = torch.zeros(count * m, dtype=torch.float64, device="cuda")
        base = torch.arange(count, device="cuda").repeat_interleave(k) * m
        for p in s["payloads"]:
            rec = p.view(torch.int32)[2 * at:2 * (at + count * k)].view(-1, 2)
            q.index_put_((base + rec[:, 0],), rec[:, 1].contiguous().view(torch.float32).double(), accumulate=True)
        at += count * k
        if len(shape) == 1:
            yield torch.einsum("cu,un->cn", q.view(count, n), basis).reshape(-1)
        else:
            r = torch.einsum("abuv,ui,vj->aibj", q.view(shape[0] // n, shape[1] // n, n, n), basis, basis)
            yield r.reshape(shape)


def exact(case, seed):
    s = prepare(case, seed)
    like = lambda flat: torch.zeros(flat.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    view = lambda flat, t: flat[t.storage_offset():t.storage_offset() + t.numel()].view(t.shape)  # noqa: E731
    op = case["op"]
    if op == "ortho":
        out = like(s["out"])
        for g, o in zip(s["gs"], s["outs"]):
            view(out, o).copy_(_exact_polar(g))
        return out
    x = like(s["x"])
    if op == "adamw":
        g, t = s["g"].double(), int(s["step"]) + 1
        m = BETA1 * s["m"].double() + (1 - BETA1) * g
        v = BETA2 * s["v"].double() + (1 - BETA2) * g * g
        step = (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
        x.copy_(s["x"].double() * (1 - LR * WD) - LR * step)
        return {"m": m, "v": v, "x": x, "step": None}
    if op == "muon":
        m = MU * s["m"].double() + s["g"].double()
        u = s["g"].double() + MU * m
        rs = (view(u, t) for t in s["ms"])
    else:
        rs = _exact_received(s)
    for t, r in zip(s["xs"], rs):
        new, old = view(x, t), t.double()
        if t.dim() == 2:
            new.copy_((1 - LR * WD) * old - LR * 0.2 * max(t.shape) ** 0.5 * _exact_polar(r))
        else:
            new.copy_((1 - LR * WD) * old - LR * torch.sgn(r))
    return {"m": m, "x": x} if op == "muon" else x
