"""Low-rank adapters and dropout beside the restructured FFN, as timed cases.

Three operators.  ``adapters``: out = base + s_a B_a A_a x for rows of many requests, each with its own adapter (or
none), beside a projection that all of them share; in training the rows of x pass a dropout first and z = A x is kept.
``adapters_grad``: its gradients by x, A and B.  ``dropout``: the keep mask of a counter-based generator applied to a
matrix (with a residual added in the forward pass); the mask is a function of (seed, offset, row, column) and is never
stored.  Model dimensions are those of ``workloads.WORKLOADS`` or generic ones; rank 8 and alpha 32 are the paper's
fine-tuning setting.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ALPHA = 32.0


# ------------------------------------------------------------------ the cases
def _adapters(name, rows, n, rank, d_in, d_out, *, op="adapters", dtype="bf16", ids="mixed", p=0.0, base=True):
    c = dict(op=op, rows=rows, n=n, rank=rank, d_in=d_in, d_out=d_out, dtype=dtype, ids=ids, p=p, base=base)
    return dict(c, name=name) if name else c


def _dropout(name, rows, cols, *, op="dropout", dtype="bf16", p=0.1, residual=True):
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, p=p, residual=residual)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request, the decode step of a single user: launch and latency
        _adapters("one_token", 1, 8, 8, 4096, 4096),
        # a decode batch in which nearly every request has an adapter of its own
        _adapters("decode_64_of_64", 64, 64, 16, 4096, 4096),
        # a larger decode batch over few tenants, beside a widening projection
        _adapters("decode_200_wide", 200, 24, 32, 5120, 13824),
        # prompts of eight requests, packed one after another
        _adapters("prompts_8117", 8117, 8, 16, 4096, 4096, ids="segments"),
        # the forward of a fine-tuning step: one adapter, dropout before it, z kept for the gradients
        _adapters("tune_4096", 4096, 1, 8, 4096, 11008, ids="one", p=0.05),
        # a toy layer in fp32, as in unit tests
        _adapters("tiny_fp32_64", 64, 3, 8, 256, 1024, dtype="fp32"),
        # the gradients of a fine-tuning step at the paper's rank
        _adapters("tune_4096_grad", 4096, 1, 8, 4096, 4096, op="adapters_grad", ids="one", p=0.05, base=False),
        # four adapters of large rank tuned at once on a long packed batch, added to the projection's own dx
        _adapters("tune_16384_r64_grad", 16384, 4, 64, 5120, 5120, op="adapters_grad", ids="segments"),
        # the toy layer's gradients in fp32, rows of three adapters mixed
        _adapters("tiny_fp32_1000_grad", 1000, 3, 16, 256, 1024, op="adapters_grad", dtype="fp32", p=0.1),
        # dropout of a sublayer's output, added to the residual stream, 13B-shaped
        _dropout("residual_16384", 16384, 5120),
        # a small ragged micro-batch of a toy model in fp32, forward
        _dropout("small_fp32_77", 77, 250, dtype="fp32", p=0.25),
        # the backward pass of a dropout over rows of odd width
        _dropout("grad_4099_odd", 4099, 1377, op="dropout_grad", p=0.05, residual=False),
    ]


MOST_BYTES = 6.5e8      # somewhat less than the largest listed case moves


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        if rng.random() < 0.3:
            grad = rng.random() < 0.4
            c = _dropout("", log(1, 16384), log(1, 14336), op="dropout_grad" if grad else "dropout", dtype=dtype,
                         p=rng.choice([0.05, 0.1, 0.25, 0.5]), residual=not grad and rng.random() < 0.7)
        else:
            grad = rng.random() < 0.45
            ids = rng.choice(["mixed", "segments", "one"])
            rows = log(16, 16384) if grad else log(1, 16384)
            c = _adapters("", rows, 1 if ids == "one" else log(1, 128 if rows <= 2048 else 16), 8 * log(1, 8),
                          8 * log(8, 1792), 8 * log(8, 1792), op="adapters_grad" if grad else "adapters", dtype=dtype,
                          ids=ids, p=rng.choice([0.0, 0.0, 0.05, 0.1]), base=rng.random() < 0.7)
        if work(c)["bytes"] <= MOST_BYTES and (c["op"].startswith("dropout") or c["rows"] * c["n"] * c["rank"] <= 3e6):
            return c


# ------------------------------------------------------------------ inputs
def _row_ids(case, g):
    """The adapter of every row; -1: none (requests of the bare model, padding)."""
    rows, n, kind = case["rows"], case["n"], case["ids"]
    if kind == "one":
        return None
    if kind == "mixed":
        ids = torch.randint(0, n, (rows,), generator=g, device="cuda")
        if rows > 1:
            ids = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.06, torch.full_like(ids, -1), ids)
        return ids.to(torch.int32)
    cuts = torch.sort(torch.randint(0, rows + 1, (n,), generator=g, device="cuda")).values      # n + 1 segments
    ids = torch.bucketize(torch.arange(rows, device="cuda"), cuts, right=True)
    order = torch.randperm(n + 1, generator=g, device="cuda") - 1                               # one of them without an adapter
    return order[ids].to(torch.int32)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    s = dict(case=case, key=1_000_003 * seed + 17, offset=seed % 1000)
    if case["op"].startswith("dropout"):
        s["x"] = normal(case["rows"], case["cols"])
        s["residual"] = normal(case["rows"], case["cols"]) if case["residual"] else None
        return s
    rows, n, r, d_in, d_out = (case[k] for k in ("rows", "n", "rank", "d_in", "d_out"))
    s["ids"] = _row_ids(case, g)
    s["a"] = normal(n, r, d_in, std=1.0 / math.sqrt(d_in))
    s["b"] = normal(n, d_out, r, std=0.02)
    s["scale"] = torch.full((n,), ALPHA / r, device="cuda") * (0.5 + torch.rand(n, generator=g, device="cuda"))
    s["x"] = normal(rows, d_in)
    if case["op"] == "adapters":
        s["base"] = normal(rows, d_out) if case["base"] else None
    else:
        s["dy"] = normal(rows, d_out, std=1e-2)
        s["z"] = torch.randn(rows, r, generator=g, device="cuda")
        if s["ids"] is not None:
            s["z"] *= (s["ids"] >= 0).unsqueeze(1)
        s["base"] = normal(rows, d_in, std=1e-2) if case["base"] else None
    return s


# ------------------------------------------------------------------ plain forms
def _mul_hi_lo(a, m):
    """The two halves of the 64-bit product of 32-bit numbers (held in int64, whose product wraps to the same bits)."""
    prod = a * m
    return (prod >> 32) & 0xFFFFFFFF, prod & 0xFFFFFFFF


def _keep(rows, cols, p, key, offset):
    """Philox 4x32 of ten rounds (Salmon et al. 2011) on the counter (column / 8, row, offset), eight 16-bit draws a block."""
    c0 = torch.arange((cols + 7) // 8, device="cuda").unsqueeze(0).expand(rows, -1)
    c1 = torch.arange(rows, device="cuda").unsqueeze(1).expand_as(c0)
    c2, c3 = torch.full_like(c0, offset & 0xFFFFFFFF), torch.full_like(c0, offset >> 32)
    k0, k1 = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        h0, l0 = _mul_hi_lo(c0, 0xD2511F53)
        h1, l1 = _mul_hi_lo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = torch.stack([h for w in (c0, c1, c2, c3) for h in (w & 0xFFFF, w >> 16)], dim=-1)
    return halves.reshape(rows, -1)[:, :cols] >= int(p * 65536 + 0.5)


def _dropped(x, case, s):
    """x in 32 bits with the mask and its scale applied."""
    if case["p"] == 0:
        return x.float()
    inv = 65536.0 / (65536 - int(case["p"] * 65536 + 0.5))
    return torch.where(_keep(*x.shape, case["p"], s["key"], s["offset"]), x.float() * inv, torch.zeros((), device="cuda"))


def _own_columns(ids, rows, n, r):
    """[rows, n * r]: whether a column of the stacked adapters belongs to the row's own adapter."""
    if ids is None:
        return torch.ones(rows, n * r, dtype=torch.bool, device="cuda")
    return (ids.unsqueeze(1) == torch.arange(n, device="cuda").unsqueeze(0)).repeat_interleave(r, dim=1)


def _plain_adapters(s):
    case, n, r = s["case"], s["case"]["n"], s["case"]["rank"]
    xd = _dropped(s["x"], case, s)
    mine = _own_columns(s["ids"], case["rows"], n, r)
    z_all = torch.where(mine, xd @ s["a"].float().reshape(n * r, -1).t(), 0.0)
    b_all = (s["b"].float() * s["scale"].view(n, 1, 1)).permute(0, 2, 1).reshape(n * r, -1)
    out = z_all @ b_all
    if s["base"] is not None:
        out = out + s["base"].float()
    out = out.to(s["x"].dtype)
    return (out, z_all.view(-1, n, r).sum(1)) if case["p"] > 0 else out


def _plain_adapters_grad(s):
    case, n, r = s["case"], s["case"]["n"], s["case"]["rank"]
    dtype, dy = s["x"].dtype, s["dy"].float()
    mine = _own_columns(s["ids"], case["rows"], n, r)
    b_all = (s["b"].float() * s["scale"].view(n, 1, 1)).permute(0, 2, 1).reshape(n * r, -1)
    e_all = torch.where(mine, dy @ b_all.t(), 0.0)
    grad_a = (e_all.t() @ _dropped(s["x"], case, s)).view(n, r, -1)
    z_all = torch.where(mine, s["z"].unsqueeze(1).expand(-1, n, -1).reshape(-1, n * r), 0.0)
    grad_b = (z_all.t() @ dy).view(n, r, -1).permute(0, 2, 1) * s["scale"].view(n, 1, 1)
    dx = _dropped(e_all @ s["a"].float().reshape(n * r, -1), case, s)
    if s["base"] is not None:
        dx = dx + s["base"].float()
    return dx.to(dtype), grad_a.to(dtype), grad_b.to(dtype)


def _plain_dropout(s):
    out = _dropped(s["x"], s["case"], s)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["x"].dtype)


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2502_04416_b200 import binding
        drop = binding.Dropout(case["p"], state["key"], state["offset"]) if case["p"] > 0 else None
        if case["op"] == "adapters":
            return binding.adapter_forward(state["x"], state["a"], state["b"], state["ids"], state["scale"],
                                           base=state["base"], dropout=drop, want_z=case["p"] > 0)
        if case["op"] == "adapters_grad":
            return binding.adapter_backward(state["dy"], state["x"], state["z"], state["a"], state["b"], state["ids"],
                                            state["scale"], dx_base=state["base"], dropout=drop)
        return binding.dropout(state["x"], drop, residual=state["residual"])
    if case["op"] == "adapters":
        return _plain_adapters(state)
    if case["op"] == "adapters_grad":
        return _plain_adapters_grad(state)
    return _plain_dropout(state)


def work(case):
    """Each input read once, each output written once; weights of the adapters that rows can name (at most one a row)."""
    e = 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if case["op"].startswith("dropout"):
        n = rows * case["cols"]
        return {"bytes": float(n * e * (3 if case["residual"] else 2)), "flops": float(2 * n)}
    n, r, d_in, d_out = (case[k] for k in ("n", "rank", "d_in", "d_out"))
    weights = min(n, rows) * r * (d_in + d_out) * e
    ids = 0 if case["ids"] == "one" else 4 * rows
    if case["op"] == "adapters":
        z = rows * r * 4 if case["p"] > 0 else 0
        return {"bytes": float(weights + ids + z + rows * (d_in + d_out * (2 if case["base"] else 1)) * e),
                "flops": float(2 * rows * r * (d_in + d_out))}
    return {"bytes": float(weights + n * r * (d_in + d_out) * e + ids + rows * r * 4
                           + rows * (d_out + d_in * (3 if case["base"] else 2)) * e),
            "flops": float(4 * rows * r * (d_in + d_out))}


# ------------------------------------------------------------------ the definition in 64 bits
def _philox_keep(rows, cols, p, key, offset):
    """The keep mask by unsigned 64-bit words on the host."""
    low = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    blocks = -(-cols // 8)
    x = np.tile(np.arange(blocks, dtype=np.uint64), rows)
    y = np.repeat(np.arange(rows, dtype=np.uint64), blocks)
    u = np.full_like(x, offset & 0xFFFFFFFF)
    v = np.full_like(x, offset >> 32)
    a, b = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        p0, p1 = x * np.uint64(0xD2511F53), u * np.uint64(0xCD9E8D57)
        x, y, u, v = (p1 >> sh) ^ y ^ np.uint64(a), p1 & low, (p0 >> sh) ^ v ^ np.uint64(b), p0 & low
        a, b = (a + 0x9E3779B9) % 2**32, (b + 0xBB67AE85) % 2**32
    bits = np.stack([x, y, u, v], axis=1).astype("<u4").view("<u2")       # little-endian: the low half comes first
    return torch.from_numpy((bits >= np.floor(p * 65536 + 0.5)).reshape(rows, blocks * 8)[:, :cols].copy()).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["p"] > 0:
        if x.numel() > 1.7e8:
            return None
        mask = _philox_keep(x.shape[0], x.shape[1], case["p"], s["key"], s["offset"]).double()
        mask *= 1.0 / (1.0 - math.floor(case["p"] * 65536 + 0.5) / 65536)
    else:
        mask = torch.ones((), dtype=torch.float64, device="cuda")
    if case["op"].startswith("dropout"):
        return x * mask + (0.0 if s["residual"] is None else s["residual"].double())
    rows, n, r = case["rows"], case["n"], case["rank"]
    ids = s["ids"].long() if s["ids"] is not None else torch.zeros(rows, dtype=torch.long, device="cuda")
    members = [torch.nonzero(ids == k).flatten() for k in range(n)]
    xd = x * mask
    if case["op"] == "adapters":
        out = torch.zeros(rows, case["d_out"], dtype=torch.float64, device="cuda")
        if s["base"] is not None:
            out += s["base"].double()
        z = torch.zeros(rows, r, dtype=torch.float64, device="cuda")
        for k, m in enumerate(members):
            z[m] = torch.einsum("td,rd->tr", xd[m], s["a"][k].double())
            out[m] += s["scale"][k].double() * torch.einsum("tr,or->to", z[m], s["b"][k].double())
        return (out, z) if case["p"] > 0 else out
    dy, z = s["dy"].double(), s["z"].double()
    dx = torch.zeros_like(x)
    grad_a = torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda")
    grad_b = torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for k, m in enumerate(members):
        sk, a, b = s["scale"][k].double(), s["a"][k].double(), s["b"][k].double()
        e = sk * torch.einsum("to,or->tr", dy[m], b)
        dx[m] = torch.einsum("tr,rd->td", e, a)
        grad_a[k] = torch.einsum("tr,td->rd", e, xd[m])
        grad_b[k] = sk * torch.einsum("to,tr->or", dy[m], z[m])
    dx = dx * mask
    return (dx if s["base"] is None else dx + s["base"].double()), grad_a, grad_b
