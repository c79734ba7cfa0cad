"""Performance cases of the grouped products and of the low-rank adapters.

Grouped products: rows of activations sorted by group (tokens sorted by the expert that a router gave
them to), offsets[g] .. offsets[g + 1] - 1 being the rows of group g, and one weight per group, the bf16
matrices that mwu_decode or mwu_keep_n_of_m leave of compressed experts, stacked.

  product      Y[m] = X[m] W_g^T                      mwu_gemm_grouped
  input_grad   dX[m] = dY[m] W_g                      mwu_gemm_grouped_dx
  weight_grad  dW_g = dY_g^T X_g                      mwu_gemm_grouped_dw
  train        all three on the same groups

Low-rank adapters beside a shared projection: segments of rows (the requests of a batch), each with the
number of its adapter (-1: none).

  adapters      Y[m] = Y0[m] + s_a (X[m] A_a^T) B_a^T     mwu_adapters_add
  adapter_grad  a training step's gradients of X, A and B, which are grouped products with a side as long
                as the rank: T = X A^T, dT = dY B, dX = dT A, dA_g = dT_g^T X_g, dB_g = dY_g^T T_g

The lengths of groups and segments follow from the case alone, the values from the seed: weights
N(0, 0.02^2) with a quarter of their 1x4 blocks pruned to zero, activations and gradients N(0, 1).
Rows that belong to no group or segment keep what the output held.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _grouped(kind, groups, m, rows, cols, mix, behind=0, fp32_out=False):
    """m rows in `groups` groups drawn with `mix`, `behind` more rows that belong to none."""
    return {"kind": kind, "groups": groups, "m": m, "rows": rows, "cols": cols, "mix": mix, "behind": behind,
            "fp32_out": fp32_out}


def _adapters(tokens, prompts, prompt_rows, adapters, rank, rows, cols, mix, fp32_out=False):
    """`tokens` requests of one row and `prompts` requests that share prompt_rows rows, in a mixed order."""
    return {"kind": "adapters", "tokens": tokens, "prompts": prompts, "prompt_rows": prompt_rows,
            "adapters": adapters, "rank": rank, "rows": rows, "cols": cols, "mix": mix, "fp32_out": fp32_out}


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # one token given to two of eight small experts: latency
    add("experts_one_token", _grouped("product", 8, 2, 1024, 1024, 1))
    # 128 tokens being generated, two experts each: every expert's weights are read for a few rows
    add("experts_decode", _grouped("product", 64, 256, 2048, 4096, 2))
    # a prompt of 8192 tokens, two experts each: tensor cores
    add("experts_prompt", _grouped("product", 16, 16384, 4096, 4096, 3))
    # sizes that divide nothing, a buffer longer than what was routed, fp32 results
    add("experts_ragged_fp32", _grouped("product", 7, 2903, 1000, 1216, 4, behind=98, fp32_out=True))
    # the backward pass of such a layer with respect to its input
    add("experts_input_grad", _grouped("input_grad", 16, 8192, 4096, 4096, 5))
    # and with respect to the experts: the fp32 gradients that the W-step adds to rho * U_next
    add("experts_weight_grad", _grouped("weight_grad", 16, 16384, 2048, 4096, 6, fp32_out=True))
    # a whole step of a layer whose sizes divide nothing
    add("experts_train_ragged", _grouped("train", 12, 5003, 1416, 1096, 7, behind=21))
    # one token of one request with an adapter
    add("adapter_one_token", _adapters(1, 0, 0, 4, 16, 4096, 4096, 8))
    # 64 requests generating, 32 adapters on an FFN up-projection
    add("adapters_decode", _adapters(64, 0, 0, 32, 32, 16384, 4096, 9))
    # prompts of six requests
    add("adapters_prompts", _adapters(0, 6, 8192, 4, 64, 4096, 4096, 10))
    # prompts and single tokens in one batch, some without an adapter, odd sizes, fp32 results
    add("adapters_mixed_fp32", _adapters(61, 5, 2777, 16, 24, 1000, 1216, 11, fp32_out=True))
    # training four adapters on one layer
    add("adapters_grad", {"kind": "adapter_grad", "groups": 4, "m": 8192, "rank": 64, "rows": 4096, "cols": 4096, "mix": 12})
    return out


# ---------------------------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------------------------
_MAX_MACS = 16384 * 4096 * 4096
_MAX_WEIGHTS = 64 * 2048 * 4096


def _log(rng, lo, hi):
    """Log-uniform whole number in [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["product", "product", "input_grad", "weight_grad", "train", "adapters", "adapters", "adapter_grad"])
    mix = rng.randrange(1 << 20)
    while True:
        rows, cols = 8 * _log(rng, 8, 768), 8 * _log(rng, 8, 768)
        if rng.random() < 0.5:
            rows, cols = max(128, rows // 128 * 128), max(128, cols // 128 * 128)
        if kind == "adapters":
            tokens, prompts = rng.choice([0, _log(rng, 1, 128)]), rng.choice([0, _log(rng, 1, 8)])
            if tokens + prompts == 0:
                continue
            prompt_rows = _log(rng, 16 * prompts, 8192) if prompts else 0
            rank = rng.choice([4, 8, 16, 16, 32, 64, 128, rng.randrange(1, 129)])
            # (the plain form pads every request to the longest)
            if (tokens + prompts) * (prompt_rows / max(1, prompts) + 1) * (rows + cols) <= 1 << 30:
                return _adapters(tokens, prompts, prompt_rows, _log(rng, 1, 64), rank, rows, cols, mix, rng.random() < 0.25)
            continue
        groups, m = _log(rng, 1, 64), _log(rng, 1, 16384)
        if kind == "adapter_grad":
            groups = min(groups, 16)
            if m * (rows + cols) <= 1 << 27:
                return {"kind": kind, "groups": groups, "m": m, "rank": 8 * _log(rng, 1, 16), "rows": rows, "cols": cols,
                        "mix": mix}
            continue
        if groups * rows * cols * (2 if kind == "weight_grad" else 3 if kind == "train" else 1) > _MAX_WEIGHTS:
            continue
        if m * rows * cols * (3 if kind == "train" else 1) > _MAX_MACS // 2:
            continue
        return _grouped(kind, groups, m, rows, cols, mix, rng.choice([0, 0, rng.randrange(1, 100)]),
                        kind == "weight_grad" or rng.random() < 0.25)


# ---------------------------------------------------------------------------------------------
# lengths: from the case alone
# ---------------------------------------------------------------------------------------------
def _lengths(total, parts, mix, least=0):
    """`total` rows in `parts` runs of uneven length, some of them empty when rows are few."""
    r = random.Random(mix)
    want = [math.exp(r.gauss(0.0, 0.6)) for _ in range(parts)]
    if parts > 4 and not least:
        want[r.randrange(parts)] = 0.0                  # an expert that nobody asked for
    got = [least] * parts
    for p in r.choices(range(parts), want, k=total - least * parts):
        got[p] += 1
    return got


def _segments(case):
    """(lengths, adapters) of the requests of an adapter case, in batch order."""
    r = random.Random(case["mix"])
    runs = [1] * case["tokens"]
    if case["prompts"]:
        runs += _lengths(case["prompt_rows"], case["prompts"], case["mix"] + 1, least=1)
    r.shuffle(runs)
    # one request in eight works without an adapter
    which = [-1 if len(runs) > 4 and r.random() < 0.125 else r.randrange(case["adapters"]) for _ in runs]
    return runs, which


def _group_lengths(case):
    return _lengths(case["m"], case["groups"], case["mix"])


def _offsets(lengths):
    at, out = 0, [0]
    for n in lengths:
        at += n
        out.append(at)
    return out


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _weights(gen, n, rows, cols):
    w = torch.empty((n, rows, cols), dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=gen)
    if cols % 4 == 0:
        keep = torch.rand((n, rows, cols // 4), generator=gen, device="cuda") >= 0.25
        w.view(n, rows, cols // 4, 4).mul_(keep.unsqueeze(-1))
    return w


def _normal(gen, *shape):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(generator=gen)


def _slots(lengths):
    """Row -> its place among runs that are all as long as the longest."""
    longest = max(1, max(lengths))
    at = [g * longest + i for g, n in enumerate(lengths) for i in range(n)]
    return torch.tensor(at, dtype=torch.int64, device="cuda"), longest


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, rows, cols = case["kind"], case["rows"], case["cols"]
    s = {"kind": kind, "rows": rows, "cols": cols, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if kind == "adapters":
        lengths, which = _segments(case)
        m, rank = sum(lengths), case["rank"]
        pad = (rank + 7) // 8 * 8                       # rows of B start on 16-byte boundaries
        s["out"] = F32 if case["fp32_out"] else BF16
        s["rank"], s["ldb"] = rank, pad
        s["X"] = _normal(gen, m, cols)
        s["A"] = torch.empty((case["adapters"], rank, cols), dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=gen)
        s["B"] = torch.empty((case["adapters"], rows, pad), dtype=BF16, device="cuda").normal_(0.0, 0.1, generator=gen)
        s["scale"] = torch.rand(case["adapters"], generator=gen, device="cuda") + 0.5
        s["which"] = torch.tensor(which, dtype=torch.int32, device="cuda")
        s["Y0"] = _normal(gen, m, rows).to(s["out"])
        s["Y"] = torch.empty((m, rows), dtype=s["out"], device="cuda")
    elif kind == "adapter_grad":
        lengths, m, rank = _group_lengths(case), case["m"], case["rank"]
        s["rank"] = rank
        s["X"], s["dY"] = _normal(gen, m, cols), _normal(gen, m, rows)
        s["A"] = torch.empty((case["groups"], rank, cols), dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=gen)
        s["B"] = torch.empty((case["groups"], rows, rank), dtype=BF16, device="cuda").normal_(0.0, 0.1, generator=gen)
        s["T"], s["dT"] = (torch.empty((m, rank), dtype=BF16, device="cuda") for _ in range(2))
        s["dX"], s["dA"], s["dB"] = (torch.empty_like(s[k]) for k in ("X", "A", "B"))
    else:
        lengths = _group_lengths(case)
        m = case["m"] + case["behind"]
        s["out"] = F32 if case["fp32_out"] else BF16
        if kind != "weight_grad":
            s["W"] = _weights(gen, case["groups"], rows, cols)
        if kind != "input_grad":
            s["X"] = _normal(gen, m, cols)
        if kind != "product":
            s["dY"] = _normal(gen, m, rows)
        if kind in ("product", "train"):
            s["Y"] = _normal(gen, m, rows).to(s["out"])
        if kind in ("input_grad", "train"):
            s["dX"] = _normal(gen, m, cols).to(s["out"])
        if kind in ("weight_grad", "train"):
            s["dW"] = torch.empty((case["groups"], rows, cols), dtype=F32, device="cuda")
    s["m"], s["n_runs"] = m, len(lengths)
    s["offsets"] = torch.tensor(_offsets(lengths), dtype=torch.int32, device="cuda")
    s["used"] = sum(lengths)
    s["slot"], s["longest"] = _slots(lengths)
    return s


# ---------------------------------------------------------------------------------------------
# plain forms: every run padded to the longest, batched products in 32 bits
# ---------------------------------------------------------------------------------------------
def _padded(s, x):
    p = torch.zeros((s["n_runs"] * s["longest"], x.shape[1]), dtype=F32, device=x.device)
    p[s["slot"]] = x[: s["used"]].float()
    return p.view(s["n_runs"], s["longest"], x.shape[1])


def _unpadded(s, p):
    return p.reshape(s["n_runs"] * s["longest"], p.shape[2])[s["slot"]]


def _plain_grouped(s):
    out = {}
    if s["kind"] in ("product", "train"):
        s["Y"][: s["used"]] = _unpadded(s, _padded(s, s["X"]) @ s["W"].float().transpose(1, 2)).to(s["out"])
        out["Y"] = s["Y"]
    if s["kind"] in ("input_grad", "train"):
        s["dX"][: s["used"]] = _unpadded(s, _padded(s, s["dY"]) @ s["W"].float()).to(s["out"])
        out["dX"] = s["dX"]
    if s["kind"] in ("weight_grad", "train"):
        torch.matmul(_padded(s, s["dY"]).transpose(1, 2), _padded(s, s["X"]), out=s["dW"])
        out["dW"] = s["dW"]
    return out


def _plain_adapters(s):
    a = s["which"].long().clamp(min=0)
    scale = torch.where(s["which"] >= 0, s["scale"][a], torch.zeros_like(s["scale"][a]))
    t = _padded(s, s["X"]) @ s["A"][a].float().transpose(1, 2)
    low = (t @ s["B"][a][:, :, : s["rank"]].float().transpose(1, 2)) * scale[:, None, None]
    s["Y"].copy_(s["Y0"].float() + _unpadded(s, low))
    return {"Y": s["Y"]}


def _plain_adapter_grad(s):
    x, dy, a, b = _padded(s, s["X"]), _padded(s, s["dY"]), s["A"].float(), s["B"].float()
    dt = dy @ b
    s["dX"].copy_(_unpadded(s, dt @ a))
    s["dA"].copy_(dt.transpose(1, 2) @ x)
    s["dB"].copy_(dy.transpose(1, 2) @ (x @ a.transpose(1, 2)))
    return {"dX": s["dX"], "dA": s["dA"], "dB": s["dB"]}


# ---------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------
def _own_grouped(s):
    from paper_2106_08301_b200 import binding as B
    g, n, k, m, st = s["n_runs"], s["rows"], s["cols"], s["m"], s["status"]
    fp32, out = int(s["out"] == F32), {}
    if s["kind"] in ("product", "train"):
        B.mwu_gemm_grouped(g, n, k, s["W"], k, n * k, s["offsets"], s["X"], m, k, s["Y"], n, fp32, st)
        out["Y"] = s["Y"]
    if s["kind"] in ("input_grad", "train"):
        B.mwu_gemm_grouped_dx(g, n, k, s["W"], k, n * k, s["offsets"], s["dY"], m, n, s["dX"], k, fp32, st)
        out["dX"] = s["dX"]
    if s["kind"] in ("weight_grad", "train"):
        B.mwu_gemm_grouped_dw(g, n, k, s["offsets"], s["dY"], m, n, s["X"], k, s["dW"], k, n * k, 1, 0, st)
        out["dW"] = s["dW"]
    return out


def _own_adapters(s):
    from paper_2106_08301_b200 import binding as B
    n, k, r = s["rows"], s["cols"], s["rank"]
    B.mwu_adapters_add(s["A"].shape[0], r, n, k, s["A"], k, r * k, s["B"], s["ldb"], n * s["ldb"], s["scale"], s["n_runs"],
                       s["offsets"], s["which"], s["X"], s["m"], k, s["Y0"], s["Y"], n, int(s["out"] == F32), s["status"])
    return {"Y": s["Y"]}


def _own_adapter_grad(s):
    from paper_2106_08301_b200 import binding as B
    g, n, k, r, m, off, st = s["n_runs"], s["rows"], s["cols"], s["rank"], s["m"], s["offsets"], s["status"]
    B.mwu_gemm_grouped(g, r, k, s["A"], k, r * k, off, s["X"], m, k, s["T"], r, 0, st)
    B.mwu_gemm_grouped_dx(g, n, r, s["B"], r, n * r, off, s["dY"], m, n, s["dT"], r, 0, st)
    B.mwu_gemm_grouped_dx(g, r, k, s["A"], k, r * k, off, s["dT"], m, r, s["dX"], k, 0, st)
    B.mwu_gemm_grouped_dw(g, r, k, off, s["dT"], m, r, s["X"], k, s["dA"], k, r * k, 0, 0, st)
    B.mwu_gemm_grouped_dw(g, n, r, off, s["dY"], m, n, s["T"], r, s["dB"], r, n * r, 0, 0, st)
    return {"dX": s["dX"], "dA": s["dA"], "dB": s["dB"]}


def run(state):
    kind = state["kind"]
    if kind == "adapters":
        return _own_adapters(state) if own else _plain_adapters(state)
    if kind == "adapter_grad":
        return _own_adapter_grad(state) if own else _plain_adapter_grad(state)
    return _own_grouped(state) if own else _plain_grouped(state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    kind, n, k = case["kind"], case["rows"], case["cols"]
    out = 4 if case.get("fp32_out") else 2
    if kind == "adapters":
        lengths, which = _segments(case)
        m, r = sum(lengths), case["rank"]
        served = sum(x for x, a in zip(lengths, which) if a >= 0)
        adapters = len({a for a in which if a >= 0})
        return {"bytes": served * k * 2 + 2 * m * n * out + adapters * r * (n + k) * 2, "flops": 2 * served * r * (n + k)}
    m = case["m"]
    if kind == "adapter_grad":
        r, g = case["rank"], case["groups"]
        return {"bytes": 2 * (2 * m * k + m * n + 2 * g * r * (n + k)), "flops": m * r * (4 * n + 6 * k)}
    live = sum(x > 0 for x in _group_lengths(case))
    w = live * n * k * 2
    b = {"product": w + 2 * m * k + out * m * n, "input_grad": w + 2 * m * n + out * m * k,
         "weight_grad": 2 * m * (n + k) + 4 * case["groups"] * n * k,
         "train": w + 2 * m * (n + k) + out * m * (n + k) + 4 * case["groups"] * n * k}[kind]
    return {"bytes": b, "flops": 2 * m * n * k * (3 if kind == "train" else 1)}


# ---------------------------------------------------------------------------------------------
# the definition, in 64 bits, run by run
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind, at = s["kind"], s["offsets"].tolist()
    spans = [(g, slice(at[g], at[g + 1])) for g in range(s["n_runs"])]
    if kind == "adapters":
        y = s["Y0"].to(F64)
        for (g, rows), a in zip(spans, s["which"].tolist()):
            if a >= 0:
                low = s["A"][a].to(F64) @ s["X"][rows].to(F64).T
                y[rows] += float(s["scale"][a]) * (s["B"][a, :, : s["rank"]].to(F64) @ low).T
        return {"Y": y}
    if kind == "adapter_grad":
        dx, da, db = s["X"].to(F64), s["A"].to(F64), s["B"].to(F64)
        for g, rows in spans:
            x, dy, a, b = s["X"][rows].to(F64), s["dY"][rows].to(F64), s["A"][g].to(F64), s["B"][g].to(F64)
            dx[rows] = dy @ (b @ a)
            da[g] = (b.T @ dy.T) @ x
            db[g] = dy.T @ torch.einsum("mk,rk->mr", x, a)
        return {"dX": dx, "dA": da, "dB": db}
    out = {}
    if kind in ("product", "train"):
        out["Y"] = s["Y"].to(F64)
        for g, rows in spans:
            out["Y"][rows] = torch.einsum("mk,nk->mn", s["X"][rows].to(F64), s["W"][g].to(F64))
    if kind in ("input_grad", "train"):
        out["dX"] = s["dX"].to(F64)
        for g, rows in spans:
            out["dX"][rows] = torch.einsum("mn,nk->mk", s["dY"][rows].to(F64), s["W"][g].to(F64))
    if kind in ("weight_grad", "train"):
        out["dW"] = torch.zeros(s["dW"].shape, dtype=F64, device="cuda")
        for g, rows in spans:
            out["dW"][g] = torch.einsum("mn,mk->nk", s["dY"][rows].to(F64), s["X"][rows].to(F64))
    return out
