"""The grouped products of layers with experts and with low-rank adapters: the calls whose speed matters to a user of them,
from one decoding step to a large batch, next to the same results from elementary operations.

Tokens are rows of row-major tensors here, which is what the C interface calls columns: a (tokens, width) tensor is a
column-major width x tokens matrix.  `call` says which operator a case runs:

  experts       y[t] = W[e] x[t] for the rows t of group e (a layer of experts, forward)
  experts_dx    x's gradient: W[e]^T g[t]
  experts_dw    the weights' gradients: W[e] <- sum over the group's rows of g[t] x[t]^T (+ what is there already)
  adapters      y[t] = W x[t] + s[a] U[a] (D[a] x[t]), a the adapter of the request that row t belongs to
  adapters_dx   x's gradient of that: W^T g[t] + s[a] D[a]^T (U[a]^T g[t])

Rows that belong to no group keep what they held (experts, experts_dx), contribute nothing (experts_dw), or have no
adapter (adapters, adapters_dx).
"""
import math

import numpy as np
import torch

own = False

_LARGEST_FLOPS = 2.0 * 32768 * 4096 * 4096


def _case(call, mode, groups, rows, K, M, sizes="skewed", behind=0, rank=0, adapters=0, beta=0.0, inputs="normal"):
    """rows: of all groups together; behind: rows behind the last group; K and M: width of x and of y"""
    return {"call": call, "mode": mode, "groups": groups, "rows": rows, "K": K, "M": M, "sizes": sizes, "behind": behind,
            "rank": rank, "adapters": adapters, "beta": beta, "inputs": inputs}


def listed():
    def named(name, *args, **more):
        return dict(_case(*args, **more), name=name)

    return [
        # one decoding step of eight tokens, two experts each, in a small layer: launches and latency
        named("experts_decode_8x16", "experts", "fp16", 8, 16, 1024, 768),
        # a decoding step of a batch over many experts: each one's weights are read for a row or two
        named("experts_decode_64x128", "experts", "fp16", 64, 128, 2048, 1536),
        # a prompt, or a training batch of ordinary size
        named("experts_8x8192", "experts", "fp16", 8, 8192, 2048, 4096),
        # nothing even about it: odd widths, empty and tiny groups, padding behind the last one, values of any magnitude
        named("experts_ragged_bf16", "experts", "bf16", 37, 3001, 1003, 1309, behind=95, inputs="wide"),
        # the largest batch
        named("experts_32x32768", "experts", "fp16", 32, 32768, 4096, 4096),
        # training: the gradient that goes on to the layer before
        named("experts_dx_16x8192", "experts_dx", "fp16", 16, 8192, 2048, 1408),
        # training: the weights' gradients, from scratch and added to those of the batches before
        named("experts_dw_8x8192", "experts_dw", "fp16", 8, 8192, 2048, 4096),
        named("experts_dw_64x4101_bf16", "experts_dw", "bf16", 64, 4101, 1024, 768, beta=1.0, inputs="wide"),
        # a decoding step of 32 requests, an adapter each, beside a projection
        named("adapters_decode_32", "adapters", "fp16", 32, 32, 4096, 4096, sizes="ones", rank=16, adapters=64),
        # prompts of a few requests, some of them without an adapter
        named("adapters_prompt_4096", "adapters", "fp16", 9, 4096, 4096, 4096, behind=0, rank=32, adapters=6),
        # many short requests, odd sizes, values of any magnitude
        named("adapters_ragged_bf16", "adapters", "bf16", 61, 1031, 1500, 2049, behind=9, rank=20, adapters=16, inputs="wide"),
        # training one adapter for each of four tasks
        named("adapters_dx_6000", "adapters_dx", "fp16", 4, 6000, 2048, 5120, rank=64, adapters=4),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    call = rng.choice(["experts", "experts", "experts_dx", "experts_dw", "adapters", "adapters", "adapters_dx"])
    mode = rng.choice(["fp16", "fp16", "bf16"])
    shared = call.startswith("adapters")
    while True:
        groups, rows = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 32768)
        K, M = _log_uniform(rng, 128, 8192), _log_uniform(rng, 128, 8192)
        if rng.random() < 0.7:      # most layers have round widths
            K, M = (max(128, (v + 32) // 64 * 64) for v in (K, M))
        if 2.0 * rows * K * M <= 0.25 * _LARGEST_FLOPS and (1 if shared else groups) * K * M <= 2 ** 28 and rows * max(K, M) <= 2 ** 27:
            break
    sizes = rng.choice(["skewed", "skewed", "even"])
    if rows <= 64 and rng.random() < 0.5:
        sizes, groups = "ones", rows
        if not shared and groups * K * M > 2 ** 28:
            sizes, groups = "even", 1
    inputs = "normal" if mode == "fp16" else rng.choice(["normal", "wide"])
    return _case(call, mode, groups, rows, K, M, sizes=sizes, behind=rng.choice([0, 0, 3, 64]),
                 rank=rng.choice([4, 8, 16, 16, 32, 48, 64]) if shared else 0, adapters=_log_uniform(rng, 1, 32) if shared else 0,
                 beta=rng.choice([0.0, 1.0]) if call == "experts_dw" else 0.0, inputs=inputs)


def _sizes(case, seed):
    """Rows of each group: what a router or a batch of requests brings."""
    groups, rows = case["groups"], case["rows"]
    random = np.random.RandomState(seed % (1 << 31))
    if case["sizes"] == "ones":
        return np.ones(groups, dtype=np.int64)
    share = np.exp(random.normal(0.0, 0.6, groups)) if case["sizes"] == "skewed" else np.ones(groups)
    at = np.floor(np.cumsum(share) / share.sum() * rows + 0.5).astype(np.int64)
    at[-1] = rows
    return np.diff(np.concatenate([[0], at]))


def _normal(gen, shape, scale, wide):
    """Normal values; `wide`: each row of a magnitude of its own, 2^-60 to 2^20 times the others'."""
    out = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale)
    if wide:
        out *= torch.exp2(torch.randint(-60, 21, (*shape[:-1], 1), generator=gen, device="cuda").float())
    return out


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    call, groups, K, M, rank, count = (case[k] for k in ("call", "groups", "K", "M", "rank", "adapters"))
    total, wide = case["rows"] + case["behind"], case["inputs"] == "wide"
    sizes = _sizes(case, seed)
    s = {"offsets": torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)])).cuda(), "most": max(1, int(sizes.max()))}
    if call != "experts_dw":
        weights = (M, K) if call.startswith("adapters") else (groups, M, K)
        s["W"] = _normal(gen, weights, K ** -0.5, False)
    if not call.endswith("_dx"):
        s["x"] = _normal(gen, (total, K), 1.0, wide)
    if call.endswith("_dx") or call == "experts_dw":
        s["g"] = _normal(gen, (total, M), 0.01, wide and call != "experts_dw")
    if rank:
        s["D"] = _normal(gen, (count, rank, K), K ** -0.5, False)
        s["U"] = _normal(gen, (count, M, rank), 0.5 * rank ** -0.5, False)
        s["scales"] = 0.5 + torch.rand(count, generator=gen, device="cuda")
        # (a request in eight has no adapter)
        random = np.random.RandomState((seed + 1) % (1 << 31))
        index = np.where(random.rand(groups) < 0.125, -1, random.randint(0, count, groups))
        s["index"] = torch.from_numpy(index.astype(np.int32)).cuda()
    if case["beta"]:
        s["before"] = _normal(gen, (groups, M, K), 0.01, False)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    call, K, M, total = case["call"], case["K"], case["M"], case["rows"] + case["behind"]
    out = (case["groups"], M, K) if call == "experts_dw" else (total, K if call.endswith("_dx") else M)
    s["out"] = torch.zeros(out, dtype=torch.float32, device="cuda")
    if case["rank"]:
        s["hidden"] = torch.zeros((total, case["rank"]), dtype=torch.float32, device="cuda")
    s["case"] = case
    return s


# ---- the plain forms

def _padded(s, x):
    """The rows of each group as a matrix of its own, with zeros behind: (groups, most, width)"""
    offsets = s["offsets"]
    at = offsets[:-1, None] + torch.arange(s["most"], device="cuda")
    inside = at < offsets[1:, None]
    return x[at.clamp(max=x.shape[0] - 1)] * inside[:, :, None]


def _rows(s, total):
    """Of every row: its group, its place in it, and whether there is one"""
    offsets, rows = s["offsets"], torch.arange(total, device="cuda")
    inside = (rows >= offsets[0]) & (rows < offsets[-1])
    group = (torch.searchsorted(offsets, rows, right=True) - 1).clamp(0, offsets.numel() - 2)
    place = torch.where(inside, rows - offsets[group], torch.zeros_like(rows))
    return group, place, inside[:, None]


def _plain(s):
    case = s["case"]
    call = case["call"]
    if call == "experts_dw":
        grads = torch.bmm(_padded(s, s["g"]).transpose(1, 2), _padded(s, s["x"]))
        return grads + case["beta"] * s["before"] if case["beta"] else grads
    x = s["g"] if call.endswith("_dx") else s["x"]
    group, place, inside = _rows(s, x.shape[0])
    if not case["rank"]:
        W = s["W"] if call.endswith("_dx") else s["W"].transpose(1, 2)
        return torch.where(inside, torch.bmm(_padded(s, x), W)[group, place], s["out"])
    index = s["index"].long()
    down, up = s["D"][index.clamp(min=0)], s["U"][index.clamp(min=0)]
    if call == "adapters":
        y, down, up = x @ s["W"].t(), down.transpose(1, 2), up.transpose(1, 2)
    else:
        y, down, up = x @ s["W"], up, down
    hidden = torch.bmm(_padded(s, x), down) * (index >= 0)[:, None, None]
    added = torch.bmm(hidden, up) * s["scales"][index.clamp(min=0)][:, None, None]
    zero = torch.zeros((), device="cuda")
    return y + torch.where(inside, added[group, place], zero), torch.where(inside, hidden[group, place], zero)


# ---- the framework's calls

_handles = []


def _handle():
    """The program's one handle, on its stream."""
    import paper_2203_03341_amd as ec
    if not _handles:
        _handles.append(ec.Handle())
        _handles[0].set_stream(torch.cuda.current_stream().cuda_stream)
    return ec, _handles[0]


def _own(s):
    ec, h = _handle()
    case = s["case"]
    call, groups, K, M = case["call"], case["groups"], case["K"], case["M"]
    mode = ec.MODE_FP16_SPLIT if case["mode"] == "fp16" else ec.MODE_BF16_FULL
    total = case["rows"] + case["behind"]
    if call == "experts":
        h.sgemm_grouped(ec.OP_T, ec.OP_N, groups, M, total, K, 1.0, s["W"], K, M * K, s["x"], K, s["offsets"], 0.0, s["out"], M, mode)
    elif call == "experts_dx":
        h.sgemm_grouped(ec.OP_N, ec.OP_N, groups, K, total, M, 1.0, s["W"], K, M * K, s["g"], M, s["offsets"], 0.0, s["out"], K, mode)
    elif call == "experts_dw":
        if case["beta"]:    # the step adds to what the batches before have left
            s["out"].copy_(s["before"])
        h.sgemm_grouped_depth(ec.OP_N, ec.OP_T, groups, K, M, total, 1.0, s["x"], K, s["g"], M, s["offsets"], case["beta"], s["out"], K,
                              M * K, mode)
    else:
        rank, count = case["rank"], case["adapters"]
        if call == "adapters":
            h.sgemm_adapters(ec.OP_T, ec.OP_N, M, total, K, 1.0, s["W"], K, s["x"], K, groups, s["offsets"], s["index"], count, rank,
                             ec.OP_T, s["D"], K, rank * K, ec.OP_T, s["U"], rank, M * rank, s["scales"], s["hidden"], rank, 0.0,
                             s["out"], M, mode)
        else:
            h.sgemm_adapters(ec.OP_N, ec.OP_N, K, total, M, 1.0, s["W"], K, s["g"], M, groups, s["offsets"], s["index"], count, rank,
                             ec.OP_N, s["U"], rank, M * rank, ec.OP_N, s["D"], K, rank * K, s["scales"], s["hidden"], rank, 0.0,
                             s["out"], K, mode)
        return s["out"], s["hidden"]
    return s["out"]


def run(s):
    return _own(s) if own else _plain(s)


def work(case):
    call, groups, rows, K, M, rank = (case[k] for k in ("call", "groups", "rows", "K", "M", "rank"))
    total = rows + case["behind"]
    if not rank:    # what no group holds is neither read nor written; a group without rows needs no weights
        weights = groups if call == "experts_dw" else min(groups, rows)
        return {"bytes": 4.0 * (rows * (K + M) + weights * K * M * (2 if case["beta"] else 1)), "flops": 2.0 * rows * K * M}
    used = min(groups, case["adapters"], rows)
    return {"bytes": 4.0 * (total * (K + M) + K * M + used * rank * (K + M) + total * rank),
            "flops": 2.0 * (total * K * M + rows * rank * (K + M))}


def exact(case, seed):
    """The same in 64 bits, group by group"""
    s = _inputs(case, seed)
    call, K, M, total = case["call"], case["K"], case["M"], case["rows"] + case["behind"]
    at = s["offsets"].tolist()
    runs = [(e, at[e], at[e + 1]) for e in range(case["groups"]) if at[e + 1] > at[e]]
    if call == "experts_dw":
        out = case["beta"] * s["before"].double() if case["beta"] else torch.zeros((case["groups"], M, K), dtype=torch.float64, device="cuda")
        for e, lo, hi in runs:
            out[e] += s["g"][lo:hi].double().t().contiguous() @ s["x"][lo:hi].double()
        return out
    backward = call.endswith("_dx")
    x = s["g"] if backward else s["x"]
    out = torch.zeros((total, K if backward else M), dtype=torch.float64, device="cuda")
    if not case["rank"]:
        for e, lo, hi in runs:
            W = s["W"][e].double()
            out[lo:hi] = x[lo:hi].double() @ (W if backward else W.t().contiguous())
        return out
    W = s["W"].double()
    out += x.double() @ (W if backward else W.t().contiguous())
    hidden = torch.zeros((total, case["rank"]), dtype=torch.float64, device="cuda")
    index = s["index"].tolist()
    for e, lo, hi in runs:
        a = index[e]
        if a >= 0:
            D, U = s["D"][a].double(), s["U"][a].double()
            hidden[lo:hi] = x[lo:hi].double() @ (U if backward else D.t().contiguous())
            out[lo:hi] += float(s["scales"][a]) * (hidden[lo:hi] @ (D if backward else U.t().contiguous()))
    return out, hidden
