"""Operators for many low-rank adapters beside one shared weight, and for the step that follows their gradients.

Three calls are measured.  `ab_adapter_forward` serves many requests at once: every row goes through the dense weight that all share and
through the factor pair of its own adapter.  `ab_adapter_backward` is the training step of the same layer: K groups (or K fine-tunings)
train their own pairs on their own rows beside one frozen weight.  `ab_grad_clip` takes the gradients of all factors of a model, forms
their global norm and scales them; the optimizer step comes behind it.

A row's adapter is its entry of an int32 map; -1 means that the row has the shared weight alone (a request without an adapter, a padded
row).  With a = map[i], s = scale[a]:

    T_i = s B_a x_i        y_i = W x_i + A_a T_i        U_i = s A_a^T dY_i        dX_i = W^T dY_i + B_a^T U_i
    dA_a = sum of dY_i T_i^T,  dB_a = sum of U_i x_i^T  over the rows i with map[i] = a

Sizes are those of this repository's workloads (the small fp32 layer, ViT-B/16 attention at 50,432 rows, widths 776 and 1000) or generic.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_TYPE = {BF16: torch.bfloat16, F32: torch.float32}


def listed():
    return [
        # One request generating: one token through a 4096-wide projection.  Latency: the weight is read once.
        {"name": "adapter_one_token", "op": "forward", "rows": 1, "m": 4096, "n": 4096, "r": 16, "L": 32, "layout": "single",
         "dtype": BF16},
        # 64 requests generating, nearly each with an adapter of its own.
        {"name": "adapter_64_tokens", "op": "forward", "rows": 64, "m": 4096, "n": 4096, "r": 16, "L": 128, "layout": "single",
         "dtype": BF16},
        # A batch in which some requests generate and others bring prompts; odd count of rows, widths of no tile.
        {"name": "adapter_mixed_333", "op": "forward", "rows": 333, "m": 1000, "n": 776, "r": 24, "L": 40, "layout": "mixed",
         "dtype": BF16},
        # Prompts of ragged lengths, wide result.
        {"name": "adapter_prompts_6173", "op": "forward", "rows": 6173, "m": 8192, "n": 2048, "r": 64, "L": 16, "layout": "prompts",
         "dtype": BF16},
        # fp32, sizes that are multiples of nothing.
        {"name": "adapter_prompts_fp32", "op": "forward", "rows": 1531, "m": 1001, "n": 777, "r": 12, "L": 7, "layout": "prompts",
         "dtype": F32},
        # The small fp32 layer, two groups of 64 rows: latency of a training step.
        {"name": "adapter_train_small_fp32", "op": "train", "rows": 128, "m": 256, "n": 512, "r": 32, "L": 2, "layout": "groups",
         "dtype": F32},
        # Four groups training their own factors of a ViT-B/16 attention weight, 64 images of 197 tokens each.
        {"name": "adapter_train_vit_groups", "op": "train", "rows": 50432, "m": 768, "n": 768, "r": 64, "L": 4, "layout": "groups",
         "dtype": BF16},
        # Fine-tunings of a 4096-wide projection side by side, packed sequences of different lengths.
        {"name": "adapter_train_packed", "op": "train", "rows": 8191, "m": 4096, "n": 4096, "r": 16, "L": 8, "layout": "prompts",
         "dtype": BF16},
        # Gradients of one layer's adapters: 16 small tensors, launch-bound.
        {"name": "clip_one_layer", "op": "clip", "tensors": 16, "total": 262144, "dtype": F32},
        # All factors of ViT-B/16 (144 tensors of odd sizes, as a rank rule leaves them), fits L2.
        {"name": "clip_vit_factors", "op": "clip", "tensors": 144, "total": 31850496, "dtype": F32},
        # Gradients in bf16, well beyond L2.
        {"name": "clip_large_bf16", "op": "clip", "tensors": 291, "total": 536870912, "dtype": BF16},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "train", "train", "clip"])
    if kind == "clip":
        total = _log_int(rng, 1000, 200_000_000)
        return {"op": "clip", "tensors": min(total, _log_int(rng, 1, 400)), "total": total, "dtype": rng.choice([F32, F32, BF16])}
    dtype = rng.choice([BF16, BF16, BF16, F32])
    step = 8 if dtype == BF16 and rng.random() < 0.85 else 1
    m, n = (max(step, _log_int(rng, 64, 3900) // step * step) for _ in range(2))
    r = min(rng.choice([4, 8, 8, 12, 16, 16, 24, 32, 48, 64, 72, 128, 136]), m, n)
    most = 8192 if dtype == BF16 and step == 8 else 1024
    return {"op": kind, "rows": _log_int(rng, 1, most), "m": m, "n": n, "r": r, "L": _log_int(rng, 1, 64),
            "layout": rng.choice(["single", "mixed", "prompts", "groups"]), "dtype": dtype}


def _map(case, gen):
    """The adapter of every row, on the host."""
    N, L, layout = case["rows"], case["L"], case["layout"]
    if layout == "groups":                       # L equal runs, every row with an adapter
        return torch.arange(N) * L // N
    ids = torch.randint(0, L, (N,), generator=gen)
    ids[torch.rand(N, generator=gen) < 0.06] = -1
    if layout == "single":                       # a request a row
        return ids
    # runs: between one and three times as many cuts as would make runs of 600 rows; the adapter of a run's first row is the run's
    cuts = torch.randint(0, N, (max(1, N // 300),), generator=gen)
    start = torch.zeros(N, dtype=torch.bool)
    start[cuts] = True
    start[0] = True
    if layout == "mixed":                        # the first quarter are single tokens, the rest prompts
        start[: N // 4 + 1] = True
    first = torch.where(start, torch.arange(N), torch.zeros(N, dtype=torch.long)).cummax(0).values
    return ids[first]


def _sizes(case):
    """Element counts of the clipped tensors: uneven, fixed by the case."""
    k, total = case["tensors"], case["total"]
    share = [1.0 + 0.9 * math.sin(1.7 * i) for i in range(k)]
    size = [max(1, int(total * s / sum(share))) for s in share]
    size[0] = max(1, size[0] + total - sum(size))
    return size


def prepare(case, seed):
    dev, dt = "cuda", _TYPE[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape, std=1.0):
        if dt == torch.float32 or math.prod(shape) < 1 << 28:
            return (torch.randn(*shape, device=dev, generator=g) * std).to(dt)
        return torch.randn(*shape, device=dev, generator=g, dtype=dt).mul_(std)

    if case["op"] == "clip":
        # tensors whose magnitudes differ by orders, as factors' gradients do, behind one another in one arena
        size = _sizes(case)
        arena = randn(sum(size), std=1e-3)
        at, grads, outs, out = 0, [], [], torch.empty_like(arena)
        for i, s in enumerate(size):
            grads.append(arena[at:at + s].mul_(1.0 + (i % 7)))
            outs.append(out[at:at + s])
            at += s
        return {"op": "clip", "grads": grads, "outs": outs, "whole": outs if len(outs) <= 16 else [out],
                "max_norm": 1e-3 * math.sqrt(case["total"])}

    N, m, n, r, L = (case[k] for k in ("rows", "m", "n", "r", "L"))
    host = torch.Generator().manual_seed(seed)
    state = {"op": case["op"], "x": randn(N, n), "W": randn(m, n, std=n ** -0.5), "A": randn(L, m, r, std=0.5 * r ** -0.5),
             "B": randn(L, r, n, std=n ** -0.5), "scale": 0.5 + torch.rand(L, device=dev, generator=g),
             "map": _map(case, host).to(torch.int32).to(dev)}
    if case["op"] == "train":
        state["dY"] = randn(N, m)
    return state


def _run_own(s):
    from paper_2405_01067_b200 import binding as ab
    if s["op"] == "clip":
        if "plan" not in s:                      # a program whose gradients stay where they are keeps their list
            s["plan"] = ab.ClipPlan(s["grads"], out=s["outs"])
        _, norm = ab.ab_grad_clip(s["plan"], s["max_norm"])
        return {"out": s["whole"], "norm": norm}
    if "ws" not in s:                            # and its workspace
        s["ws"] = ab.workspace(ab.ab_adapter_workspace_bytes(s["x"], s["A"], s["B"]), "cuda")
    if s["op"] == "forward":
        y, _ = ab.ab_adapter_forward(s["x"], s["W"], s["A"], s["B"], s["map"], scale=s["scale"], ws=s["ws"])
        return {"y": y}
    y, T = ab.ab_adapter_forward(s["x"], s["W"], s["A"], s["B"], s["map"], scale=s["scale"], save_T=True, ws=s["ws"])
    dX, dA, dB = ab.ab_adapter_backward(s["x"], s["dY"], s["W"], s["A"], s["B"], s["map"], scale=s["scale"], T_saved=T, ws=s["ws"])
    return {"y": y, "dX": dX, "dA": dA, "dB": dB}


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "clip":
        grads, outs = state["grads"], state["outs"]
        # squares in 32 bits, added in 64: the sum runs over up to half a billion of them
        total = torch.stack([(g.float() ** 2).sum(dtype=torch.float64) for g in grads]).sum()
        norm = total.sqrt()
        c = torch.where(norm > state["max_norm"], state["max_norm"] / norm, torch.ones_like(norm)).float()
        [o.copy_(g.float() * c) for g, o in zip(grads, outs)]
        return {"out": state["whole"], "norm": norm.float()}
    x, W, A, B = (state[k].float() for k in ("x", "W", "A", "B"))
    L, m, r = A.shape
    dt, n, ids = state["x"].dtype, x.shape[1], state["map"].long()
    # 1 where the column group of an adapter is the row's own: the rows through all adapters at once, the others' columns set to 0
    mine = (ids[:, None] == torch.arange(L, device=ids.device)).repeat_interleave(r, 1)
    s = state["scale"].repeat_interleave(r)
    B_all, A_all = B.reshape(L * r, n), A.permute(1, 0, 2).reshape(m, L * r)
    T = torch.where(mine, (x @ B_all.T) * s, 0.0)
    y = (x @ W.T + T @ A_all.T).to(dt)
    if state["op"] == "forward":
        return {"y": y}
    dY = state["dY"].float()
    U = torch.where(mine, (dY @ A_all) * s, 0.0)
    dX = (dY @ W + U @ B_all).to(dt)
    dA = (dY.T @ T).reshape(m, L, r).permute(1, 0, 2).contiguous()
    dB = (U.T @ x).reshape(L, r, n)
    return {"y": y, "dX": dX, "dA": dA, "dB": dB}


def _adapters_used(case):
    N, L = case["rows"], case["L"]
    requests = {"groups": L, "single": N, "mixed": N // 4 + max(1, N // 300), "prompts": max(1, N // 300)}[case["layout"]]
    return min(L, requests, N)


def work(case):
    size = 2 if case["dtype"] == BF16 else 4
    if case["op"] == "clip":
        return {"bytes": 2 * size * case["total"], "flops": 3 * case["total"]}
    N, m, n, r, L = (case[k] for k in ("rows", "m", "n", "r", "L"))
    pairs = _adapters_used(case) * r * (m + n)
    if case["op"] == "forward":
        return {"bytes": size * (N * n + m * n + pairs + N * m) + 4 * N, "flops": 2 * N * (m * n + r * (m + n))}
    # x, dY, W, A, B in, y, dX, dA, dB (fp32) out; T once, U once
    return {"bytes": size * (2 * N * (n + m) + m * n + pairs) + 4 * L * r * (m + n) + 4 * N,
            "flops": 2 * N * (2 * m * n + 3 * r * (m + n))}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        chunk = 1 << 26
        base = s["grads"][0]._base
        total = 0.0
        for at in range(0, base.numel(), chunk):
            part = base[at:at + chunk].double()
            total += float(part.dot(part))
        norm = math.sqrt(total)
        c = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
        if base.dtype == torch.float32 and base.numel() <= 1 << 26:
            outs = [g.double() * c for g in s["grads"]] if len(s["grads"]) <= 16 else [base.double() * c]
        else:
            outs = [None]
        return {"out": outs, "norm": torch.tensor(norm, dtype=torch.float64)}
    x, W = s["x"].double(), s["W"].double()
    ids = s["map"].long()
    y = x.mm(W.t())
    train = case["op"] == "train"
    if train:
        dY = s["dY"].double()
        dX = dY.mm(W)
        dA = torch.zeros(s["A"].shape, dtype=torch.float64, device=x.device)
        dB = torch.zeros(s["B"].shape, dtype=torch.float64, device=x.device)
    for a in range(case["L"]):
        rows = torch.nonzero(ids == a).flatten()
        if rows.numel() == 0:
            continue
        Aa, Ba, sa = s["A"][a].double(), s["B"][a].double(), float(s["scale"][a])
        xa = x.index_select(0, rows)
        Ta = sa * xa.mm(Ba.t())
        y.index_add_(0, rows, Ta.mm(Aa.t()))
        if train:
            ga = dY.index_select(0, rows)
            Ua = sa * ga.mm(Aa)
            dX.index_add_(0, rows, Ua.mm(Ba))
            dA[a] = ga.t().mm(Ta)
            dB[a] = Ua.t().mm(xa)
    return {"y": y, "dX": dX, "dA": dA, "dB": dB} if train else {"y": y}
