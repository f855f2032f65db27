"""Performance cases of the operators around the expert products of a training
step: tokens sorted by expert and back, with the gradients of both, and SwiGLU
whose activations are kept for the backward pass in e4m3 (a scale per row and
128 columns).

``listed`` holds the standing cases, ``draw`` makes more of the same ranges,
``prepare`` builds what a training program holds before the call, ``run`` makes
one pass, ``work`` counts the bytes and operations that the pass cannot do
without and ``exact`` gives its outputs in float64.  With ``own`` false ``run``
computes the operators from elementary torch operations in 32 bits.

Operators (``op``):
  sort       asap_moe_sort and asap_moe_permute: the place of every (token, slot)
             in its expert's segment, and the tokens' rows copied to their places
  back       asap_moe_unpermute: sums of the experts' rows, token by token, with
             weights, or without (the gradient of the rows that were copied)
  back_grad  asap_moe_unpermute_backward: the gradients of rows and weights
  save       asap_moe_swiglu_save: silu(gate) * up, with gate and up kept in e4m3
  save_grad  asap_moe_swiglu_backward: gradients from what was kept, and the
             activations again for the next product's weight gradient
  restore    asap_moe_fp8_dequantize: e4m3 rows of the tokens back as rows of the experts

``drop`` is the share of entries that no expert takes (index -1): padding tokens,
whose slots are all without an expert, and single slots.
"""
import math

import torch

own = False

DEV = "cuda"
BLK = 128
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a handful of tokens of a wide layer with 256 experts: launches and latency
        dict(name="sort_8", op="sort", n=8, k=8, experts=256, cols=7168, type="bf16", drop=0.0),
        # the longest micro-batch of the skewed workload
        dict(name="sort_8045", op="sort", n=8045, k=8, experts=256, cols=7168, type="bf16", drop=0.0),
        # few wide experts, two per token, in fp16; some padding tokens
        dict(name="back_fp16_3584", op="back", n=3584, k=2, experts=8, cols=4096, type="fp16", drop=0.1, weights=True),
        # the gradient of a micro-batch's rows: plain sums over its eight experts
        dict(name="back_sum_5185", op="back", n=5185, k=8, experts=256, cols=7168, type="bf16", drop=0.0, weights=False),
        # a small layer in fp32, as gradients are checked in
        dict(name="back_grad_fp32_160", op="back_grad", n=160, k=2, experts=8, cols=256, type="fp32", drop=0.1),
        # the benchmark's micro-batch
        dict(name="back_grad_4096", op="back_grad", n=4096, k=8, experts=256, cols=7168, type="bf16", drop=0.0),
        # the rows of a few tokens
        dict(name="save_64", op="save", n=64, cols=2048, type="bf16", drop=0.0),
        # the benchmark's micro-batch times eight experts
        dict(name="save_32768", op="save", n=32768, cols=2048, type="bf16", drop=0.0),
        # rows of wide experts, an odd count of which a part is filled
        dict(name="save_grad_2217", op="save_grad", n=2217, cols=14336, type="bf16", drop=0.1),
        dict(name="save_grad_32768", op="save_grad", n=32768, cols=2048, type="bf16", drop=0.0),
        # tokens kept in e4m3, as the rows that the first product's weight gradient reads: odd widths, and the benchmark's
        dict(name="restore_odd_1179", op="restore", n=1179, k=2, experts=8, cols=2052, type="fp16", drop=0.1),
        dict(name="restore_4096", op="restore", n=4096, k=8, experts=256, cols=7168, type="bf16", drop=0.0),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sort", "back", "back_grad", "save", "save_grad", "restore"])
    case = dict(op=op, type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), drop=rng.choice([0.0, 0.0, 0.1, 0.3]))
    kind = rng.random()  # widths: of layers, even ones, any
    if op in ("save", "save_grad"):
        cols, n = _log_uniform(rng, 64, 14336), _log_uniform(rng, 1, 65536)
        most = 32768 * 2048
    else:
        cols, n = _log_uniform(rng, 64, 7168), _log_uniform(rng, 1, 32768)
        case["experts"] = rng.choice([8, 16, 60, 64, 128, 256])
        case["k"] = rng.randint(1, 8)
        # (rows read and written, as the largest listed case has them)
        most = 4096 * 7168 * 17 // (2 * case["k"] + 1)
    cols = (cols + 127) // 128 * 128 if kind < 0.5 else (cols + 7) // 8 * 8 if kind < 0.8 else cols
    if case["type"] == "fp32":
        most //= 2
    case.update(cols=cols, n=max(1, min(n, most // cols)))
    if op == "back":
        case["weights"] = rng.random() < 0.7
    return case


# ------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1013 + stream)
    return g


def _randn(shape, seed, stream, std=1.0):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV).mul_(std)


def _blocks(c):
    return (c + BLK - 1) // BLK


def _experts(case, seed):
    """[n, k] int32: experts of skewed popularity, each once in a row at most, -1 where none takes the entry."""
    n, k, E = case["n"], case["k"], case["experts"]
    popular = torch.randperm(E, generator=_gen(seed, 1), device=DEV).float().add_(1.0).log_().mul_(-0.6)
    idx = torch.sort(_randn((n, E), seed, 2) + popular, dim=1, descending=True, stable=True).indices[:, :k]
    pad = int(n * case["drop"] / 2)  # whole tokens, at the end
    slots = torch.rand((n, k), generator=_gen(seed, 3), device=DEV) < case["drop"] / 2
    slots[n - pad:] = True
    return torch.where(slots, torch.full_like(idx, -1), idx).to(torch.int32)


def _places(idx, experts):
    """(offsets [E + 1], places [n, k], entries by place [n k]) of entries sorted by expert; -1 where there is none."""
    e = idx.flatten().long()
    e = torch.where((e >= 0) & (e < experts), e, torch.full_like(e, experts))
    e, order = torch.sort(e, stable=True)
    at = torch.arange(e.numel(), device=e.device)
    place = torch.empty_like(at)
    place[order] = torch.where(e < experts, at, torch.full_like(at, -1))
    offsets = (e[None, :] < torch.arange(experts + 1, device=e.device)[:, None]).sum(1)
    return offsets.to(torch.int32), place.view(idx.shape).to(torch.int32), order


def _encode(v):
    """fp32 [r, c] to (e4m3 [r, c], scales [r, ceil(c / 128)])."""
    r, c = v.shape
    p = torch.nn.functional.pad(v, (0, _blocks(c) * BLK - c)).view(r, -1, BLK)
    amax = p.abs().amax(dim=2)
    s = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return (p / s[:, :, None]).clamp(-448.0, 448.0).to(F8).view(r, -1)[:, :c], s


def _rows(shape, seed, stream, kind):
    """Activations, a few channels of them much larger than the others."""
    x = _randn(shape, seed, stream)
    x *= torch.exp(_randn((1, shape[1]), seed, stream + 1))
    return x.to(kind)


def _filled(case):
    return case["n"] - int(case["n"] * case["drop"])


def prepare(case, seed):
    op, n, c, kind = case["op"], case["n"], case["cols"], TYPES[case["type"]]
    st = dict(op=op, type=kind)
    if op in ("save", "save_grad"):
        y = _rows((n, 2 * c), seed, 11, kind)  # gate and up, as one product leaves them
        q, s = torch.zeros((n, 2 * c), dtype=F8, device=DEV), torch.zeros((n, 2 * _blocks(c)), device=DEV)
        # where the segments end, as the sort leaves it on the device; the rows behind are not filled
        st.update(cols=c, n_rows=torch.full((1,), _filled(case), dtype=torch.int32, device=DEV), q=q, s=s,
                  h=torch.zeros((n, c), dtype=kind, device=DEV))
        if op == "save":
            st["y"] = y
        else:
            for half, at in ((0, 0), (c, _blocks(c))):
                q[:, half:half + c], s[:, at:at + _blocks(c)] = _encode(y[:, half:half + c].float())
            st.update(d_h=_randn((n, c), seed, 15, 0.05).to(kind), d_y=torch.zeros((n, 2 * c), dtype=kind, device=DEV))
        return st
    k, E = case["k"], case["experts"]
    idx = _experts(case, seed)
    st.update(experts=E, idx=idx, offsets=torch.zeros(E + 1, dtype=torch.int32, device=DEV),
              perm=torch.zeros((n, k), dtype=torch.int32, device=DEV))
    if op == "sort":
        st["x"] = _rows((n, c), seed, 21, kind)
        st["x_perm"] = torch.zeros((n * k, c), dtype=kind, device=DEV)
        # (more than asap_moe_sort_workspace_size of up to 256 experts asks for)
        st["ws"] = torch.zeros(max(256, 8 * n * k + 16384 * (n * k // 1024 + 1)), dtype=torch.uint8, device=DEV)
        return st
    st["perm"] = _places(idx, E)[1]
    if op == "restore":
        st["q"], st["s"] = _encode(_rows((n, c), seed, 31, kind).float())
        st["x_perm"] = torch.zeros((n * k, c), dtype=kind, device=DEV)
        return st
    w = torch.rand((n, k), generator=_gen(seed, 41), device=DEV) + 0.1
    st["w"] = w.div_(w.sum(1, keepdim=True)).mul_(2.5) if case.get("weights", True) else None
    st["y"] = _randn((n * k, c), seed, 42).to(kind)
    if op == "back":
        st["out"] = torch.zeros((n, c), dtype=kind, device=DEV)
    else:
        st.update(d_out=_randn((n, c), seed, 43, 0.05).to(kind), d_y=torch.zeros((n * k, c), dtype=kind, device=DEV),
                  d_w=torch.zeros((n, k), device=DEV))
    return st


# ------------------------------------------------------------------ the calls

def run(st):
    op = st["op"]
    if not own:
        return {"sort": _sort32, "back": _back32, "back_grad": _back_grad32, "save": _save32, "save_grad": _save_grad32,
                "restore": _restore32}[op](st)
    from paper_2606_22541_gb300 import api
    if op == "sort":
        api.asap_moe_sort(st["idx"], st["experts"], st["offsets"], st["perm"], st["ws"])
        api.asap_moe_permute(st["x"], st["perm"], st["x_perm"])
        return [st["offsets"], st["perm"], st["x_perm"]]
    if op == "back":
        api.asap_moe_unpermute(st["y"], st["w"], st["perm"], st["out"])
        return st["out"]
    if op == "back_grad":
        api.asap_moe_unpermute_backward(st["d_out"], st["y"], st["w"], st["perm"], st["d_y"], st["d_w"])
        return [st["d_y"], st["d_w"]]
    if op == "restore":
        api.asap_moe_fp8_dequantize(st["q"], st["s"], st["x_perm"], st["perm"])
        return st["x_perm"]
    c, b = st["cols"], st["s"].shape[1] // 2
    kept = (st["q"][:, :c], st["s"][:, :b], st["q"][:, c:], st["s"][:, b:])
    if op == "save":
        api.asap_moe_swiglu_save(st["y"][:, :c], st["y"][:, c:], st["h"], *kept, n_rows=st["n_rows"])
        return [st["h"], st["q"], st["s"]]
    api.asap_moe_swiglu_backward(st["d_h"], *kept, st["d_y"][:, :c], st["d_y"][:, c:], st["h"], n_rows=st["n_rows"])
    return [st["d_y"], st["h"]]


# ------------------------------------------------------------------ plain forms, 32 bits

def _sort32(st):
    offsets, perm, order = _places(st["idx"], st["experts"])
    taken = torch.arange(order.numel(), device=order.device) < offsets[-1]
    rows = st["x"][torch.div(order, perm.shape[1], rounding_mode="floor")]
    return [offsets, perm, torch.where(taken[:, None], rows, torch.zeros_like(rows))]


def _gathered32(y, perm):
    """[n, k, c] fp32: the rows of each token, zeros where it has none."""
    rows = y[perm.clamp(min=0).long()].float()
    return torch.where((perm >= 0)[:, :, None], rows, torch.zeros_like(rows))


def _back32(st):
    rows = _gathered32(st["y"], st["perm"])
    if st["w"] is not None:
        rows = rows * st["w"][:, :, None]
    return rows.sum(1).to(st["type"])


def _scattered32(rows, perm, like):
    """[n, k, c] rows at their places in a tensor like ``like``, zeros elsewhere."""
    out = torch.zeros((like.shape[0] + 1, like.shape[1]), dtype=like.dtype, device=like.device)
    out[torch.where(perm >= 0, perm, torch.full_like(perm, like.shape[0])).long()] = rows.to(like.dtype)
    return out[:-1]


def _back_grad32(st):
    d_out, perm = st["d_out"].float(), st["perm"]
    d_w = (_gathered32(st["y"], perm) * d_out[:, None, :]).sum(2)
    return [_scattered32(d_out[:, None, :] * st["w"][:, :, None], perm, st["d_y"]), d_w]


def _filled32(st, v):
    """v with zeros in the rows that are not filled."""
    rows = torch.arange(v.shape[0], device=v.device) < st["n_rows"]
    return torch.where(rows[:, None], v, torch.zeros_like(v))


def _save32(st):
    c = st["cols"]
    g, u = st["y"][:, :c].float(), st["y"][:, c:].float()
    h = g / (1.0 + torch.exp(-g)) * u
    gq, gs = _encode(_filled32(st, g))
    uq, us = _encode(_filled32(st, u))
    return [_filled32(st, h).to(st["type"]), torch.cat([gq.view(torch.uint8), uq.view(torch.uint8)], 1).view(F8),
            _filled32(st, torch.cat([gs, us], 1))]


def _decode32(q, s):
    return q.float() * s.repeat_interleave(BLK, 1)[:, :q.shape[1]]


def _save_grad32(st):
    c, b = st["cols"], st["s"].shape[1] // 2
    g, u = _decode32(st["q"][:, :c], st["s"][:, :b]), _decode32(st["q"][:, c:], st["s"][:, b:])
    d, p = st["d_h"].float(), 1.0 / (1.0 + torch.exp(-g))
    d_y = torch.cat([d * u * p * (1.0 + g * (1.0 - p)), d * g * p], 1)
    return [_filled32(st, d_y).to(st["type"]), _filled32(st, g * p * u).to(st["type"])]


def _restore32(st):
    rows = _decode32(st["q"], st["s"])
    return _scattered32(rows[:, None, :].expand(-1, st["perm"].shape[1], -1), st["perm"], st["x_perm"])


# ------------------------------------------------------------------ work

def work(case):
    op, n, c = case["op"], case["n"], case["cols"]
    b = 4 if case["type"] == "fp32" else 2
    if op in ("save", "save_grad"):
        r = _filled(case)
        kept = 2 * c + 8 * _blocks(c)  # e4m3 and scales
        if op == "save":
            return dict(bytes=r * (3 * b * c + kept), flops=12 * r * c)
        return dict(bytes=r * (4 * b * c + kept), flops=16 * r * c)
    m = n * case["k"]
    pad = int(n * case["drop"] / 2)
    rows = int((m - pad * case["k"]) * (1.0 - case["drop"] / 2))  # entries that an expert takes
    tokens = n - pad
    if op == "sort":
        return dict(bytes=8 * m + 4 * (case["experts"] + 1) + (tokens + rows) * c * b, flops=0)
    if op == "back":
        return dict(bytes=(8 if case["weights"] else 4) * m + (n + rows) * c * b, flops=2 * rows * c)
    if op == "back_grad":
        return dict(bytes=12 * m + (tokens + 2 * rows) * c * b, flops=3 * rows * c)
    return dict(bytes=4 * m + tokens * (c + 4 * _blocks(c)) + rows * c * b, flops=rows * c)


# ------------------------------------------------------------------ 64 bits

def _order64(idx, experts):
    """(entries that an expert takes in the order of their places, how many each expert has)."""
    flat = idx.reshape(-1).to(torch.int64)
    taken = torch.nonzero((flat >= 0) & (flat < experts)).reshape(-1)
    key = flat[taken] * flat.numel() + taken
    return taken[torch.argsort(key)], torch.bincount(flat[taken], minlength=experts)


def exact(case, seed):
    st = prepare(case, seed)
    op, c = case["op"], case["cols"]
    if op in ("save", "save_grad"):
        r, b = int(st["n_rows"].item()), _blocks(c)
        h = torch.zeros((case["n"], c), dtype=torch.float64, device=DEV)
        if op == "save":
            q = torch.zeros((case["n"], 2 * c), dtype=torch.float64, device=DEV)
            s = torch.zeros((case["n"], 2 * b), dtype=torch.float64, device=DEV)
            y = st["y"][:r].double()
            h[:r] = torch.nn.functional.silu(y[:, :c]) * y[:, c:]
            wide = torch.zeros((r, 2, b * BLK), dtype=torch.float64, device=DEV)
            wide[:, :, :c] = y.view(r, 2, c)
            wide = wide.view(r, 2, b, BLK)
            top = wide.abs().max(dim=3, keepdim=True).values
            sc = torch.where(top == 0, torch.ones_like(top), top / 448)
            q[:r] = (wide / sc).clamp(-448, 448).float().to(F8).double().view(r, 2, -1)[:, :, :c].reshape(r, 2 * c)
            s[:r] = sc.reshape(r, 2 * b)
            return [h, q, s]
        column = torch.arange(c, device=DEV) // BLK
        v = st["q"][:r].to(torch.float32).double()
        g, u = v[:, :c] * st["s"][:r, column].double(), v[:, c:] * st["s"][:r, column + b].double()
        d, p = st["d_h"][:r].double(), torch.sigmoid(g)
        d_y = torch.zeros((case["n"], 2 * c), dtype=torch.float64, device=DEV)
        d_y[:r, :c] = d * u * (p + g * p * (1 - p))
        d_y[:r, c:] = d * torch.nn.functional.silu(g)
        h[:r] = torch.nn.functional.silu(g) * u
        return [d_y, h]
    k, n = case["k"], case["n"]
    entries, count = _order64(st["idx"], case["experts"])
    token = entries // k
    m = entries.numel()
    if op == "sort":
        perm = torch.full((n * k,), -1, dtype=torch.int32, device=DEV)
        perm[entries] = torch.arange(m, dtype=torch.int32, device=DEV)
        offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).to(torch.int32)
        x_perm = torch.zeros((n * k, c), dtype=torch.float64, device=DEV)
        x_perm[:m] = st["x"][token].double()
        return [offsets, perm.view(n, k), x_perm]
    if op == "restore":
        x_perm = torch.zeros((n * k, c), dtype=torch.float64, device=DEV)
        column = torch.arange(c, device=DEV) // BLK
        x_perm[:m] = (st["q"].to(torch.float32).double() * st["s"][:, column].double())[token]
        return x_perm
    y = st["y"][:m].double()
    w = torch.ones(m, dtype=torch.float64, device=DEV) if st["w"] is None else st["w"].reshape(-1)[entries].double()
    if op == "back":
        return torch.zeros((n, c), dtype=torch.float64, device=DEV).index_add_(0, token, y * w[:, None])
    d_y = torch.zeros((n * k, c), dtype=torch.float64, device=DEV)
    d = st["d_out"].double()[token]
    d_y[:m] = d * w[:, None]
    d_w = torch.zeros(n * k, dtype=torch.float64, device=DEV)
    d_w[entries] = (d * y).sum(1)
    return [d_y, d_w.view(n, k)]
