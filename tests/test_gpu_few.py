"""asap_moe_layer_few (the layer for 1 to 64 tokens) against a float64 layer of
plain torch operations, over gatings, dtypes, expert counts, ragged token counts
and the places where its work is split."""
from dataclasses import replace

import pytest
import torch

from paper_2606_22541_gb300 import _native, api, inputs
from paper_2606_22541_gb300.configs import DSV3, DSV3_FP8, MIXTRAL, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda"

# Output tolerances, normwise per token.  bf16 outputs are rounded once: at most
# 2^-9 = 1.95e-3 of each value.  Everything before is held in 32 bits but for h: as
# two bf16 (2^-17) or, as the format says, e4m3.  The reference quantises as the
# kernel does (fp32 scale and quotient) and x exactly so; an h that lies within its
# fp32 error (some 2e-6 of the group's largest value) of the boundary between two
# e4m3 values may take the other one, an error of at most 1/16 of the value for
# about 2 * 2e-6 / (1/16) of the values: sqrt(6.4e-5) / 16 = 5e-4, four times that
# with margin for a single token.
TOL = {"bf16": 2.1e-3, "fp8_e4m3_block128": 4e-3}

SMALL = dict(hidden=512, inter=256, shared_inter=256)
CONFIGS = [
    TINY,
    inputs.small_variant(DSV3, name="few_ds", **SMALL),
    inputs.small_variant(DSV3_FP8, name="few_f8", zipf_s=None, **SMALL),
    inputs.small_variant(MIXTRAL, name="few_mx", hidden=1024, inter=384),
    # one expert; all experts chosen; an odd count with groups of unequal lane teams; 8 slots of softmax
    replace(TINY, name="few_e1", n_experts=1, top_k=1, hidden=768),
    replace(TINY, name="few_all", n_experts=5, top_k=5, gating="softmax_renorm"),
    replace(DSV3, name="few_g6", n_experts=48, n_groups=6, topk_groups=3, top_k=6, hidden=256, inter=128,
            shared_inter=384, microbatches=[]),
    replace(DSV3_FP8, name="few_g1", n_experts=40, n_groups=1, topk_groups=1, top_k=7, hidden=1280, inter=640,
            shared_inter=128, zipf_s=None, microbatches=[]),
    replace(TINY, name="few_soft", n_experts=200, top_k=8, hidden=1792, inter=128),
]


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def make(cfg, seed=0, bias=True):
    w = inputs.make_weights(replace(cfg, seed=cfg.seed + seed), DEV)
    if bias and cfg.gating == "sigmoid_grouped":
        g = torch.Generator(device=DEV)
        g.manual_seed(77 + seed)
        w["router_bias"] = torch.randn(cfg.n_experts, generator=g, device=DEV) * 0.05
    return w


def tokens(cfg, n, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(1234 + 97 * n + seed)
    return torch.randn((n, cfg.hidden), generator=g, device=DEV).bfloat16()


def quantised(v):
    """As the e4m3 matrices meet activations (fp32 scale and quotient)."""
    b = v.float().reshape(v.shape[0], -1, 128)
    s = b.abs().amax(2, keepdim=True) * torch.tensor(1.0 / 448.0, device=DEV)
    s = torch.where(s > 0, s, torch.ones_like(s))
    return ((b / s).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s.double()).reshape(v.shape)


def dense(w, name, e=None):
    scale = w.get(("s_" if name.startswith("w_") else "sh_s_") + name.split("_")[1])
    v = w[name] if e is None else w[name][e]
    if scale is None:
        return v.double()
    s = scale if e is None else scale[e]
    return v.double() * s.double().repeat_interleave(128, 0).repeat_interleave(128, 1)


def gate64(cfg, logits, bias):
    """(idx, w, decided): decided tokens keep their experts under fp32 logit errors."""
    n, E, k = logits.shape[0], cfg.n_experts, cfg.top_k
    eps = 2e-5

    def kth(v, m):
        s = v.sort(1, descending=True).values
        return torch.full((n,), 1.0, device=DEV) if m >= v.shape[1] else (s[:, m - 1] - s[:, m])

    if cfg.gating == "sigmoid_grouped":
        s = logits.sigmoid()
        sel = s + (0 if bias is None else bias.double())
        g = sel.view(n, cfg.n_groups, -1)
        score = g.topk(2, dim=2).values.sum(2)
        kept = score.topk(cfg.topk_groups, dim=1).indices
        mask = torch.zeros((n, cfg.n_groups), dtype=torch.bool, device=DEV).scatter_(1, kept, True)
        open_ = torch.where(mask[:, :, None], g, torch.full_like(g, -9.0)).reshape(n, E)
        idx = open_.topk(k, dim=1).indices
        w = s.gather(1, idx)
        decided = (kth(score, cfg.topk_groups) > eps) & (kth(open_, k) > eps)
        return idx, w / w.sum(1, keepdim=True) * cfg.route_scale, decided
    idx = logits.topk(k, dim=1).indices
    p = logits.softmax(1).gather(1, idx)
    if cfg.gating == "softmax_renorm":
        p = p / p.sum(1, keepdim=True)
    return idx, p, kth(logits, k) > eps


def layer64(cfg, w, x):
    fp8 = cfg.dtype != "bf16"
    idx, p, decided = gate64(cfg, x.double() @ w["router_w"].double().t(), w.get("router_bias"))
    xq = quantised(x) if fp8 else x.double()

    def ffn(rows, pre, e=None):
        g, u = rows @ dense(w, pre + "gate", e).t(), rows @ dense(w, pre + "up", e).t()
        h = g * g.sigmoid() * u
        return (quantised(h) if fp8 else h) @ dense(w, pre + "down", e).t()

    out = torch.zeros((x.shape[0], cfg.hidden), dtype=torch.float64, device=DEV)
    for e in idx.unique().tolist():
        t, j = (idx == e).nonzero(as_tuple=True)
        out[t] += p[t, j, None] * ffn(xq[t], "w_", e)
    if cfg.n_shared:
        out += ffn(xq, "sh_")
    return out, decided


def check(cfg, got, ref, decided):
    err = (got.double() - ref).norm(dim=1) / ref.norm(dim=1)
    assert decided.float().mean() > 0.5
    worst = float(err[decided].max())
    assert worst <= TOL[cfg.dtype], worst


def few(h, x, **kw):
    out = torch.full_like(x, 7.0)
    ws = api.workspace(h, x.shape[0])
    ws.fill_(0xFF)  # what the workspace held does not matter
    api.asap_moe_layer_few(h, x, out, ws, **kw)
    return out


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
def test_layer_against_float64(cfg):
    w = make(cfg)
    h = api.asap_moe_create(cfg, w, 64)
    for n in (1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 33, 48, 63, 64):
        x = tokens(cfg, n)
        ref, decided = layer64(cfg, w, x)
        check(cfg, few(h, x), ref, decided)
        assert api.asap_moe_status(h) == (0, 0)
    h.close()


@pytest.mark.parametrize("cfg", [MIXTRAL, replace(DSV3, name="few_big"), replace(DSV3_FP8, name="few_big8", zipf_s=None)],
                         ids=lambda c: c.name)
@pytest.mark.parametrize("n", [1, 6, 64])
def test_full_width_layers(cfg, n):
    """Full hidden and intermediate sizes (many K slices and tiles); 16 experts keep the reference small."""
    cfg = replace(cfg, n_experts=min(cfg.n_experts, 16), topk_groups=min(cfg.topk_groups, 4))
    w = make(cfg, seed=n)
    h = api.asap_moe_create(cfg, w, 64)
    x = tokens(cfg, n)
    ref, decided = layer64(cfg, w, x)
    check(cfg, few(h, x), ref, decided)
    assert api.asap_moe_status(h) == (0, 0)
    h.close()


@pytest.mark.parametrize("cfg", CONFIGS[1:3], ids=lambda c: c.name)
def test_tokens_that_share_every_expert(cfg):
    """64 rows in each of the chosen experts: the widest operand."""
    w = make(cfg)
    h = api.asap_moe_create(cfg, w, 64)
    x = tokens(cfg, 1).expand(64, -1).contiguous()
    ref, decided = layer64(cfg, w, x)
    got = few(h, x)
    check(cfg, got, ref, decided)
    assert torch.equal(got, got[:1].expand_as(got))
    h.close()


@pytest.mark.parametrize("cfg", CONFIGS[:4], ids=lambda c: c.name)
def test_the_same_call_gives_the_same_bits(cfg):
    h = api.asap_moe_create(cfg, make(cfg), 64)
    for n in (1, 5, 24, 64):
        x = tokens(cfg, n)
        first = few(h, x)
        for _ in range(5):
            assert torch.equal(first, few(h, x))
    h.close()


def test_ties_go_to_the_lower_expert():
    """Two pairs of identical rows in the router: each time the lower index is taken."""
    cfg = replace(TINY, name="few_tie", n_experts=64, top_k=3)
    w = make(cfg)
    w["router_w"][40] = w["router_w"][3]
    w["router_w"][63] = w["router_w"][9]
    w["router_w"][9] *= 3  # (so that they are chosen for about half of the tokens)
    w["router_w"][63] = w["router_w"][9]
    h = api.asap_moe_create(cfg, w, 64)
    x = tokens(cfg, 64)
    logits = x.double() @ w["router_w"].double().t()
    order = logits.sort(dim=1, descending=True, stable=True).indices[:, :3]
    # tokens whose third and fourth logits are the tied pair
    tied = [t for t in range(64) if order[t, 2] in (3, 9)
            and logits[t].sort(descending=True).values[3] == logits[t, order[t, 2]]]
    assert len(tied) >= 3
    p = logits.softmax(1).gather(1, order)
    ref = torch.zeros((64, cfg.hidden), dtype=torch.float64, device=DEV)
    for j in range(3):
        for e in order[:, j].unique().tolist():
            t = (order[:, j] == e).nonzero()[:, 0]
            g, u = x[t].double() @ w["w_gate"][e].double().t(), x[t].double() @ w["w_up"][e].double().t()
            ref[t] += p[t, j, None] * ((g * g.sigmoid() * u) @ w["w_down"][e].double().t())
    got = few(h, x).double()
    err = (got[tied] - ref[tied]).norm(dim=1) / ref[tied].norm(dim=1)
    assert float(err.max()) <= TOL["bf16"]
    h.close()


def test_layers_by_device_id():
    cfg = CONFIGS[2]
    ws = [make(cfg, seed=s) for s in range(3)]
    h = api.asap_moe_create_layers(cfg, ws, 64)
    x = tokens(cfg, 12)
    layer = torch.zeros(1, dtype=torch.int32, device=DEV)
    for l in (2, 0, 1):
        layer.fill_(l)
        ref, decided = layer64(cfg, ws[l], x)
        check(cfg, few(h, x, layer_id=layer), ref, decided)
    assert api.asap_moe_status(h) == (0, 0)
    # an id outside the table is recorded, and layer 0 used
    layer.fill_(3)
    assert torch.equal(few(h, x, layer_id=layer), few(h, x))
    assert api.asap_moe_status(h) == (_native.ASAP_ERR_DEVICE_STATUS, 16)
    # calls of different layers enqueued before any has run
    outs = []
    for l in (1, 2, 0, 2):
        layer.fill_(l)
        outs.append((l, few(h, x, layer_id=layer)))
    for l, out in outs:
        layer.fill_(l)
        assert torch.equal(out, few(h, x, layer_id=layer))
    h.close()


def test_a_token_that_is_no_number_stays_alone():
    """NaN and infinite hidden states reach their own output row only."""
    for cfg in CONFIGS[1:3]:
        h = api.asap_moe_create(cfg, make(cfg), 64)
        x = tokens(cfg, 20)
        clean = few(h, x)
        x2 = x.clone()
        x2[3, 5] = float("nan")
        x2[11, 100] = float("inf")
        got = few(h, x2)
        keep = [t for t in range(20) if t not in (3, 11)]
        assert torch.equal(got[keep], clean[keep])
        assert got[3].isnan().all() and not got[11].isfinite().all()
        h.close()


@pytest.mark.parametrize("cfg", CONFIGS[1:3], ids=lambda c: c.name)
def test_calls_back_to_back_on_one_workspace_and_beside_the_prompt_path(cfg):
    """No synchronisation between calls of other sizes, and layer calls in between on the same stream."""
    h = api.asap_moe_create(cfg, make(cfg), 300)
    sizes = [1, 64, 9, 300, 3, 17, 1, 300, 40, 8]
    xs = [tokens(cfg, n, seed=i) for i, n in enumerate(sizes)]
    ws = api.workspace(h, 300)
    big = torch.empty(max(ws.numel(), api.workspace(h, 64).numel()), dtype=torch.uint8, device=DEV)

    def run(x, space):
        out = torch.full_like(x, 7.0)
        if x.shape[0] > 64:
            api.asap_moe_layer(h, x, out, space)
        else:
            api.asap_moe_layer_few(h, x, out, space)
        return out

    want = []
    for x in xs:
        want.append(run(x, torch.empty_like(big)))
        torch.cuda.synchronize()
    for _ in range(3):
        got = [run(x, big) for x in xs]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert api.asap_moe_status(h) == (0, 0)
    h.close()


def test_streams_and_graph():
    cfg = CONFIGS[2]
    h = api.asap_moe_create(cfg, make(cfg), 64)
    xs = [tokens(cfg, n, seed=n) for n in (1, 5, 33, 64)]
    want = [few(h, x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [[torch.full_like(x, 7.0) for x in xs] for _ in range(8)]
    spaces = [api.workspace(h, x.shape[0]) for x in xs]
    torch.cuda.synchronize()
    for round_ in outs:  # calls of four streams side by side
        for x, out, ws, s in zip(xs, round_, spaces, streams):
            api.asap_moe_layer_few(h, x, out, ws, stream=s)
    torch.cuda.synchronize()
    for round_ in outs:
        for out, ref in zip(round_, want):
            assert torch.equal(out, ref)
    out = torch.empty_like(xs[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            api.asap_moe_layer_few(h, xs[2], out, spaces[2])
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[2])
    assert api.asap_moe_status(h) == (0, 0)
    h.close()


def test_refusals():
    cfg = TINY
    h = api.asap_moe_create(cfg, make(cfg), 100)
    x = tokens(cfg, 64)
    out = torch.full_like(x, 7.0)
    ws = api.workspace(h, 64)

    def code(x, out, ws, **kw):
        with pytest.raises(_native.AsapError) as e:
            api.asap_moe_layer_few(h, x, out, ws, **kw)
        return e.value.code

    big = tokens(cfg, 65)
    assert code(big, torch.empty_like(big), api.workspace(h, 65)) == _native.ASAP_ERR_INVALID
    assert code(x, out, ws[:ws.numel() - 256]) == _native.ASAP_ERR_WORKSPACE
    assert code(x, out, None) == _native.ASAP_ERR_WORKSPACE
    assert code(x, out, ws[1:]) == _native.ASAP_ERR_INVALID
    flat = torch.empty(64 * cfg.hidden + 8, dtype=torch.bfloat16, device=DEV)
    assert code(flat[1:1 + 64 * cfg.hidden].view(64, -1), out, ws) == _native.ASAP_ERR_INVALID
    assert code(x, flat[4:4 + 64 * cfg.hidden].view(64, -1), ws) == _native.ASAP_ERR_INVALID
    ids = torch.zeros(16, dtype=torch.uint8, device=DEV)
    assert code(x, out, ws, layer_id=ids[2:]) == _native.ASAP_ERR_INVALID
    torch.cuda.synchronize()
    assert (out == 7.0).all() and api.asap_moe_status(h) == (0, 0)
    api.asap_moe_layer_few(h, x[:0], out[:0], None)  # no tokens: nothing to do
    h.close()
    small = api.asap_moe_create(cfg, make(cfg), 5)  # max_tokens bounds the call too
    with pytest.raises(_native.AsapError):
        api.asap_moe_layer_few(small, x[:6], out[:6], ws)
    small.close()
