"""Tokens sorted by expert and back on plain tensors, with the gradients: against
plain implementations in 64 bits.

Tolerances (u = 2^-24, half a step of fp32; e = finfo(type).eps / 2, half a step of
the type): a sum of m fp32 terms in any order is within m u sum |term| of its
value, each product within u; the result is rounded once, e |value| (or half of
the smallest subnormal step of the type)."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import _native, api

pytestmark = pytest.mark.gpu
DEV, F8 = "cuda", torch.float8_e4m3fn
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SUBNORMAL = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=gen(seed), device=DEV).to(dtype)


def strided(rows, cols, pad, offset, dtype, fill):
    """(flat, a [rows, cols] view of it): row stride cols + pad, ``offset`` elements in."""
    ld = cols + pad
    flat = torch.full((rows * ld + offset + 32,), fill, device=DEV).to(dtype)
    return flat, flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def experts(n, k, E, seed, drop=0.0):
    """[n, k] int32: distinct experts per token where k allows it, some entries outside [0, E)."""
    g = gen(seed)
    if k <= E:
        idx = torch.rand((n, E), generator=g, device=DEV).topk(k, dim=1).indices
    else:
        idx = torch.randint(0, E, (n, k), generator=g, device=DEV)
    out = torch.rand((n, k), generator=g, device=DEV) < drop
    bad = torch.randint(0, 4, (n, k), generator=g, device=DEV)
    wrong = torch.tensor([-1, E, -2 ** 31, 2 ** 31 - 1], device=DEV)[bad]
    return torch.where(out, wrong, idx).to(torch.int32)


def sort_plain(idx, E):
    """(offsets, perm_dst, perm_src of the places taken) by a plain walk."""
    flat = idx.flatten().tolist()
    k = idx.shape[1]
    segments = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            segments[e].append(i)
    offsets, perm, src = [0], [-1] * len(flat), []
    for seg in segments:
        for i in seg:
            perm[i] = len(src)
            src.append(i // k)
        offsets.append(len(src))
    t = lambda v: torch.tensor(v, dtype=torch.int32)
    return t(offsets), t(perm).view(idx.shape), t(src)


def sort(idx, E, src=False):
    n, k = idx.shape
    off = torch.full((E + 1,), -9, dtype=torch.int32, device=DEV)
    perm = torch.full((n, k), -9, dtype=torch.int32, device=DEV)
    ps = torch.full((n * k,), -9, dtype=torch.int32, device=DEV) if src else None
    api.asap_moe_sort(idx, E, off, perm, api.sort_workspace(n, k, E), ps)
    return off, perm, ps


# ------------------------------------------------------------------ sort

@pytest.mark.parametrize("n,k,E", [
    (1, 1, 1), (1, 8, 256), (3, 2, 8), (8, 8, 256), (31, 1, 2), (33, 3, 7), (512, 8, 256), (513, 8, 256), (4096, 1, 1),
    (4097, 1, 1), (1000, 17, 60), (700, 8, 1024), (5000, 8, 1024), (8045, 8, 256), (2000, 33, 1000), (16384, 8, 64),
    (40000, 2, 8), (66000, 4, 128), (300, 64, 5)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_sort(n, k, E, drop):
    idx = experts(n, k, E, n + k, drop)
    off, perm, src = sort(idx, E, src=True)
    ro, rp, rs = sort_plain(idx, E)
    assert torch.equal(off.cpu(), ro) and torch.equal(perm.cpu(), rp)
    taken = int(ro[-1])
    assert torch.equal(src[:taken].cpu(), rs) and (src[taken:] == -9).all()


def test_sort_of_one_million_tokens():
    n, k, E = 1 << 20, 8, 256
    idx = experts(n, k, E, 3, 0.05)
    off, perm, src = sort(idx, E, src=True)
    key = torch.where((idx >= 0) & (idx < E), idx, E).flatten().long()
    order = torch.sort(key, stable=True).indices
    taken = int(off[-1])
    count = torch.bincount(key, minlength=E + 1)[:E]
    assert taken == int(count.sum()) and torch.equal(off[1:].long(), count.cumsum(0))
    assert torch.equal(perm.flatten()[order[:taken]].long(), torch.arange(taken, device=DEV))
    assert (perm.flatten()[order[taken:]] == -1).all() and torch.equal(src[:taken].long(), order[:taken] // k)


@pytest.mark.parametrize("n", [0, 5, 3000])
def test_sort_with_nothing_taken(n):
    idx = torch.full((n, 2), -1, dtype=torch.int32, device=DEV)
    off, perm, src = sort(idx, 16, src=True)
    assert (off == 0).all() and (perm == -1).all() and (src == -9).all()


def test_sort_all_to_the_last_expert():
    idx = torch.full((9000, 1), 1023, dtype=torch.int32, device=DEV)
    off, perm, _ = sort(idx, 1024)
    assert (off[:1024] == 0).all() and int(off[1024]) == 9000
    assert torch.equal(perm.flatten(), torch.arange(9000, dtype=torch.int32, device=DEV))


# ------------------------------------------------------------------ rows

SHAPES = [  # n, k, E, cols
    (1, 1, 1, 1), (1, 8, 256, 7168), (5, 3, 8, 7), (33, 2, 8, 255), (64, 2, 8, 256), (40, 8, 64, 1024), (17, 4, 16, 2052),
    (9, 9, 16, 130), (6, 20, 64, 515), (300, 8, 256, 640), (3, 2, 8, 14336), (130, 5, 8, 33)]
LAYOUTS = [(0, 0), (8, 8), (4, 4), (2, 2), (1, 1), (0, 3)]   # padding of a row, offset of the first


def setup(n, k, E, drop=0.2):
    idx = experts(n, k, E, 7 * n + k, drop if n > 1 else 0.0)
    if n > 2:
        idx[n // 2] = -1   # a token with no expert at all
    _, perm, _ = sort(idx, E)
    return perm


def named(perm, rows):
    """Which rows some entry names."""
    m = torch.zeros(rows, dtype=torch.bool, device=DEV)
    m[perm[perm >= 0].long()] = True
    return m


@pytest.mark.parametrize("n,k,E,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES + [F8])
def test_permute_copies_bits(n, k, E, c, pad, offset, dtype):
    perm = setup(n, k, E)
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[dtype.itemsize]
    xf, x = strided(n, c, pad, offset, torch.float32, 0.0)
    x = xf.to(dtype)[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c]
    x.view(bits).copy_(torch.randint(0, 2 ** (8 * dtype.itemsize - 1), (n, c), generator=gen(5), device=DEV))
    rows = n * k + 3
    yflat, y = strided(rows, c, pad, offset, dtype, 1.0)
    want = yflat.clone()
    api.asap_moe_permute(x, perm, y)
    w = want[offset:offset + rows * (c + pad)].view(rows, c + pad)[:, :c]
    t, j = torch.nonzero(perm >= 0, as_tuple=True)
    w.view(bits)[perm[t, j].long()] = x.view(bits)[t]
    assert torch.equal(yflat.view(bits), want.view(bits))   # (nothing beside the named rows is written)


def gathered(y, perm):
    rows = y[perm.clamp(min=0).long()].double()
    return torch.where((perm >= 0)[:, :, None], rows, torch.zeros_like(rows))


@pytest.mark.parametrize("n,k,E,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weights", [True, False])
def test_unpermute(n, k, E, c, pad, offset, dtype, weights):
    perm = setup(n, k, E)
    rows = n * k
    _, y = strided(rows, c, pad, offset, dtype, math.nan)
    y.copy_(randn((rows, c), 1))
    y[~named(perm, rows)] = math.nan          # rows behind the last segment are nobody's
    w = torch.randn((n, k), generator=gen(2), device=DEV) if weights else None
    if weights:
        w[perm < 0] = math.nan                # and so are the weights of entries without a row
    flat, out = strided(n, c, pad, offset, dtype, 3.0)
    keep = flat.clone()
    api.asap_moe_unpermute(y, w, perm, out)
    wd = torch.ones((n, k), device=DEV).double() if w is None else torch.where(perm >= 0, w, torch.zeros_like(w)).double()
    terms = gathered(y, perm) * wd[:, :, None]
    ref, size = terms.sum(1), terms.abs().sum(1)
    e = torch.finfo(dtype).eps / 2
    assert ((out.double() - ref).abs() <= e * ref.abs() + (k + 1) * U * (1 + e) * size + SUBNORMAL[dtype]).all()
    assert (out[(perm < 0).all(1)] == 0).all()
    keep[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c] = out
    assert torch.equal(flat, keep)


@pytest.mark.parametrize("n,k,E,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_unpermute_backward(n, k, E, c, pad, offset, dtype):
    perm = setup(n, k, E)
    rows = n * k + 2
    _, d_out = strided(n, c, pad, offset, dtype, math.nan)
    d_out.copy_(randn((n, c), 3))
    _, y = strided(rows, c, pad, offset, dtype, math.nan)
    y.copy_(randn((rows, c), 4))
    y[~named(perm, rows)] = math.nan
    w = torch.randn((n, k), generator=gen(2), device=DEV)
    w[perm < 0] = math.nan
    flat, d_y = strided(rows, c, pad, offset, dtype, 3.0)
    keep = flat.clone()
    d_w = torch.full((n, k), 5.0, device=DEV)
    api.asap_moe_unpermute_backward(d_out, y, w, perm, d_y, d_w)
    e = torch.finfo(dtype).eps / 2
    t, j = torch.nonzero(perm >= 0, as_tuple=True)
    ref = torch.full((rows, c), 3.0, device=DEV).double()
    ref[perm[t, j].long()] = w[t, j, None].double() * d_out[t].double()
    assert ((d_y.double() - ref).abs() <= (e + 2 * U) * ref.abs() + SUBNORMAL[dtype]).all()
    assert (d_y[~named(perm, rows)] == 3.0).all()
    keep[offset:offset + rows * (c + pad)].view(rows, c + pad)[:, :c] = d_y
    assert torch.equal(flat, keep)
    terms = gathered(y, perm) * d_out.double()[:, None, :]
    # (partial sums of neighbouring columns: far fewer than c additions in a row)
    assert ((d_w.double() - terms.sum(2)).abs() <= min(c, c / 32 + 24) * U * terms.abs().sum(2)).all()
    assert (d_w[perm < 0] == 0).all()
    # one of the two alone: the same bits
    d_w2, d_y2 = torch.full_like(d_w, 7.0), torch.full((rows, c), 3.0, device=DEV, dtype=dtype)
    api.asap_moe_unpermute_backward(d_out, y, w, perm, None, d_w2)
    api.asap_moe_unpermute_backward(d_out, None, w, perm, d_y2, None)
    assert torch.equal(d_w, d_w2) and torch.equal(d_y2, d_y)
    ones = torch.full_like(d_y2, 3.0)
    api.asap_moe_unpermute_backward(d_out, y, None, perm, ones, None)   # no weights: copies
    copies = torch.full_like(d_y2, 3.0)
    api.asap_moe_permute(d_out, perm, copies)
    assert torch.equal(ones, copies)


def test_gradients_against_differences():
    """out is linear in y and in w: differences of the forward call in fp32 are its gradients, up to the rounding of the
    two outputs (each within (k + 1) u of the sum of its terms' sizes, over a step of 1/4 or more)."""
    n, k, E, c = 12, 3, 8, 40
    perm = setup(n, k, E)
    rows = n * k
    y, w, d_out = randn((rows, c), 1), randn((n, k), 2), randn((n, c), 3)

    def loss(y, w):
        out = torch.empty((n, c), device=DEV)
        api.asap_moe_unpermute(y, w, perm, out)
        return (out.double() * d_out.double()).sum(1)    # by token

    d_y, d_w = torch.zeros_like(y), torch.zeros_like(w)
    api.asap_moe_unpermute_backward(d_out, y, w, perm, d_y, d_w)
    size = (gathered(y, perm).abs() * w.abs()[:, :, None].double()).sum(1)
    tol = (4 * (k + 1) * U * (size + 2) * d_out.abs().double()).sum(1) * 8
    base = loss(y, w)
    for j in range(k):
        v = w.clone()
        v[:, j] += 0.5
        got = (loss(y, v) - base) / (v - w)[:, j].double()
        assert ((got - d_w[:, j].double()).abs() <= tol * 2 + c * U * 16).all()
    for col in (0, 17, 39):
        for j in range(k):
            z = y.clone()
            r = perm[:, j].clamp(min=0).long()
            has = perm[:, j] >= 0
            z[r[has], col] += 0.5
            got = (loss(z, w) - base)[has] / (z - y)[r[has], col].double()
            assert ((got - d_y[r[has], col].double()).abs() <= (tol * 2)[has] + 1e-6).all()


@pytest.mark.parametrize("n,k,E,c", SHAPES)
@pytest.mark.parametrize("pad,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("places", [True, False])
def test_dequantize_gives_the_products_bits(n, k, E, c, pad, offset, dtype, places):
    perm = setup(n, k, E) if places else None
    _, q = strided(n, c, pad, offset, F8, 1.0)
    codes = torch.randint(0, 256, (n, c), generator=gen(1), device=DEV).to(torch.uint8)   # (NaNs among them)
    q.view(torch.uint8).copy_(codes)
    b = -(-c // 128)
    _, s = strided(n, b, pad, offset, torch.float32, 2.0)
    s.copy_(torch.rand((n, b), generator=gen(2), device=DEV) * 0.1)
    rows = n * k if places else n
    flat, x = strided(rows, c, pad, offset, dtype, 3.0)
    keep = flat.clone()
    api.asap_moe_fp8_dequantize(q, s, x, perm)
    v = (q.float() * s.repeat_interleave(128, 1)[:, :c]).to(dtype)
    w = keep[offset:offset + rows * (c + pad)].view(rows, c + pad)[:, :c]
    if places:
        t, j = torch.nonzero(perm >= 0, as_tuple=True)
        w[perm[t, j].long()] = v[t]
    else:
        w.copy_(v)
    assert torch.equal(flat.nan_to_num(77.0), keep.nan_to_num(77.0))


def test_quantise_and_dequantise():
    x = randn((37, 1000), 1, torch.bfloat16)
    q, s = torch.empty((37, 1000), dtype=F8, device=DEV), torch.empty((37, 8), device=DEV)
    api.asap_moe_fp8_quantize(x, q, s)
    y = torch.empty((37, 1000), device=DEV)
    api.asap_moe_fp8_dequantize(q, s, y)
    # half a step of e4m3 (2^-4), or of its subnormals (2^-10 scales)
    step = s.repeat_interleave(128, 1)[:, :1000].double()
    assert ((y.double() - x.double()).abs() <= 2.0 ** -4 * (1 + 1e-6) * x.double().abs() + 2.0 ** -10 * step).all()


# ------------------------------------------------------------------ calls as programs make them

def test_rows_that_do_not_exist_are_skipped_and_recorded():
    n, k, c, rows = 6, 2, 64, 5
    perm = torch.tensor([[0, 1], [2, -1], [5, 3], [-7, 4], [2 ** 31 - 1, -1], [-2 ** 31, -1]], dtype=torch.int32, device=DEV)
    good = (perm >= 0) & (perm < rows)
    x, y = randn((n, c), 1), randn((rows, c), 2)
    for call in (lambda p, st: api.asap_moe_permute(x, p, out, status=st),
                 lambda p, st: api.asap_moe_unpermute(y, None, p, back, status=st),
                 lambda p, st: api.asap_moe_unpermute_backward(x, y, None, p, out, d_w, status=st),
                 lambda p, st: api.asap_moe_fp8_dequantize(x.to(F8), torch.ones((n, 1), device=DEV), out, p, status=st)):
        out, back, d_w = torch.full((rows, c), 9.0, device=DEV), torch.empty((n, c), device=DEV), torch.empty((n, k), device=DEV)
        word = torch.zeros(1, dtype=torch.int32, device=DEV)
        call(torch.where(good, perm, torch.full_like(perm, -1)), word)
        assert word.item() == 0
        want = [t.clone() for t in (out, back, d_w)]
        call(perm, word)
        assert word.item() == 2
        call(perm, None)     # nowhere to record it: skipped all the same
        for a, b in zip((out, back, d_w), want):
            assert torch.equal(a.nan_to_num(4), b.nan_to_num(4))


def test_no_rows_at_all():
    n, k, c = 5, 2, 32
    perm = torch.full((n, k), -1, dtype=torch.int32, device=DEV)
    none = torch.empty((0, c), device=DEV)
    out, d_w = torch.full((n, c), 9.0, device=DEV), torch.full((n, k), 9.0, device=DEV)
    api.asap_moe_unpermute(none, d_w, perm, out)
    assert (out == 0).all()
    api.asap_moe_permute(out, perm, none)
    api.asap_moe_unpermute_backward(out, none, None, perm, none, d_w)
    assert (d_w == 0).all()
    d_w.fill_(9.0)     # no columns: empty sums
    api.asap_moe_unpermute_backward(out[:, :0], out[:, :0], None, perm, None, d_w)
    assert (d_w == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan(dtype):
    n, k, c = 4, 2, 256
    perm = torch.tensor([[0, 1], [2, 3], [4, 5], [6, 7]], dtype=torch.int32, device=DEV)
    y = randn((8, c), 1, dtype)
    y[0, 3], y[1, 3], y[2, 5], y[4, 7], y[5, 7] = math.inf, 1.0, math.nan, math.inf, -math.inf
    w = torch.ones((n, k), device=DEV)
    out = torch.empty((n, c), dtype=dtype, device=DEV)
    api.asap_moe_unpermute(y, w, perm, out)
    assert out[0, 3] == math.inf and out[1, 5].isnan() and out[2, 7].isnan()
    assert out.isfinite().sum() == n * c - 3
    d_w = torch.empty((n, k), device=DEV)
    api.asap_moe_unpermute_backward(torch.ones_like(out), y, w, perm, torch.empty_like(y), d_w)
    assert d_w[0, 0] == math.inf and d_w[1, 0].isnan() and d_w[2, 0] == math.inf and d_w[2, 1] == -math.inf
    assert d_w.isfinite().sum() == 4


def test_offsets_past_32_bits():
    """Rows 2^31 bytes apart."""
    ld, c, rows = (1 << 30) + 64, 200, 4
    flat = torch.zeros((rows - 1) * ld + c, dtype=torch.bfloat16, device=DEV)
    y = flat.as_strided((rows, c), (ld, 1))
    perm = torch.tensor([[3, 0], [1, 2]], dtype=torch.int32, device=DEV)
    x = randn((2, c), 1, torch.bfloat16)
    api.asap_moe_permute(x, perm, y)
    assert torch.equal(y[3], x[0]) and torch.equal(y[0], x[0]) and torch.equal(y[2], x[1])
    out = torch.empty_like(x)
    api.asap_moe_unpermute(y, None, perm, out)
    assert torch.equal(out, 2 * x)
    d_w = torch.empty((2, 2), device=DEV)
    api.asap_moe_unpermute_backward(x, y, None, perm, y, None)
    api.asap_moe_unpermute_backward(x, y, None, perm, None, d_w)
    ref = (x.double() ** 2).sum(1)
    assert ((d_w.double() - ref[:, None]).abs() <= c * U * ref[:, None]).all()
    q = torch.zeros((rows - 1) * ld + c, dtype=torch.uint8, device=DEV).as_strided((rows, c), (ld, 1))
    q[3] = 0x38   # 1.0
    z = torch.empty((rows, c), device=DEV)
    api.asap_moe_fp8_dequantize(q, torch.full((rows, 2), 0.5, device=DEV), z)
    assert (z[3] == 0.5).all() and (z[:3] == 0).all()


def test_streams_and_graphs():
    """The chain on a stream of its own, and captured once and replayed on new inputs, two graphs at a time."""
    n, k, E, c = 600, 8, 64, 512
    ins = [(experts(n, k, E, s, 0.1), randn((n, c), s, torch.bfloat16), torch.rand((n, k), generator=gen(s), device=DEV))
           for s in range(3)]

    def buffers():
        i32 = dict(dtype=torch.int32, device=DEV)
        b16 = dict(dtype=torch.bfloat16, device=DEV)
        return dict(off=torch.zeros(E + 1, **i32), perm=torch.zeros((n, k), **i32), ws=api.sort_workspace(n, k, E),
                    xp=torch.zeros((n * k, c), **b16), out=torch.zeros((n, c), **b16), dy=torch.zeros((n * k, c), **b16),
                    dw=torch.zeros((n, k), device=DEV), q=torch.empty((n, c), dtype=F8, device=DEV),
                    s=torch.empty((n, c // 128), device=DEV), idx=ins[0][0].clone(), x=ins[0][1].clone(), w=ins[0][2].clone())

    def chain(b, stream=None):
        api.asap_moe_sort(b["idx"], E, b["off"], b["perm"], b["ws"], stream=stream)
        api.asap_moe_permute(b["x"], b["perm"], b["xp"], stream=stream)
        api.asap_moe_unpermute(b["xp"], b["w"], b["perm"], b["out"], stream=stream)
        api.asap_moe_unpermute_backward(b["x"], b["xp"], b["w"], b["perm"], b["dy"], b["dw"], stream=stream)
        api.asap_moe_fp8_quantize(b["x"], b["q"], b["s"], stream=stream)
        api.asap_moe_fp8_dequantize(b["q"], b["s"], b["xp"], b["perm"], stream=stream)

    names = ("off", "perm", "xp", "out", "dy", "dw")
    want = []
    for i in ins:
        b = buffers()
        for name, v in zip(("idx", "x", "w"), i):
            b[name].copy_(v)
        chain(b)
        torch.cuda.synchronize()
        want.append([b[m].clone() for m in names])
    side = torch.cuda.Stream()
    b = buffers()
    torch.cuda.synchronize()
    chain(b, stream=side)
    side.synchronize()
    assert all(torch.equal(b[m], v) for m, v in zip(names, want[0]))
    graphs = []
    for _ in range(2):
        b, g = buffers(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            chain(b)
        graphs.append((g, b, torch.cuda.Stream()))
    for i, j in ((0, 1), (2, 0), (1, 2)):
        for (g, b, st), which in zip(graphs, (i, j)):
            for name, v in zip(("idx", "x", "w"), ins[which]):
                b[name].copy_(v)
            b["xp"].zero_()
            b["dy"].zero_()
        torch.cuda.synchronize()
        for g, b, st in graphs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for (g, b, st), which in zip(graphs, (i, j)):
            assert all(torch.equal(b[m], v) for m, v in zip(names, want[which]))


def test_refusals():
    n, k, E, c = 4, 2, 8, 64
    perm = torch.zeros((n, k), dtype=torch.int32, device=DEV)
    x, y, w = randn((n, c), 1), randn((n * k, c), 2), randn((n, k), 3)
    bad = [
        lambda: api.asap_moe_permute(x.t().contiguous().t(), perm, y),       # columns not contiguous
        lambda: api.asap_moe_permute(x, perm.t().contiguous().t(), y),       # places not contiguous
        lambda: api.asap_moe_permute(x, perm.long(), y),
        lambda: api.asap_moe_permute(x[:1].expand(n, c), perm, y),           # rows that are one row
        lambda: api.asap_moe_unpermute(y, w.t().contiguous().t(), perm, x),
        lambda: api.asap_moe_unpermute(y, w.half(), perm, x),
        lambda: api.asap_moe_unpermute(y.cpu(), w, perm, x),
        lambda: api.asap_moe_unpermute_backward(x, y, w, perm, y.half(), w),
        lambda: api.asap_moe_unpermute_backward(x, y, w, perm, y, w[:, :1]),
        lambda: api.asap_moe_unpermute_backward(x, None, w, perm, y, w),
        lambda: api.asap_moe_sort(perm, E, perm.view(-1), perm),             # too few offsets
        lambda: api.asap_moe_permute(x, perm, y, status=torch.zeros(1, device=DEV)),
        lambda: api.asap_moe_fp8_dequantize(x.to(F8), w, y, perm),           # scales of another width
        lambda: api.asap_moe_fp8_dequantize(x, w[:, :1].contiguous(), y, perm),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    off = torch.zeros(257, dtype=torch.int32, device=DEV)
    many = torch.zeros((9000, 8), dtype=torch.int32, device=DEV)
    with pytest.raises(_native.AsapError, match="workspace"):
        api.asap_moe_sort(many, 256, off, torch.zeros_like(many))
    with pytest.raises(_native.AsapError, match="n_experts"):
        api.asap_moe_sort(perm, 1025, torch.zeros(1026, dtype=torch.int32, device=DEV), perm.clone())
