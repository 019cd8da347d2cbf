"""The local-gradient operators against their 64-bit forms.

Tolerances (u = 2^-24, half a step of fp32; w = half a step of the stored type,
2^-24 or 2^-8): a value rounded once from fp32 is within w of it, and
  * embed: one fp32 product                      -> (u + w) |ref|
  * embed_grad: k - 1 fp32 additions, a product  -> (k + 1) u sum|dy| + w |ref|
  * act_pack, act_unpack: codes and values exact
  * act_wgrad: m additions, each within a whole fp32 step of the running sum
    (the matrix unit may truncate), three times as many for fp32 dy, and a
    product                                      -> (2 m + 1) u sum|dy x| + w |ref|
(second-order terms: the factor 1.01).  Where every partial sum is a whole
number below 2^24 all additions are exact in any order, and results are the
references rounded once: such inputs pin the indexing at any length.
"""
import numpy as np
import pytest
import torch

import paper_2507_07114_amd as ll
import workloads as wl
from oracle import local as ol
from workloads import device as wd

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
SENTINEL = 77.0


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def np64(t):
    return t.detach().cpu().double().numpy()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def padded(n, t, width, ld, dtype, shift=0, fill=SENTINEL):
    """[n][t][width] view with row stride ld, `shift` elements off the
    allocation's alignment, inside a buffer full of `fill`; returns both."""
    base = torch.full((shift + n * t * ld,), fill, dtype=dtype, device=DEV)
    return base, base[shift:].view(n, t, ld)[:, :, :width]


def outside(base, view):
    """Values of `base` not covered by `view`."""
    b = base.clone()
    v = b.as_strided(view.size(), view.stride(), view.storage_offset())
    v.zero_()
    return b


def row_buffer(n, size, offset, dtype, fill=SENTINEL):
    per16 = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = (offset + size + 3 + per16 - 1) // per16 * per16
    return torch.full((n, ld), fill, dtype=dtype, device=DEV)


def ints(shape, lo, hi, seed, dtype):
    return torch.randint(lo, hi + 1, shape, generator=gen(seed), device=DEV).to(dtype)


def lengths_of(lens, t, n):
    """(device lengths or None, host counts)."""
    if lens is None:
        return None, [t] * n
    return (torch.tensor(lens, dtype=torch.int32, device=DEV),
            [min(max(int(m), 0), t) for m in lens])


# ---- embedding lookup -----------------------------------------------------

# n, t, h, v, offset, first, table, out, int64 ids, lengths, ld_o - h, shift
EMBED = [
    (1, 1, 1, 1, 0, 0, F32, F32, False, None, 0, 0),
    (1, 1, 4096, 50, 8, 0, BF16, BF16, False, None, 0, 0),
    (3, 7, 33, 20, 5, 2, BF16, F32, True, None, 3, 1),
    (2, 130, 256, 300, 0, -4, F32, BF16, False, [200, 5], 0, 0),
    (4, 65, 1001, 64, 3, 0, F32, F32, True, [0, 65, -3, 1], 0, 0),
    (2, 64, 520, 40, 8, 10, BF16, BF16, False, [64, 63], 8, 0),
    (5, 3, 8, 1000, 16, 0, BF16, BF16, True, None, 0, 4),
    (1, 513, 12, 77, 4, 1000, F32, BF16, False, None, 4, 0),
    (2, 100, 2056, 90, 1, 0, BF16, BF16, False, None, 0, 0),
]


@pytest.mark.parametrize("n,t,h,v,offset,first,rdt,odt,wide,lens,pad,shift", EMBED)
def test_embed(n, t, h, v, offset, first, rdt, odt, wide, lens, pad, shift):
    reps = row_buffer(n, v * h, offset, rdt)
    reps.normal_(0, 1, generator=gen(1))
    tok = torch.randint(first - 3, first + v + 3, (n, t), generator=gen(2), device=DEV,
                        dtype=torch.int64 if wide else torch.int32)
    base, out = padded(n, t, h, h + pad, odt, shift)
    before = outside(base, out)
    dl, hl = lengths_of(lens, t, n)
    ll.ll_embed(tok, reps, out, v=v, first=first, offset=offset, scale=1.7, lengths=dl)
    torch.cuda.synchronize()
    assert torch.equal(outside(base, out), before)
    scale = float(np.float32(1.7))
    for i in range(n):
        table = np64(reps[i, offset:offset + v * h]).reshape(v, h)
        want = ol.embed(tok[i].tolist(), table, first, scale)
        got = np64(out[i])
        m = hl[i]
        assert (got[m:] == SENTINEL).all()
        assert (np.abs(got[:m] - want[:m]) <= 1.01 * (U + half_step(odt)) * np.abs(want[:m])).all()
        none = (want[:m] == 0).all(axis=1)
        assert not np.signbit(got[:m][none]).any()


def test_embed_far_ids_and_non_finite_rows():
    v, h = 6, 40
    reps = row_buffer(1, v * h, 0, F32)
    reps.fill_(1.0)
    reps[0, 2 * h] = float("inf")
    reps[0, 3 * h] = float("nan")
    big = 1 << 62
    tok = torch.tensor([[2, 3, 5, 6, -1, big, -big, 1 << 40]], device=DEV)
    out = torch.full((1, 8, h), SENTINEL, dtype=BF16, device=DEV)
    ll.ll_embed(tok, reps, out, v=v)
    o = out[0].float().cpu()
    assert torch.isinf(o[0, 0]) and torch.isnan(o[1, 0]) and (o[2] == 1).all()
    assert (o[0, 1:] == 1).all() and (o[3:] == 0).all()
    # the same ids at the far ends of the 64-bit range
    tok = torch.tensor([[-(1 << 63), -(1 << 63) + 2, (1 << 63) - 1]], device=DEV)
    out.fill_(SENTINEL)
    ll.ll_embed(tok, reps, out[:, :3].contiguous(), v=v, first=0)
    o3 = torch.full((1, 3, h), SENTINEL, dtype=F32, device=DEV)
    ll.ll_embed(tok, reps, o3, v=v, first=-(1 << 63))
    assert (o3[0, 0] == 1).all() and torch.isinf(o3[0, 1, 0]) and (o3[0, 2] == 0).all()


# ---- embedding gradient ------------------------------------------------------

# n, t, h, v, offset, first, dy, grads, int64 ids, lengths, ld_y - h, shift, ids
GRAD = [
    (1, 1, 1, 1, 0, 0, F32, F32, False, None, 0, 0, "any"),
    (1, 1, 4096, 50, 8, 0, BF16, BF16, False, None, 0, 0, "any"),
    (3, 70, 33, 20, 5, 2, BF16, F32, True, None, 3, 1, "any"),
    (2, 1030, 256, 300, 0, -4, F32, BF16, False, [2000, 5], 0, 0, "any"),
    (4, 65, 1001, 64, 3, 0, F32, F32, True, [0, 65, -3, 1], 0, 0, "any"),
    (2, 640, 520, 700, 8, 10, BF16, BF16, False, [640, 639], 8, 0, "few"),
    (5, 3, 8, 1000, 16, 0, BF16, BF16, True, None, 0, 4, "any"),
    (2, 3000, 72, 5, 4, 0, BF16, F32, False, None, 0, 0, "one"),
    (1, 4099, 64, 2500, 0, 0, F32, F32, False, None, 0, 0, "few"),
    (3, 129, 2056, 40, 1, 0, BF16, BF16, False, None, 0, 0, "none"),
    (1, 9000, 130, 1027, 2, 0, BF16, BF16, False, [8193], 0, 0, "any"),
    # 256, 512 and more tokens go different ways
    (2, 256, 72, 33, 0, 0, F32, BF16, True, [256, 200], 0, 0, "few"),
    (2, 257, 72, 33, 0, 0, BF16, BF16, False, [257, 64], 0, 0, "few"),
    (3, 512, 24, 700, 1, 0, BF16, F32, False, None, 0, 0, "few"),
    (2, 513, 24, 700, 0, 5, F32, BF16, True, [513, 500], 1, 0, "few"),
    (1, 511, 5000, 9, 2, 0, F32, F32, False, None, 0, 1, "any"),
    (2, 513, 9, 2, 0, 0, BF16, BF16, False, None, 0, 0, "one"),
    (3, 200, 24, 40000, 3, -7, BF16, F32, False, None, 0, 1, "one"),
    (1, 300, 4100, 3, 0, 0, BF16, BF16, False, None, 1, 0, "any"),
    (2, 400, 1, 70001, 0, 0, F32, F32, True, None, 0, 0, "any"),
]


def draw_ids(kind, n, t, v, first, wide, seed=3):
    dt = torch.int64 if wide else torch.int32
    if kind == "any":
        return torch.randint(first - 2, first + v + 2, (n, t), generator=gen(seed), device=DEV,
                             dtype=dt)
    if kind == "few":  # a few rows take nearly all tokens
        x = torch.rand((n, t), generator=gen(seed), device=DEV).pow(12) * v
        return (x.to(dt) + first).clamp_max(first + v - 1)
    if kind == "one":
        return torch.full((n, t), first + v - 1, device=DEV, dtype=dt)
    return torch.full((n, t), first - 1, device=DEV, dtype=dt)  # none is held


def run_embed_grad(tok, dy, grads, **kw):
    n, t = tok.shape
    need = ll.ll_embed_grad_workspace_bytes(n, t, dy.shape[2], kw["v"])
    ws = torch.randint(0, 256, (max(need, 16),), dtype=torch.uint8, device=DEV)
    ll.ll_embed_grad(tok, dy, grads, workspace=ws, **kw)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,t,h,v,offset,first,ydt,gdt,wide,lens,pad,shift,ids", GRAD)
def test_embed_grad(n, t, h, v, offset, first, ydt, gdt, wide, lens, pad, shift, ids, accumulate):
    tok = draw_ids(ids, n, t, v, first, wide)
    _, dy = padded(n, t, h, h + pad, ydt, shift)
    dy.normal_(0, 1, generator=gen(4))
    dl, hl = lengths_of(lens, t, n)
    for i in range(n):
        dy[i, hl[i]:] = float("nan")  # behind the batch: not read
        dy[i][(tok[i] < first) | (tok[i] >= first + v)] = float("nan")  # not in the table
    grads = row_buffer(n, v * h, offset, gdt)
    grads.normal_(0, 1, generator=gen(5))
    old = grads.clone()
    run_embed_grad(tok, dy, grads, v=v, first=first, offset=offset, scale=-1.3,
                   accumulate=accumulate, lengths=dl)
    torch.cuda.synchronize()
    assert torch.equal(grads[:, :offset], old[:, :offset])
    assert torch.equal(grads[:, offset + v * h:], old[:, offset + v * h:])
    scale = float(np.float32(-1.3))
    for i in range(n):
        m = hl[i]
        want, count, size = ol.embed_grad(tok[i, :m].tolist(), np64(dy[i, :m]), v, first, scale)
        got = np64(grads[i, offset:offset + v * h]).reshape(v, h)
        was = np64(old[i, offset:offset + v * h]).reshape(v, h)
        none = count == 0
        if accumulate:
            assert np.array_equal(got[none], was[none])
            want, size = want + was, size + np.abs(was)
        else:
            assert (got[none] == 0).all() and not np.signbit(got[none]).any()
        bound = (count[:, None] + 2) * U * size + half_step(gdt) * np.abs(want)
        assert (np.abs(got - want)[~none] <= 1.01 * bound[~none]).all()


@pytest.mark.parametrize("ids", ["any", "few", "one"])
@pytest.mark.parametrize("n,t,h,v,ydt", [(1, 40000, 96, 600, BF16), (2, 20001, 67, 31, F32),
                                         (3, 2500, 512, 70000, BF16)])
def test_embed_grad_whole_numbers_are_exact(n, t, h, v, ydt, ids):
    tok = draw_ids(ids, n, t, v, 0, False)
    dy = ints((n, t, h), -7, 7, 6, ydt)
    grads = row_buffer(n, v * h, 0, F32)
    run_embed_grad(tok, dy, grads, v=v, scale=0.5)
    want = torch.zeros((n, v, h), dtype=torch.float64, device=DEV)
    for i in range(n):
        at = torch.nonzero((tok[i] >= 0) & (tok[i] < v)).flatten()
        want[i].index_add_(0, tok[i, at].long(), dy[i, at].double())
    assert torch.equal(grads[:, :v * h].reshape(n, v, h).double(), 0.5 * want)


def test_embed_grad_without_tokens_writes_zeros():
    grads = row_buffer(2, 30, 5, BF16)
    tok = torch.zeros((2, 0), dtype=torch.int32, device=DEV)
    run_embed_grad(tok, torch.zeros((2, 0, 3), dtype=BF16, device=DEV), grads, v=10, offset=5)
    assert (grads[:, 5:35] == 0).all() and (grads[:, :5] == SENTINEL).all()
    assert (grads[:, 35:] == SENTINEL).all()
    grads.fill_(SENTINEL)
    run_embed_grad(tok, torch.zeros((2, 0, 3), dtype=BF16, device=DEV), grads, v=10, offset=5,
                   accumulate=True)
    assert (grads == SENTINEL).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("t", [70, 400, 1500])
def test_tokens_and_rows_inside_wider_ones(t, wide):
    # ids in a slice of a wider tensor, tables in the middle of wider row buffers,
    # workers of a batch cut from a larger one
    n, h, v, off = 3, 37, 90, 11
    tok = draw_ids("any", n, t, v, -3, wide)
    wider = torch.full((n + 2, t + 13), -77, dtype=tok.dtype, device=DEV)
    wider[1:-1, 5:5 + t] = tok
    cut = wider[1:-1, 5:5 + t]
    table = torch.randn((n, v * h), generator=gen(50), device=DEV).to(BF16)
    rows = torch.full((n + 1, 8 * 1000), SENTINEL, dtype=BF16, device=DEV)
    rows[1:, off:off + v * h] = table
    plain = row_buffer(n, v * h, 0, BF16)
    plain[:, :v * h] = table
    out, ref = torch.empty((2, n, t, h), dtype=F32, device=DEV)
    ll.ll_embed(cut, rows[1:, :4000], out, v=v, first=-3, offset=off)
    ll.ll_embed(tok, plain, ref, v=v, first=-3)
    assert torch.equal(out, ref) and out.abs().sum() > 0
    dy = torch.randn((n, t, h), generator=gen(51), device=DEV)
    before = rows.clone()
    run_embed_grad(cut, dy, rows[1:, :4000], v=v, first=-3, offset=off)
    run_embed_grad(tok, dy, plain, v=v, first=-3)
    assert torch.equal(rows[1:, off:off + v * h], plain[:, :v * h])
    rows[1:, off:off + v * h] = before[1:, off:off + v * h]
    assert torch.equal(rows, before)


def test_embed_grad_repeats_bit_for_bit():
    n, t, h, v = 2, 6000, 264, 500
    tok = draw_ids("few", n, t, v, 0, False)
    dy = torch.randn((n, t, h), generator=gen(7), device=DEV)
    a, b = row_buffer(n, v * h, 0, F32), row_buffer(n, v * h, 0, F32)
    run_embed_grad(tok, dy, a, v=v)
    for _ in range(3):
        run_embed_grad(tok, dy, b, v=v)
        assert torch.equal(a, b)


def test_embed_grad_is_the_lookups_difference():
    # fp32 whole numbers: the central difference of a linear loss is exact
    n, t, h, v, off = 2, 50, 24, 9, 4
    tok = draw_ids("any", n, t, v, 0, True)
    c = ints((n, t, h), -4, 4, 8, F32)
    reps = row_buffer(n, v * h, off, F32)
    reps.copy_(ints(tuple(reps.shape), -9, 9, 9, F32))
    grads = row_buffer(n, v * h, off, F32)
    run_embed_grad(tok, c, grads, v=v, offset=off, scale=2.0)
    out = torch.empty((n, t, h), device=DEV)

    def loss(r):
        ll.ll_embed(tok, r, out, v=v, offset=off, scale=2.0)
        return (c.double() * out.double()).sum((1, 2))

    for at in (0, 23, 24, 5 * 24 + 7, v * h - 1):
        up, down = reps.clone(), reps.clone()
        up[:, off + at] += 1
        down[:, off + at] -= 1
        assert torch.equal((loss(up) - loss(down)) / 2, grads[:, off + at].double())


# ---- 8-bit checkpoints --------------------------------------------------------

# n, t, h, x, out, lengths, ld_x - h, ld_q - h, ld_s - groups, shift
PACK = [
    (1, 1, 1, F32, F32, None, 0, 0, 0, 0),
    (1, 1, 4096, BF16, BF16, None, 0, 0, 0, 0),
    (2, 5, 31, BF16, F32, None, 1, 1, 1, 1),
    (3, 9, 70, F32, BF16, [9, 0, 4], 0, 0, 0, 0),
    (2, 33, 264, BF16, BF16, [40, -1], 8, 8, 0, 0),
    (1, 17, 2056, F32, F32, None, 0, 8, 3, 0),
    (4, 3, 1000, BF16, BF16, None, 24, 0, 0, 3),
    (2, 64, 96, F32, BF16, None, 4, 16, 1, 0),
    (1, 300, 515, BF16, F32, [299], 0, 13, 0, 0),
]


def wild(shape, dtype, seed):
    """Values over the whole range of fp32, zeros, whole groups of zeros, and
    the borders of the scale rule."""
    g = gen(seed)
    x = torch.randn(shape, generator=g, device=DEV)
    e = torch.randint(-130, 120, (*shape[:-1], (shape[-1] + 31) // 32), generator=g, device=DEV)
    e = e.repeat_interleave(32, -1)[..., :shape[-1]]
    near = torch.randint(-12, 1, shape, generator=g, device=DEV)
    x = torch.ldexp(x, (e + near).float().clamp(-140, 120))
    x[torch.rand(shape, generator=g, device=DEV) < 0.05] = 0.0
    x[torch.rand(shape[:-1], generator=g, device=DEV) < 0.1] = 0.0
    flat = x.view(-1)
    flat[: 1] = 448.0
    if flat.numel() > 64:
        flat[32:33] = 448.0 * 1.0001 if dtype == F32 else 450.0
        flat[40:41] = -0.0
    return x.to(dtype)


@pytest.mark.parametrize("n,t,h,xdt,odt,lens,px,pq,ps,shift", PACK)
def test_act_pack_and_unpack(n, t, h, xdt, odt, lens, px, pq, ps, shift):
    groups = (h + 31) // 32
    xb, x = padded(n, t, h, h + px, xdt, shift)
    x.copy_(wild((n, t, h), xdt, 10))
    if t > 2:  # values that are not finite, alone and as a whole group
        x[0, 1, 0] = float("inf")
        x[0, 2, : min(h, 32)] = float("nan")
    xcopy = xb.clone()
    qb, q = padded(n, t, h, h + pq, torch.uint8, shift, fill=171)
    sb, s = padded(n, t, groups, groups + ps, torch.uint8, shift, fill=171)
    qo, so = outside(qb, q), outside(sb, s)
    dl, hl = lengths_of(lens, t, n)
    ll.ll_act_pack(x, q, s, lengths=dl)
    torch.cuda.synchronize()
    assert torch.equal(outside(qb, q), qo) and torch.equal(outside(sb, s), so)
    assert torch.equal(xb.view(torch.uint8), xcopy.view(torch.uint8))
    ob, out = padded(n, t, h, h + px, odt, shift)
    oo = outside(ob, out)
    ll.ll_act_unpack(q, s, out, lengths=dl)
    torch.cuda.synchronize()
    assert torch.equal(outside(ob, out), oo)
    for i in range(n):
        m = hl[i]
        assert (q[i, m:] == 171).all() and (s[i, m:] == 171).all()
        assert (out[i, m:] == SENTINEL).all()
        wq, ws = ol.pack(np64(x[i, :m]))
        assert np.array_equal(s[i, :m].cpu().numpy(), ws)
        assert np.array_equal(q[i, :m].cpu().numpy(), wq)
        assert np.array_equal(np64(out[i, :m]), ol.unpack(wq, ws), equal_nan=True)


@pytest.mark.parametrize("odt", [F32, BF16])
def test_act_unpack_every_code_and_scale(odt):
    q = torch.arange(256, dtype=torch.uint8, device=DEV).repeat(238, 1)[None].contiguous()
    s = torch.arange(10, 248, dtype=torch.uint8, device=DEV)[None, :, None].repeat(1, 1, 8)
    out = torch.empty((1, 238, 256), dtype=odt, device=DEV)
    ll.ll_act_unpack(q, s.contiguous(), out)
    # codes and scales that ll_act_pack does not write reach past fp32
    want = torch.from_numpy(ol.unpack(q[0].cpu().numpy(), s[0].cpu().numpy())).to(odt)
    assert np.array_equal(np64(out[0]), np64(want), equal_nan=True)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_act_pack_of_the_largest_values(dt):
    top = torch.finfo(dt).max
    x = torch.tensor([[[top, -top, top / 2, 1.0, top * 0.96875, top * 0.9]]], dtype=dt, device=DEV)
    q = torch.empty((1, 1, 6), dtype=torch.uint8, device=DEV)
    s = torch.empty((1, 1, 1), dtype=torch.uint8, device=DEV)
    ll.ll_act_pack(x, q, s)
    wq, ws = ol.pack(np64(x[0]))
    assert np.array_equal(q[0].cpu().numpy(), wq) and np.array_equal(s[0].cpu().numpy(), ws)
    out = torch.empty_like(x)
    ll.ll_act_unpack(q, s, out)
    assert torch.isfinite(out).all()
    assert (np.abs(np64(out) - np64(x)) <= np64(x.abs()) / 16 + 2.0 ** 110).all()


# ---- weight gradient -------------------------------------------------------------

# n, t, o, h, dy, grads, offset, lengths, ld_y - o, ld_q - h, ld_s - groups, shift
WGRAD = [
    (1, 1, 1, 1, F32, F32, 0, None, 0, 0, 0, 0),
    (1, 1, 300, 520, BF16, BF16, 8, None, 0, 0, 0, 0),
    (2, 33, 64, 64, BF16, F32, 0, None, 0, 0, 0, 0),
    (3, 65, 33, 70, F32, BF16, 5, [65, 0, 7], 1, 1, 1, 1),
    (1, 200, 256, 256, BF16, BF16, 0, None, 0, 0, 0, 0),
    (2, 333, 130, 264, F32, F32, 3, [400, -2], 2, 8, 0, 0),
    (1, 64, 1000, 96, BF16, BF16, 1, None, 24, 16, 1, 0),
    (2, 129, 257, 513, BF16, F32, 4, [129, 128], 7, 15, 0, 0),
    (1, 2000, 40, 48, F32, F32, 0, None, 0, 0, 0, 0),
    (4, 31, 8, 2056, BF16, BF16, 16, None, 0, 0, 0, 0),
    (1, 5000, 96, 160, BF16, BF16, 0, [4097], 0, 0, 0, 0),
    (1, 96, 515, 300, F32, BF16, 2, None, 0, 0, 0, 2),
    # as many tiles as compute units and more
    (66, 75, 264, 520, BF16, BF16, 3, [75, 0, 33] * 22, 8, 8, 0, 0),
    (65, 41, 512, 264, F32, F32, 0, None, 1, 1, 1, 1),
    (67, 1, 520, 272, BF16, F32, 1, [1, 0] * 33 + [1], 0, 3, 0, 1),
]


def run_wgrad(dy, q, s, grads, **kw):
    n, t, o = dy.shape
    need = ll.ll_act_wgrad_workspace_bytes(n, t, o, q.shape[2])
    ws = torch.randint(0, 256, (max(need, 16),), dtype=torch.uint8, device=DEV)
    ll.ll_act_wgrad(dy, q, s, grads, workspace=ws, **kw)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,t,o,h,ydt,gdt,offset,lens,py,pq,ps,shift", WGRAD)
def test_act_wgrad(n, t, o, h, ydt, gdt, offset, lens, py, pq, ps, shift, accumulate):
    groups = (h + 31) // 32
    dl, hl = lengths_of(lens, t, n)
    _, dy = padded(n, t, o, o + py, ydt, shift, fill=float("nan"))
    dy.normal_(0, 1, generator=gen(11))
    x = torch.randn((n, t, h), generator=gen(12), device=DEV) * 3
    _, q = padded(n, t, h, h + pq, torch.uint8, shift, fill=0x7F)
    _, s = padded(n, t, groups, groups + ps, torch.uint8, shift, fill=255)
    ll.ll_act_pack(x, q, s)
    for i in range(n):  # behind the batch: not read
        dy[i, hl[i]:] = float("nan")
        q[i, hl[i]:] = 0x7F
    grads = row_buffer(n, o * h, offset, gdt)
    grads.normal_(0, 1, generator=gen(13))
    old = grads.clone()
    run_wgrad(dy, q, s, grads, offset=offset, scale=0.7, accumulate=accumulate, lengths=dl)
    torch.cuda.synchronize()
    assert torch.equal(grads[:, :offset], old[:, :offset])
    assert torch.equal(grads[:, offset + o * h:], old[:, offset + o * h:])
    scale = float(np.float32(0.7))
    terms = 3 if ydt == F32 else 1
    for i in range(n):
        m = hl[i]
        want, size = ol.wgrad(np64(dy[i, :m]), ol.unpack(q[i, :m].cpu().numpy(),
                                                         s[i, :m].cpu().numpy()), scale)
        got = np64(grads[i, offset:offset + o * h]).reshape(o, h)
        if accumulate:
            was = np64(old[i, offset:offset + o * h]).reshape(o, h)
            want, size = want + was, size + np.abs(was)
        bound = (2 * terms * m + 2) * U * size + half_step(gdt) * np.abs(want)
        assert (np.abs(got - want) <= 1.01 * bound).all(), np.abs(got - want).max()


@pytest.mark.parametrize("ydt,top", [(BF16, 8), (F32, 500)])
@pytest.mark.parametrize("n,t,o,h", [(1, 4096, 256, 256), (2, 1000, 520, 264), (1, 9001, 65, 40),
                                     (3, 130, 770, 1030), (1, 700, 1025, 2049),
                                     (70, 37, 264, 520), (1, 290, 4096, 4104),
                                     (256, 100, 40, 16),
                                     # few tokens, more tiles than fit at once
                                     (3, 10, 2900, 3300), (1, 65, 4097, 4200),
                                     # a round of whole tiles and one cut into
                                     # runs; runs of large tiles; many runs
                                     (1, 1024, 4096, 4352), (1, 8192, 2048, 2040),
                                     (2, 8192, 136, 256), (1, 8001, 300, 257)])
def test_act_wgrad_whole_numbers_are_exact(n, t, o, h, ydt, top):
    # |x| <= 3 and |dy| <= top: every partial sum is below 9001 * 3 * 500 < 2^24
    dy = ints((n, t, o), -top, top, 14, ydt)
    x = ints((n, t, h), -3, 3, 15, BF16)
    q = torch.empty((n, t, h), dtype=torch.uint8, device=DEV)
    s = torch.empty((n, t, (h + 31) // 32), dtype=torch.uint8, device=DEV)
    ll.ll_act_pack(x, q, s)
    grads = row_buffer(n, o * h, 0, F32)
    run_wgrad(dy, q, s, grads, scale=0.25)
    for i in range(n):
        want = 0.25 * torch.mm(dy[i].double().t().contiguous(), x[i].double())
        assert torch.equal(grads[i, : o * h].view(o, h).double(), want)


def test_act_wgrad_takes_all_bits_of_fp32():
    # one token, x^ = 1: the gradient is dy itself, to the last bit
    o, h = 300, 40
    dy = torch.randn((1, 1, o), generator=gen(16), device=DEV)
    dy[0, 0, :6] = torch.tensor([3.4e38, -3.4e38, 1.0000001, -2.0 ** -100, 0.0, 2.0 ** 100])
    q = torch.full((1, 1, h), 0x38, dtype=torch.uint8, device=DEV)  # 1.0
    s = torch.full((1, 1, 2), 127, dtype=torch.uint8, device=DEV)
    grads = row_buffer(1, o * h, 0, F32)
    run_wgrad(dy, q, s, grads)
    assert torch.equal(grads[0, : o * h].view(o, h), dy[0, 0][:, None].expand(o, h))
    dy[0, 0, 0], dy[0, 0, 1], dy[0, 0, 2] = float("inf"), float("-inf"), float("nan")
    run_wgrad(dy, q, s, grads)
    g = grads[0, : o * h].view(o, h)
    assert (g[0] == float("inf")).all() and (g[1] == float("-inf")).all()
    assert torch.isnan(g[2]).all() and torch.isfinite(g[3:]).all()


def test_act_wgrad_without_tokens_writes_zeros():
    grads = row_buffer(2, 12, 5, BF16)
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)
    dy = torch.zeros((2, 0, 3), dtype=BF16, device=DEV)
    run_wgrad(dy, z(2, 0, 4), z(2, 0, 1), grads, offset=5)
    assert (grads[:, 5:17] == 0).all() and (grads[:, :5] == SENTINEL).all()
    assert (grads[:, 17:] == SENTINEL).all()


def test_act_wgrad_repeats_bit_for_bit():
    n, t, o, h = 1, 6000, 130, 200
    dy = torch.randn((n, t, o), generator=gen(17), device=DEV)
    x = torch.randn((n, t, h), generator=gen(18), device=DEV)
    q = torch.empty((n, t, h), dtype=torch.uint8, device=DEV)
    s = torch.empty((n, t, 7), dtype=torch.uint8, device=DEV)
    ll.ll_act_pack(x, q, s)
    a, b = row_buffer(n, o * h, 0, F32), row_buffer(n, o * h, 0, F32)
    run_wgrad(dy, q, s, a)
    for _ in range(3):
        run_wgrad(dy, q, s, b)
        assert torch.equal(a, b)


# ---- far offsets ----


def test_rows_past_2_31_elements():
    # two replica and gradient rows of 1.2e9 bf16 elements, the table and the
    # weight at their ends: element offsets beyond 2^31, bytes beyond 2^32
    n, v, h, o, t = 2, 7, 40, 9, 300
    ld, off = 1_200_000_000, 1_200_000_000 - 7 * 40 - 9 * 40
    rows = torch.zeros((n, ld), dtype=BF16, device=DEV)
    rows[:, off:] = torch.randn((n, ld - off), generator=gen(40), device=DEV).to(BF16)
    small = rows[:, off:].clone()
    tok = draw_ids("any", n, t, v, 0, True)
    out, ref = torch.empty((2, n, t, h), dtype=BF16, device=DEV)
    ll.ll_embed(tok, rows, out, v=v, offset=off)
    ll.ll_embed(tok, small, ref, v=v)
    assert torch.equal(out, ref) and out.abs().sum() > 0
    q = torch.empty((n, t, h), dtype=torch.uint8, device=DEV)
    s = torch.empty((n, t, 2), dtype=torch.uint8, device=DEV)
    ll.ll_act_pack(out, q, s)
    dy = torch.randn((n, t, o), generator=gen(41), device=DEV).to(BF16)
    rows.zero_()
    small.zero_()
    for g, base in ((rows, off), (small, 0)):
        run_embed_grad(tok, out, g, v=v, offset=base)
        run_wgrad(dy, q, s, g, offset=base + v * h)
    assert torch.equal(rows[:, off:], small) and small.abs().sum() > 0
    assert not rows[:, :off].any()


def test_activations_past_2_31_elements():
    # token rows at the end of 2.2e9 elements; only the last tokens are filled
    n, t, h = 1, 68000, 96
    ld = 32768
    x = torch.zeros((n, t, ld), dtype=BF16, device=DEV)[:, :, :h]
    q = torch.zeros((n, t, ld), dtype=torch.uint8, device=DEV)[:, :, :h]
    s = torch.zeros((n, t, 3), dtype=torch.uint8, device=DEV)
    m = 500
    x[:, -m:] = ints((n, m, h), -3, 3, 42, BF16)
    ll.ll_act_pack(x, q, s)
    back = torch.zeros((n, t, ld), dtype=BF16, device=DEV)[:, :, :h]
    ll.ll_act_unpack(q, s, back)
    assert torch.equal(back[:, -m:], x[:, -m:]) and not back[:, :-m].any()
    o = 8
    dy = ints((n, t, o), -5, 5, 43, BF16)
    grads = row_buffer(n, o * h, 0, F32)
    run_wgrad(dy, q, s, grads)
    want = torch.mm(dy[0, -m:].double().t().contiguous(), x[0, -m:].double())
    assert torch.equal(grads[0, : o * h].view(o, h).double(), want)
    tok = torch.full((n, t), -1, dtype=torch.int32, device=DEV)
    tok[0, -m:] = torch.randint(0, 4, (m,), generator=gen(44), device=DEV, dtype=torch.int32)
    grads = row_buffer(n, 4 * h, 0, F32)
    run_embed_grad(tok, x, grads, v=4)
    want = torch.zeros((4, h), dtype=torch.float64, device=DEV)
    want.index_add_(0, tok[0, -m:].long(), x[0, -m:].double())
    assert torch.equal(grads[0, : 4 * h].view(4, h).double(), want)
    big = torch.zeros((n, t, ld), dtype=BF16, device=DEV)[:, :, :h]
    table = row_buffer(1, 4 * h, 0, BF16)
    table.normal_(generator=gen(45))
    ll.ll_embed(tok, table, big, v=4)
    assert torch.equal(big[0, -m:], table[0, : 4 * h].view(4, h)[tok[0, -m:].long()])
    assert not big[0, :-m].any()


# ---- together ----------------------------------------------------------------------

class Layer:
    """A shard of N workers that holds an embedding and a linear layer, its
    step, and the batch's constant output gradient."""

    def __init__(self, n=3, t=70, v=40, h=72, o=24, seed=20):
        self.n, self.t, self.v, self.h, self.o = n, t, v, h, o
        self.d = v * h + o * h
        ld = (self.d + 255) // 256 * 256
        self.theta = torch.randn(self.d, generator=gen(seed), device=DEV) * 0.1
        self.replicas = torch.zeros((n, ld), dtype=BF16, device=DEV)
        self.replicas[:, : self.d] = self.theta.to(BF16)
        self.grads = torch.zeros((n, ld), dtype=BF16, device=DEV)
        self.tok = torch.randint(-1, v, (n, t), generator=gen(seed + 1), device=DEV,
                                 dtype=torch.int32)
        self.lengths = torch.tensor([t, t // 2, 0][:n], dtype=torch.int32, device=DEV)
        self.x = torch.zeros((n, t, h), dtype=BF16, device=DEV)
        self.q = torch.zeros((n, t, h), dtype=torch.uint8, device=DEV)
        self.s = torch.zeros((n, t, (h + 31) // 32), dtype=torch.uint8, device=DEV)
        self.dy = torch.randn((n, t, o), generator=gen(seed + 2), device=DEV).to(BF16)
        self.dx = torch.zeros((n, t, h), dtype=BF16, device=DEV)
        self.ws = torch.zeros(max(ll.ll_embed_grad_workspace_bytes(n, t, h, v),
                                  ll.ll_act_wgrad_workspace_bytes(n, t, o, h), 16),
                              dtype=torch.uint8, device=DEV)

    def gradients(self):
        ll.ll_embed(self.tok, self.replicas, self.x, v=self.v, scale=3.0, lengths=self.lengths)
        ll.ll_act_pack(self.x, self.q, self.s, lengths=self.lengths)
        w0 = self.v * self.h
        for i in range(self.n):  # the layer's input gradient: a library product
            w = self.replicas[i, w0:w0 + self.o * self.h].view(self.o, self.h)
            self.dx[i] = torch.mm(self.dy[i].float(), w.float()).to(BF16)
        ll.ll_act_wgrad(self.dy, self.q, self.s, self.grads, offset=w0, lengths=self.lengths,
                        workspace=self.ws)
        ll.ll_embed_grad(self.tok, self.dx, self.grads, v=self.v, scale=3.0,
                         lengths=self.lengths, workspace=self.ws)

    def step(self, t):
        self.gradients()
        ll.lossy_step_fused(d=self.d, packet=64, step=t, loss_g=ll.bernoulli(0.2),
                            loss_b=ll.bernoulli(0.2), grads=self.grads, opt=ll.sgd(0.1),
                            theta=self.theta, replicas=self.replicas)


def test_layer_step_against_64_bits():
    a = Layer()
    reps = np64(a.replicas)
    a.gradients()
    torch.cuda.synchronize()
    w0 = a.v * a.h
    for i, m in enumerate(a.lengths.tolist()):
        table = reps[i, :w0].reshape(a.v, a.h)
        w = reps[i, w0:a.d].reshape(a.o, a.h)
        tok = a.tok[i, :m].tolist()
        x = ol.embed(tok, table, 0, 3.0)
        xr = torch.from_numpy(x).float().to(BF16).double().numpy()  # products exact in fp32
        assert np.array_equal(np64(a.x[i, :m]), xr)
        xq = ol.unpack(*ol.pack(xr)) if m else xr
        dy = np64(a.dy[i, :m])
        want, size = ol.wgrad(dy, xq, 1.0)
        got = np64(a.grads[i, w0:a.d]).reshape(a.o, a.h)
        assert (np.abs(got - want) <= 1.01 * ((2 * m + 2) * U * size + 2.0 ** -8 * np.abs(want))).all()
        want, count, size = ol.embed_grad(tok, np64(a.dx[i, :m]), a.v, 0, 3.0)
        got = np64(a.grads[i, :w0]).reshape(a.v, a.h)
        assert (np.abs(got - want) <= 1.01 * ((count[:, None] + 2) * U * size
                                              + 2.0 ** -8 * np.abs(want))).all()
        # and dx itself is the product of dy and the worker's own weight
        ref, mag = dy @ w, np.abs(dy) @ np.abs(w)
        assert (np.abs(np64(a.dx[i, :m]) - ref) <= 1.01 * ((2 * a.o + 2) * U * mag
                                                           + 2.0 ** -8 * np.abs(ref))).all()


def test_layer_steps_on_a_side_stream_and_repeat():
    a, b = Layer(), Layer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in range(3):
        a.step(t)
        with torch.cuda.stream(side):
            b.step(t)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(a.theta, b.theta) and torch.equal(a.replicas, b.replicas)
    assert torch.equal(a.grads, b.grads) and not torch.equal(a.replicas[0], a.replicas[1])


def test_captured_gradients_replay_like_eager():
    a, b = Layer(t=1500, h=136, o=40), Layer(t=1500, h=136, o=40)

    def kernels(s):
        ll.ll_embed(s.tok, s.replicas, s.x, v=s.v, scale=3.0, lengths=s.lengths)
        ll.ll_act_pack(s.x, s.q, s.s, lengths=s.lengths)
        ll.ll_act_unpack(s.q, s.s, s.dx, lengths=s.lengths)
        ll.ll_act_wgrad(s.dy, s.q, s.s, s.grads, offset=s.v * s.h, lengths=s.lengths,
                        workspace=s.ws)
        ll.ll_embed_grad(s.tok, s.dx, s.grads, v=s.v, scale=3.0, lengths=s.lengths,
                         workspace=s.ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kernels(b)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kernels(b)
    for rep in range(3):
        for s in (a, b):  # new data in the same buffers
            s.tok.copy_(torch.randint(-1, s.v, (s.n, s.t), generator=gen(30 + rep), device=DEV,
                                      dtype=torch.int32))
            s.lengths.copy_(torch.tensor([s.t - rep, 7 * rep, 900], dtype=torch.int32))
            for x in (s.x, s.q, s.s, s.dx, s.grads):
                x.zero_()
            s.ws.fill_(rep)
        kernels(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((a.x, b.x), (a.q, b.q), (a.s, b.s), (a.dx, b.dx), (a.grads, b.grads)):
            assert torch.equal(x, y), rep


@pytest.mark.parametrize("gdtype", ["bf16", "f32"])
def test_layer_workload_takes_its_gradients_on_its_replicas(gdtype):
    w = wl.scaled(wl.WORKLOADS["n8_layer16m_bf16_adam"], n=3, d=(50 + 24) * 72, packet=128,
                  gdtype=gdtype, loss=dict(kind=wl.BERNOULLI, p=0.3),
                  layer=dict(vocab=50, h=72, o=24, t=90))
    dev = wd.DeviceState(w)
    for step in range(3):
        dev.fused(step)  # replicas drift apart
        reps = np64(dev.replicas)
        tok, dy = wl.draw_layer_inputs(w, step + 1, DEV)
        dev.local_gradients(step + 1)
        torch.cuda.synchronize()
        w0 = 50 * 72
        for i in range(3):
            x = ol.embed(tok[i].tolist(), reps[i, :w0].reshape(50, 72), 0, 1.0)
            xq = ol.unpack(*ol.pack(x))
            g = np64(dy[i])
            want, size = ol.wgrad(g, xq, 1.0)
            got = np64(dev.grads[i, w0:w.d]).reshape(24, 72)
            terms = 3 if gdtype == "f32" else 1
            u = half_step(wl.torch_dtype(gdtype))
            assert (np.abs(got - want) <= 1.01 * ((2 * terms * 90 + 2) * U * size
                                                  + u * np.abs(want))).all()
            want, count, size = ol.embed_grad(tok[i].tolist(), np64(dev.dx[i]), 50, 0, 1.0)
            got = np64(dev.grads[i, :w0]).reshape(50, 72)
            assert (np.abs(got - want) <= 1.01 * ((count[:, None] + 2) * U * size
                                                  + u * np.abs(want))).all()
            ref, mag = g @ reps[i, w0:w.d].reshape(24, 72), np.abs(g) @ np.abs(
                reps[i, w0:w.d].reshape(24, 72))
            assert (np.abs(np64(dev.dx[i]) - ref) <= 1.01 * (2 * 24 * U * mag
                                                             + u * np.abs(ref))).all()
    assert not torch.equal(dev.replicas[0], dev.replicas[1])
    assert ll.read_drift(dev.drift)["max_abs"] > 0
