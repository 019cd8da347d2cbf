"""Every kernel of the weight gradient and of the sorted embedding gradient, on
inputs whose results are exact.

Each case names the form (tiles, runs) that it is meant for and checks that the
call takes it.  Where every partial sum is a whole number (times one power of
two) below 2^24, or all but one term of a sum are 0, the additions are exact in
any order, so the reference is the formula in 64 bits rounded once.
"""
import numpy as np
import pytest
import torch

import paper_2507_07114_amd as ll
import wgrad_plans as wp
from oracle import local as ol
from test_gpu_local import (BF16, DEV, F32, SENTINEL, draw_ids, gen, ints, lengths_of, padded,
                            row_buffer, run_embed_grad, run_wgrad)

pytestmark = pytest.mark.gpu
IDS = lambda c: "x".join(map(str, c[:4]))


def checkpoint_buffers(n, t, h, pq=0, ps=0):
    groups = (h + 31) // 32
    return (padded(n, t, h, h + pq, torch.uint8, fill=0x7F)[1],
            padded(n, t, groups, groups + ps, torch.uint8, fill=255)[1])


def check_form(case, ydt):
    n, t, o, h = case[:4]
    assert wp.plan(ydt == BF16, n, t, o, h).form == case[-2 if ydt == BF16 else -1]


def powers(shape, lo, hi, seed):
    """2^k for whole k from lo to hi, exact."""
    table = torch.tensor([2.0 ** k for k in range(lo, hi + 1)], device=DEV)
    return table[torch.randint(0, hi - lo + 1, shape, generator=gen(seed), device=DEV)]


def check_rows(grads, offset, size, want, old):
    """grads[i][offset: offset + size] as wanted and nothing else touched."""
    assert torch.equal(grads[:, :offset], old[:, :offset])
    assert torch.equal(grads[:, offset + size:], old[:, offset + size:])
    for i, w in enumerate(want):
        assert torch.equal(grads[i, offset:offset + size], w.flatten().to(grads.dtype)), i


@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("ydt,top", [(BF16, 8), (F32, 500)])
@pytest.mark.parametrize("case", wp.CASES, ids=IDS)
def test_act_wgrad_forms(case, ydt, top, gdt):
    # |x| <= 3, |dy| <= top: sums below 8192 * 3 * 500 < 2^24; what they are added to
    # is a multiple of the scale
    n, t, o, h, offset, lens, py, pq, ps = case[:9]
    check_form(case, ydt)
    dl, hl = lengths_of(lens, t, n)
    _, dy = padded(n, t, o, o + py, ydt, fill=float("nan"))
    dy.copy_(ints((n, t, o), -top, top, 60, ydt))
    x = ints((n, t, h), -3, 3, 61, BF16)
    q, s = checkpoint_buffers(n, t, h, pq, ps)
    ll.ll_act_pack(x, q, s)
    for i in range(n):  # behind the batch: not read
        dy[i, hl[i]:] = float("nan")
        q[i, hl[i]:] = 0x7F
    sums = [0.25 * torch.mm(dy[i, :hl[i]].double().t().contiguous(), x[i, :hl[i]].double())
            for i in range(n)]
    grads = row_buffer(n, o * h, offset, gdt)
    for accumulate in (False, True):
        grads.copy_(ints(tuple(grads.shape), -120, 120, 62, gdt))
        old = grads.clone()
        run_wgrad(dy, q, s, grads, offset=offset, scale=0.25, accumulate=accumulate, lengths=dl)
        torch.cuda.synchronize()
        want = sums if not accumulate else [
            a + old[i, offset:offset + o * h].view(o, h).double() for i, a in enumerate(sums)]
        check_rows(grads, offset, o * h, want, old)


def one_token_a_row(n, t, o, hl, value, ydt, py):
    """dy of which each output row has one token, value[i][row], and that token
    [n][o] (row r's lies anywhere in the batch)."""
    _, dy = padded(n, t, o, o + py, ydt)
    dy.zero_()
    r = torch.arange(o, device=DEV)
    at = torch.stack([(r * 7919 + 13 * i) % max(hl[i], 1) for i in range(n)])
    for i in range(n):
        if hl[i]:
            dy[i, at[i], r] = value[i].to(ydt)
    return dy, at


@pytest.mark.parametrize("case", wp.CASES, ids=IDS)
def test_act_wgrad_forms_take_all_bits_of_fp32(case):
    # all 24 bits of dy, times powers of two: one term a sum, so any lost or
    # misplaced bf16 term of it shows
    n, t, o, h, offset, lens, py, pq, ps = case[:9]
    check_form(case, F32)
    dl, hl = lengths_of(lens, t, n)
    odd = torch.randint(1 << 22, 1 << 23, (n, o), generator=gen(63), device=DEV) * 2 + 1
    sign = ints((n, o), 0, 1, 64, F32) * 2 - 1
    value = odd.float() * sign * powers((n, o), -60, 60, 65)
    dy, at = one_token_a_row(n, t, o, hl, value, F32, py)
    x = ints((n, t, h), -1, 1, 66, F32) * powers((n, t, h), -3, 4, 67)
    q, s = checkpoint_buffers(n, t, h, pq, ps)
    ll.ll_act_pack(x, q, s)
    grads = row_buffer(n, o * h, offset, F32)
    old = grads.clone()
    run_wgrad(dy, q, s, grads, offset=offset, lengths=dl)
    torch.cuda.synchronize()
    want = [value[i][:, None].double() * x[i, at[i]].double() if hl[i]
            else torch.zeros((o, h), device=DEV) for i in range(n)]
    check_rows(grads, offset, o * h, want, old)


@pytest.mark.parametrize("ydt", [BF16, F32])
@pytest.mark.parametrize("case", wp.CASES, ids=IDS)
def test_act_wgrad_forms_restore_every_code(case, ydt):
    # dy is 1 at one token of each row: the gradient is the restored value itself,
    # for all codes under every scale that ll_act_pack writes
    n, t, o, h, offset, lens, py, pq, ps = case[:9]
    check_form(case, ydt)
    dl, hl = lengths_of(lens, t, n)
    dy, at = one_token_a_row(n, t, o, hl, torch.ones((n, o), device=DEV), ydt, py)
    q, s = checkpoint_buffers(n, t, h, pq, ps)
    s.copy_(ints(tuple(s.shape), 10, 247, 68, torch.uint8))
    q.copy_(ints((n, t, h), 0, 255, 69, torch.uint8))
    # NaN codes stand in two columns of one worker only, values past 2^128 nowhere
    wide = s.repeat_interleave(ll.LL_ACT_GROUP, 2)[:, :, :h]
    q[(q & 0x7F) == 0x7F] = 0x81
    q[(wide == 247) & ((q & 0x7F) > 0x77)] = 0x77
    if hl[0]:
        q[0, hl[0] // 2, 7], q[0, hl[0] - 1, h - 1] = 0x7F, 0xFF
    grads = row_buffer(n, o * h, offset, F32)
    old = grads.clone()
    run_wgrad(dy, q, s, grads, offset=offset, lengths=dl)
    restored = torch.empty((n, t, h), device=DEV)
    ll.ll_act_unpack(q, s, restored)
    torch.cuda.synchronize()
    assert torch.equal(grads[:, :offset], old[:, :offset])
    assert torch.equal(grads[:, offset + o * h:], old[:, offset + o * h:])
    for i in range(n):
        got = grads[i, offset:offset + o * h].view(o, h)
        if not hl[i]:
            assert not got.any()
            continue
        want = restored[i, at[i]]
        none = torch.zeros(h, dtype=torch.bool, device=DEV)
        if i == 0:  # NaN times 0 is one, too
            none[7] = none[h - 1] = True
            assert torch.isnan(got[:, none]).all()
        assert torch.isfinite(want[:, ~none]).all()
        assert torch.equal(got[:, ~none], want[:, ~none])


FAR = [0, 2, 5, 6, -1, (1 << 32) + 1, -(1 << 32) + 2, (1 << 31) + 3, 1 << 62, -(1 << 63),
       (1 << 63) - 1, (1 << 40) + 4]


@pytest.mark.parametrize("first", [0, 3, -(1 << 63), (1 << 63) - 6, 1 << 32])
@pytest.mark.parametrize("t", [len(FAR) + 6, 300, 600])
def test_ids_far_from_the_table(t, first):
    # ids whose low 32 bits look like rows, and both ends of the 64-bit range, in the
    # lookup and on the ways of few and of many tokens of the gradient
    v, h = 6, 40
    near = [first + k for k in range(v)]
    ids = [int(x) for x in (FAR + near) * (t // len(FAR) + 1)][:t]
    ids = [x if -(1 << 63) <= x < 1 << 63 else 0 for x in ids]
    tok = torch.tensor([ids], dtype=torch.int64, device=DEV)
    table = row_buffer(1, v * h, 0, F32)
    table.copy_(ints(tuple(table.shape), 1, 9, 70, F32))
    out = torch.full((1, t, h), SENTINEL, device=DEV)
    ll.ll_embed(tok, table, out, v=v, first=first)
    rows = table[0, :v * h].view(v, h).double().cpu().numpy()
    assert np.array_equal(out[0].double().cpu().numpy(), ol.embed(ids, rows, first, 1.0))
    dy = ints((1, t, h), -7, 7, 71, F32)
    for accumulate in (False, True):
        grads = row_buffer(1, v * h, 0, F32)
        run_embed_grad(tok, dy, grads, v=v, first=first, accumulate=accumulate)
        want, count, _ = ol.embed_grad(ids, dy[0].double().cpu().numpy(), v, first, 1.0)
        assert count.all()
        want = want + (SENTINEL if accumulate else 0.0)
        assert np.array_equal(grads[0, :v * h].view(v, h).double().cpu().numpy(), want)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,t,h,v", [(64, 1100, 72, 259), (64, 300, 72, 259), (1024, 3, 9, 40),
                                     (1024, 600, 5, 33)])
def test_many_workers(n, t, h, v, accumulate):
    tok = draw_ids("any", n, t, v, 0, False)
    lens = torch.randint(-1, t + 2, (n,), generator=gen(72), device=DEV, dtype=torch.int32)
    dy = ints((n, t, h), -7, 7, 73, BF16)
    grads = row_buffer(n, v * h, 4, F32)
    grads.copy_(ints(tuple(grads.shape), -9, 9, 74, F32))
    old = grads.clone()
    run_embed_grad(tok, dy, grads, v=v, offset=4, lengths=lens, accumulate=accumulate)
    inside = torch.arange(t, device=DEV)[None, :] < lens[:, None]
    at = torch.nonzero((tok >= 0) & (tok < v) & inside)
    want = torch.zeros((n * v, h), dtype=torch.float64, device=DEV)
    want.index_add_(0, at[:, 0] * v + tok[at[:, 0], at[:, 1]], dy[at[:, 0], at[:, 1]].double())
    want = want.view(n, v * h)
    if accumulate:
        want = want + old[:, 4:4 + v * h].double()
    check_rows(grads, 4, v * h, want, old)
    # the other operators at as many workers
    out = torch.full((n, t, h), SENTINEL, device=DEV)
    ll.ll_embed(tok, old, out, v=v, offset=4, lengths=lens)
    rows = old[:, 4:4 + v * h].view(n, v, h)
    held = ((tok >= 0) & (tok < v)).unsqueeze(-1)
    ref = torch.where(held, rows[torch.arange(n, device=DEV)[:, None], tok.clamp(0, v - 1).long()],
                      torch.zeros((), device=DEV))
    assert torch.equal(out, torch.where(inside.unsqueeze(-1), ref, torch.full_like(ref, SENTINEL)))
    q, s = checkpoint_buffers(n, t, h)
    ll.ll_act_pack(out, q, s, lengths=lens)  # whole numbers up to 9: exact
    back = torch.full_like(out, SENTINEL)
    ll.ll_act_unpack(q, s, back, lengths=lens)
    assert torch.equal(back, out)
    o = 6
    dw = ints((n, t, o), -7, 7, 75, BF16)
    wgrad = row_buffer(n, o * h, 0, F32)
    run_wgrad(dw, q, s, wgrad, lengths=lens)
    x = torch.where(inside.unsqueeze(-1), ref, torch.zeros_like(ref))
    want = torch.bmm(dw.double().transpose(1, 2).contiguous(), x.double())
    assert torch.equal(wgrad[:, :o * h].view(n, o, h).double(), want)


@pytest.mark.parametrize("t,o,h", [(40, 16, 64), (600, 4096, 4096)])
@pytest.mark.parametrize("ydt", [BF16, F32])
def test_act_wgrad_of_subnormal_dy(ydt, t, o, h):
    # bf16 keeps 2^-133, and so do the matrix units
    values = [2.0 ** -126, 2.0 ** -127, -(2.0 ** -130), 3 * 2.0 ** -133, 2.0 ** -133]
    if ydt == F32:  # whose terms reach below 2^-126
        values += [(1 + 2.0 ** -23) * 2.0 ** -110, (1 + 2.0 ** -15) * 2.0 ** -118]
    dy = torch.zeros((1, t, o), dtype=ydt, device=DEV)
    dy[0, t // 2, :len(values)] = torch.tensor(values, dtype=torch.float64).to(ydt).to(DEV)
    assert dy[0, t // 2, :len(values)].double().tolist() == values
    q = torch.full((1, t, h), 0x38, dtype=torch.uint8, device=DEV)  # 1.0
    for k in (0, 40):
        s = torch.full((1, t, (h + 31) // 32), 127 + k, dtype=torch.uint8, device=DEV)
        grads = row_buffer(1, o * h, 0, F32)
        run_wgrad(dy, q, s, grads)
        want = dy[0, t // 2].double() * 2.0 ** k
        assert torch.equal(grads[0, :o * h].view(o, h).double(), want[:, None].expand(o, h))
