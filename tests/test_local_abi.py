"""C ABI of the local-gradient operators (CPU only): the header is C99, every
entry point is exported and bound, bad arguments are refused before any device
work (no call here reaches a kernel launch), and the binding refuses tensors
that do not fit."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2507_07114_amd as ll

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lossy_local.h")


def _declared():
    return re.findall(r"^LL_API\s+[\w\s\*]*?\b(\w+)\s*\(", open(HEADER).read(), flags=re.M)


def test_header_library_and_binding_agree():
    names = set(_declared())
    assert names == {"ll_embed", "ll_embed_grad", "ll_embed_grad_workspace_bytes", "ll_act_pack",
                     "ll_act_unpack", "ll_act_wgrad", "ll_act_wgrad_workspace_bytes"}
    lib = ctypes.CDLL(ll.library_path())
    for name in names:
        assert hasattr(lib, name) and callable(getattr(ll, name)) and name in ll.__all__


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_header_is_c99(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "lossy_local.h"\nint main(void) { return LL_ACT_GROUP - 32 + LL_I32; }\n')
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic",
                          f"-I{os.path.join(ROOT, 'include')}", str(src), "-o",
                          str(tmp_path / "use")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr


# Valid arguments by name, in C order; 16 and 32 stand for addresses.  No
# test calls an entry point with arguments that pass all checks.
P = 1 << 20
EMBED = dict(n=2, t=5, h=8, v=10, first=0, itype=0, tokens=P, ld_t=5, lengths=None, rdtype=1,
             replicas=P, ld_r=80, offset=0, scale=1.0, odtype=1, out=P, ld_o=8, stream=None)
GRAD = dict(n=2, t=5, h=8, v=10, first=0, itype=0, tokens=P, ld_t=5, lengths=None, ydtype=1,
            dy=P, ld_y=8, scale=1.0, gdtype=1, grads=P, ld_g=80, offset=0, accumulate=0,
            workspace=P, ws_bytes=1 << 40, stream=None)
PACK = dict(n=2, t=5, h=40, lengths=None, xdtype=1, x=P, ld_x=40, q=P, ld_q=40, s=P, ld_s=2,
            stream=None)
UNPACK = dict(n=2, t=5, h=40, lengths=None, q=P, ld_q=40, s=P, ld_s=2, odtype=1, out=P, ld_o=40,
              stream=None)
WGRAD = dict(n=2, t=5, o=3, h=40, lengths=None, ydtype=1, dy=P, ld_y=3, q=P, ld_q=40, s=P, ld_s=2,
             scale=1.0, gdtype=1, grads=P, ld_g=120, offset=0, accumulate=0, workspace=P,
             ws_bytes=1 << 40, stream=None)
BASE = {"ll_embed": EMBED, "ll_embed_grad": GRAD, "ll_act_pack": PACK, "ll_act_unpack": UNPACK,
        "ll_act_wgrad": WGRAD}

COMMON = [(dict(n=0), -1, "n=0"), (dict(n=1025), -1, "n=1025"), (dict(t=-1), -1, "negative"),
          (dict(t=1 << 30), -1, "n * t"), (dict(h=0), -1, "h=0"), (dict(h=1 << 31), -1, "h="),
          (dict(lengths=P + 2), -2, "lengths")]
TOKENS = [(dict(itype=2), -1, "itype"), (dict(tokens=None), -1, "tokens is NULL"),
          (dict(ld_t=4), -1, "tokens: ld=4"), (dict(tokens=P + 4, itype=1), -2, "tokens"),
          (dict(v=0), -1, "v=0"), (dict(v=1 << 31), -1, "v=")]
CASES = [(f, *c) for f in BASE for c in COMMON]
CASES += [(f, *c) for f in ("ll_embed", "ll_embed_grad") for c in TOKENS]
CASES += [("ll_embed", *c) for c in [
    (dict(rdtype=2), -1, "replicas: unknown dtype"), (dict(odtype=-1), -1, "odtype"),
    (dict(replicas=None), -1, "replicas is NULL"), (dict(replicas=P + 2), -2, "replicas"),
    (dict(offset=-1), -1, "offset=-1"), (dict(offset=1), -1, "exceed"), (dict(ld_r=72), -1, "exceed"),
    (dict(ld_r=84), -2, "multiple of 16"), (dict(out=None), -1, "out is NULL"),
    (dict(offset=(1 << 63) - 1), -1, "exceed"), (dict(v=(1 << 31) - 1), -1, "exceed"),
    (dict(ld_o=7), -1, "out: ld=7"), (dict(out=P + 1), -2, "out")]]
CASES += [("ll_embed_grad", *c) for c in [
    (dict(gdtype=2), -1, "grads: unknown dtype"), (dict(ydtype=3), -1, "ydtype"),
    (dict(grads=None), -1, "grads is NULL"), (dict(offset=8), -1, "exceed"),
    (dict(dy=None), -1, "dy is NULL"), (dict(dy=P + 2, ydtype=0), -2, "dy"),
    (dict(ld_y=7), -1, "dy: ld=7")]]
CASES += [("ll_act_pack", *c) for c in [
    (dict(xdtype=5), -1, "xdtype"), (dict(x=None), -1, "x is NULL"), (dict(ld_x=39), -1, "x: ld"),
    (dict(q=None), -1, "q is NULL"), (dict(s=None), -1, "s is NULL"), (dict(ld_q=39), -1, "q: ld"),
    (dict(ld_s=1), -1, "s: ld=1"), (dict(x=P + 1), -2, "x")]]
CASES += [("ll_act_unpack", *c) for c in [
    (dict(odtype=5), -1, "odtype"), (dict(out=None), -1, "out is NULL"),
    (dict(ld_o=39), -1, "out: ld"), (dict(q=None), -1, "q is NULL"), (dict(ld_s=1), -1, "s: ld=1"),
    (dict(out=P + 2, odtype=0), -2, "out")]]
CASES += [("ll_act_wgrad", *c) for c in [
    (dict(o=0), -1, "o=0"), (dict(gdtype=2), -1, "grads: unknown dtype"),
    (dict(ydtype=3), -1, "ydtype"), (dict(grads=None), -1, "grads is NULL"),
    (dict(offset=8), -1, "exceed"), (dict(dy=None), -1, "dy is NULL"),
    (dict(ld_y=2), -1, "dy: ld=2"), (dict(q=None), -1, "q is NULL"), (dict(s=None), -1, "s is NULL"),
    (dict(ld_q=39), -1, "q: ld"), (dict(ld_g=124), -2, "multiple of 16"),
    (dict(ld_y=1 << 24), -1, "2^24"), (dict(ld_q=1 << 24), -1, "2^24"),
    (dict(ld_s=1 << 24), -1, "2^24")]]
# more workgroups than a grid holds
CASES += [("ll_embed_grad", dict(n=1024, t=300, h=1, v=1 << 24, ld_t=300, ld_y=1, ld_g=1 << 24), -1,
           "too many workgroups"),
          ("ll_act_wgrad", dict(n=1024, t=1, o=1 << 20, h=1 << 7, ld_y=1 << 20, ld_q=1 << 7, ld_s=4,
                                ld_g=1 << 27), -1, "too many workgroups")]


@pytest.mark.parametrize("func,change,code,frag", CASES)
def test_refusals(func, change, code, frag):
    args = dict(BASE[func])
    args.update(change)
    f = getattr(ll._load(), func)
    assert f(*args.values()) == code
    assert frag in ll.ll_last_error()


def test_workspace_is_checked():
    for func, size in (("ll_embed_grad", (300, 20000, 512, 5000)),
                       ("ll_act_wgrad", (1, 100000, 64, 64))):
        need = getattr(ll, func + "_workspace_bytes")(*size)
        if need == 0:
            continue
        a = dict(BASE[func])
        n, t, w, x = size
        a.update(dict(n=n, t=t, h=w, v=x, ld_t=t, ld_y=w, ld_g=w * x) if func == "ll_embed_grad"
                 else dict(n=n, t=t, o=w, h=x, ld_y=w, ld_q=x, ld_s=x, ld_g=w * x))
        for change, code in ((dict(ws_bytes=need - 1), -1), (dict(workspace=None), -1),
                             (dict(workspace=P + 8), -2)):
            b = dict(a)
            b.update(change)
            assert getattr(ll._load(), func)(*b.values()) == code, change
            assert "workspace" in ll.ll_last_error()
    assert ll.ll_embed_grad_workspace_bytes(0, 1, 1, 1) == 0
    assert ll.ll_act_wgrad_workspace_bytes(1, -1, 1, 1) == 0


def test_no_tokens_is_a_no_op_for_the_token_rows():
    for func in ("ll_embed", "ll_act_pack", "ll_act_unpack"):
        a = dict(BASE[func])
        a.update(t=0)
        for k in ("tokens", "out", "x", "q", "s"):
            if k in a:
                a[k] = None
        assert getattr(ll._load(), func)(*a.values()) == 0


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses_tensors_that_do_not_fit():
    i32, u8 = torch.int32, torch.uint8
    tok, out, rows = _t(2, 5, dtype=i32), _t(2, 5, 8), _t(2, 80)
    bad = [
        lambda: ll.ll_embed(tok[0], rows, out, v=10),
        lambda: ll.ll_embed(tok.float(), rows, out, v=10),
        lambda: ll.ll_embed(tok.t().contiguous().t(), rows, out, v=10),
        lambda: ll.ll_embed(tok, rows[:1], out, v=10),
        lambda: ll.ll_embed(tok, rows, out[:, :4], v=10),
        lambda: ll.ll_embed(tok, rows, out.half(), v=10),
        lambda: ll.ll_embed(tok, rows, out, v=11),
        lambda: ll.ll_embed(tok, rows, out, v=10, offset=1),
        lambda: ll.ll_embed(tok, rows, out, v=10, offset=-1),
        lambda: ll.ll_embed(tok, rows, _t(2, 5, 16)[..., ::2], v=10),
        lambda: ll.ll_embed(tok, rows, _t(2, 6, 8)[:, :5], v=10),
        lambda: ll.ll_embed(tok, rows, out, v=10, lengths=_t(1, dtype=i32)),
        lambda: ll.ll_embed(tok, rows, out, v=10, lengths=_t(2, dtype=torch.int64)),
        lambda: ll.ll_embed(tok, rows, out, v=10),  # not on a GPU
        lambda: ll.ll_embed_grad(tok, out, rows, v=11),
        lambda: ll.ll_embed_grad(tok, out, rows.half(), v=10),
        lambda: ll.ll_embed_grad(tok, out, rows, v=10),
        lambda: ll.ll_act_pack(out[0], _t(2, 5, 8, dtype=u8), _t(2, 5, 1, dtype=u8)),
        lambda: ll.ll_act_pack(out, _t(2, 5, 9, dtype=u8), _t(2, 5, 1, dtype=u8)),
        lambda: ll.ll_act_pack(out, _t(2, 5, 8, dtype=u8), _t(2, 5, 2, dtype=u8)),
        lambda: ll.ll_act_pack(out, _t(2, 5, 8), _t(2, 5, 1, dtype=u8)),
        lambda: ll.ll_act_unpack(_t(2, 5, 8, dtype=u8), _t(2, 5, 1), out),
        lambda: ll.ll_act_wgrad(out, _t(2, 5, 8, dtype=u8), _t(2, 5, 1, dtype=u8), _t(2, 56)),
        lambda: ll.ll_act_wgrad(out, _t(2, 4, 8, dtype=u8), _t(2, 4, 1, dtype=u8), _t(2, 64)),
        lambda: ll.ll_act_wgrad(out, _t(2, 5, 8, dtype=u8), _t(2, 5, 1, dtype=u8), _t(2, 64)),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print(f"call {k} was not refused")


def test_layer_workload_inputs():
    import workloads as wl
    w = wl.WORKLOADS["n8_layer16m_bf16_adam"]
    assert (w.layer["vocab"] + w.layer["o"]) * w.layer["h"] == w.d
    w = wl.scaled(w, n=2, layer=dict(vocab=100, h=8, o=5, t=4000))
    a, b = wl.draw_layer_inputs(w, 3), wl.draw_layer_inputs(w, 3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not torch.equal(a[0], wl.draw_layer_inputs(w, 4)[0])
    assert a[0].dtype == torch.int32 and tuple(a[0].shape) == (2, 4000)
    assert int(a[0].min()) >= 0 and int(a[0].max()) < 100
    assert a[1].dtype == torch.bfloat16 and tuple(a[1].shape) == (2, 4000, 5)
    p0 = (1 / 2.7) / sum(1 / (k + 2.7) for k in range(100))  # the commonest id
    share = float((a[0] == 0).float().mean())
    assert abs(share - p0) < 5 * (p0 * (1 - p0) / 8000) ** 0.5
