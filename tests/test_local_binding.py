"""The local-gradient binding on the CPU: what its import needs of torch, and
that each refusal is for its own reason."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2507_07114_amd as ll

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_GPU_NAMES = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2507_07114_amd as ll
tokens = torch.zeros((2, 5), dtype=torch.int32)
try:
    ll.ll_embed(tokens, torch.zeros(2, 80), torch.zeros(2, 5, 8), v=10)
except ValueError as e:
    assert "on one GPU" in str(e), e
else:
    raise AssertionError("tensors on the CPU were taken")
assert ll.ll_workspace_bytes(2, 100, 10) > 0
print("ok")
"""


def test_import_with_a_torch_without_gpu_support():
    # such a torch lacks the private names that read the current stream; it has
    # no GPU tensors, so no call gets as far as them
    r = subprocess.run([sys.executable, "-c", WITHOUT_GPU_NAMES], cwd=ROOT, capture_output=True,
                       text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


U8, I32 = torch.uint8, torch.int32
TOK, OUT, ROWS = _t(2, 5, dtype=I32), _t(2, 5, 8), _t(2, 80)
Q, S = _t(2, 5, 8, dtype=U8), _t(2, 5, 1, dtype=U8)


def embed(tok=TOK, rows=ROWS, out=OUT, **kw):
    ll.ll_embed(tok, rows, out, **{"v": 10, **kw})


def embed_grad(tok=TOK, dy=OUT, rows=ROWS, **kw):
    ll.ll_embed_grad(tok, dy, rows, **{"v": 10, **kw})


def wgrad(dy=OUT, q=Q, s=S, rows=ROWS, **kw):
    ll.ll_act_wgrad(dy, q, s, rows, **kw)


# All tensors here are on the CPU, which by itself is refused, too: only the message
# tells that a tensor was refused for what is wrong with it.
REFUSED = [
    (embed, dict(tok=TOK[0]), "tokens must be 2-D"),
    (embed, dict(tok=TOK.float()), "tokens must be one of"),
    (embed, dict(tok=TOK.t().contiguous().t()), "tokens must have unit column stride"),
    (embed, dict(rows=ROWS[:1]), r"replicas must be \[2\]\[ld\]"),
    (embed, dict(rows=ROWS[0]), r"replicas must be \[2\]\[ld\]"),
    (embed, dict(rows=_t(2, 160)[:, ::2]), "replicas must have unit column stride"),
    (embed, dict(rows=ROWS.half()), "replicas must be one of"),
    (embed, dict(out=OUT[:, :4]), r"out must be \[2\]\[5\]"),
    (embed, dict(out=OUT[0]), r"out must be \[2\]\[5\]"),
    (embed, dict(out=OUT.half()), "out must be one of"),
    (embed, dict(out=_t(2, 5, 16)[..., ::2]), "out must have unit column stride"),
    (embed, dict(out=_t(2, 6, 8)[:, :5]), "workers must lie 5 rows apart"),
    (embed, dict(out=_t(5, 2, 8).transpose(0, 1)), "workers must lie 5 rows apart"),
    (embed, dict(v=11), "exceed its 80 columns"),
    (embed, dict(offset=1), "exceed its 80 columns"),
    (embed, dict(offset=-1), "offset -1 exceed"),
    (embed, dict(lengths=_t(1, dtype=I32)), "lengths"),
    (embed, dict(lengths=_t(2, dtype=torch.int64)), "lengths"),
    (embed, dict(lengths=_t(4, dtype=I32)[::2]), "lengths must be contiguous"),
    (embed, dict(), "on one GPU"),
    (embed_grad, dict(dy=OUT[:, :4]), r"dy must be \[2\]\[5\]"),
    (embed_grad, dict(dy=OUT.double()), "dy must be one of"),
    (embed_grad, dict(rows=ROWS.half()), "grads must be one of"),
    (embed_grad, dict(v=11), "exceed its 80 columns"),
    (embed_grad, dict(workspace=_t(64, dtype=U8)[::2]), "workspace must be contiguous"),
    (embed_grad, dict(), "on one GPU"),
    (wgrad, dict(dy=OUT[0]), "must be 3-D"),
    (wgrad, dict(q=Q[0]), "must be 3-D"),
    (wgrad, dict(q=Q.float()), "q must be uint8"),
    (wgrad, dict(s=S.float()), "s must be uint8"),
    (wgrad, dict(q=Q[:, :4]), r"q must be \[2\]\[5\]"),
    (wgrad, dict(s=_t(2, 5, 2, dtype=U8)), "s must have width 1"),
    (wgrad, dict(rows=_t(2, 56)), "exceed its 56 columns"),
    (wgrad, dict(rows=_t(3, 80)), r"grads must be \[2\]\[ld\]"),
    (wgrad, dict(), "on one GPU"),
    (ll.ll_act_pack, dict(x=OUT[0], q=Q, s=S), "x must be 3-D"),
    (ll.ll_act_pack, dict(x=OUT.half(), q=Q, s=S), "x must be one of"),
    (ll.ll_act_pack, dict(x=OUT, q=_t(2, 5, 9, dtype=U8), s=S), "q must have width 8"),
    (ll.ll_act_pack, dict(x=OUT, q=Q, s=_t(2, 5, 2, dtype=U8)), "s must have width 1"),
    (ll.ll_act_pack, dict(x=OUT, q=OUT, s=S), "q must be uint8"),
    (ll.ll_act_pack, dict(x=OUT, q=Q, s=S), "on one GPU"),
    (ll.ll_act_unpack, dict(q=Q, s=S, out=OUT[0]), "out must be 3-D"),
    (ll.ll_act_unpack, dict(q=Q, s=_t(2, 5, 1), out=OUT), "s must be uint8"),
    (ll.ll_act_unpack, dict(q=Q, s=S, out=OUT), "on one GPU"),
]


@pytest.mark.parametrize("call,args,reason", REFUSED)
def test_refusals_name_their_reason(call, args, reason):
    with pytest.raises(ValueError, match=reason):
        call(**args)
