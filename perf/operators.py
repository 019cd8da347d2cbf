"""Performance cases of the workers' local-gradient operators.

Step (1) of the method, for the parts of a language model whose parameters
live in the replica rows and whose gradients go into the gradient rows of the
lossy step: the embedding's lookup and gradient, 8-bit checkpoints of
activations, and a linear layer's weight gradient from such a checkpoint.

A case is a dict of plain values; see `listed` for what each stands for and
`draw` for the ranges.  Sizes are in elements.  n: workers; t: tokens per
worker; vocab: ids the tokens are drawn from; v: table rows held in the shard
(ids from v on belong to another shard); h, o: widths of a layer's input and
output; ragged: the workers' batches end at different lengths.
"""
import math

import torch

# False: elementary torch operations; True: the framework's operators.
own = False

GROUP = 32          # columns of a token that share a scale
E4M3_MAX = 448.0    # largest e4m3 value
MIN_EXP = -117      # smallest exponent of a group's scale


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _esize(name):
    return 2 if name == "bf16" else 4


def _embed(name, n, t, vocab, v, h, dtype, odtype, scale, ragged=False, pad=0):
    return dict(name=name, kind="embed", n=n, t=t, vocab=vocab, v=v, h=h, dtype=dtype,
                odtype=odtype, scale=scale, ragged=ragged, pad=pad)


def _embed_grad(name, n, t, vocab, v, h, dtype, gdtype, scale, ragged=False, pad=0):
    return dict(name=name, kind="embed_grad", n=n, t=t, vocab=vocab, v=v, h=h, dtype=dtype,
                gdtype=gdtype, scale=scale, ragged=ragged, pad=pad)


def _checkpoint(name, n, t, h, dtype, odtype, ragged=False):
    return dict(name=name, kind="checkpoint", n=n, t=t, h=h, dtype=dtype, odtype=odtype,
                ragged=ragged)


def _wgrad(name, n, t, o, h, dtype, gdtype, ragged=False, pad=0):
    return dict(name=name, kind="wgrad", n=n, t=t, o=o, h=h, dtype=dtype, gdtype=gdtype,
                ragged=ragged, pad=pad)


def listed():
    return [
        # A few tokens of four workers with fp32 replicas and a width that is
        # no multiple of a vector: launch latency.
        _embed("embed_n4_t16_h1001_f32", 4, 16, 1000, 1000, 1001, "f32", "f32", 1.0, pad=3),
        # Micro-batches of 8192 tokens on 8 workers, each looked up in the
        # worker's own bf16 replica of a 7B-sized shard (25,695 rows of 4096;
        # ids beyond belong to another shard), scaled by the root of the width.
        _embed("embed_n8_t8192_h4096_bf16", 8, 8192, 32000, 25695, 4096, "bf16", "bf16", 64.0),
        # The gradient of one small micro-batch: a whole table of which most
        # rows are zero.
        _embed_grad("embed_grad_n1_t2048_v32000_bf16", 1, 2048, 32000, 32000, 4096, "bf16",
                    "bf16", 1.0),
        # Eight workers' gradient of the same shard, written into the rows
        # that the lossy step takes.
        _embed_grad("embed_grad_n8_t8192_v25695_bf16", 8, 8192, 32000, 25695, 4096, "bf16",
                    "bf16", 64.0),
        # A small vocabulary (bytes), ragged fp32 batches: many tokens a row.
        _embed_grad("embed_grad_n4_t16001_v259_f32", 4, 16001, 259, 259, 515, "f32", "f32", 1.0,
                    ragged=True, pad=1),
        # Checkpoint written in the forward pass, restored in the backward one.
        # A short sequence on one worker: launch latency.
        _checkpoint("checkpoint_n1_t64_h4096_bf16", 1, 64, 4096, "bf16", "bf16"),
        # A feed-forward layer's inputs of 8 workers.
        _checkpoint("checkpoint_n8_t4096_h11008_bf16", 8, 4096, 11008, "bf16", "bf16"),
        # Ragged fp32 batches of an odd width.
        _checkpoint("checkpoint_n3_t3001_h2051_f32", 3, 3001, 2051, "f32", "f32", ragged=True),
        # A narrow odd layer with fp32 gradients, ragged batches.
        _wgrad("wgrad_n4_t333_o1000_h520_f32", 4, 333, 1000, 520, "f32", "f32", ragged=True,
               pad=5),
        # A square projection, one worker's micro-batch.
        _wgrad("wgrad_n1_t4096_o4096_h4096_bf16", 1, 4096, 4096, 4096, "bf16", "bf16"),
        # A small layer over a long batch: few output tiles, a long sum.
        _wgrad("wgrad_n1_t16384_o512_h1024_bf16", 1, 16384, 512, 1024, "bf16", "f32"),
        # Two workers' feed-forward projection: the largest product.
        _wgrad("wgrad_n2_t8192_o11008_h4096_bf16", 2, 8192, 11008, 4096, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "checkpoint", "wgrad"])
    n = _log(rng, 1, 8)
    dt = rng.choice(["bf16", "f32"])
    other = rng.choice(["bf16", "f32"])
    ragged = rng.random() < 0.3
    pad = rng.choice([0, 0, 1, 8])
    # half of the widths are multiples of a vector, the others any
    h = _log(rng, 33, 8192)
    if rng.random() < 0.5:
        h = max(64, h // 64 * 64)
    if kind in ("embed", "embed_grad"):
        vocab = _log(rng, 50, 64000)
        v = vocab if rng.random() < 0.5 else max(1, int(vocab * rng.uniform(0.3, 1.0)))
        half = 2 if dt == "f32" or other == "f32" else 1  # no more bytes than the largest case's
        h = min(h, max(33, 8 * 25695 * 4096 // (half * n * v)))
        t = min(_log(rng, 1, 32768), max(1, 8 * 8192 * 4096 // (half * n * h)))
        scale = rng.choice([1.0, math.sqrt(h)])
        make = _embed if kind == "embed" else _embed_grad
        return make("", n, t, vocab, v, h, dt, other, scale, ragged, pad)
    if kind == "checkpoint":
        h = min(2 * h, 11008)
        t = min(_log(rng, 1, 16384), max(1, 8 * 4096 * 11008 // (2 * n * h)))
        return _checkpoint("", n, t, h, dt, other, ragged)
    o = _log(rng, 33, 8192)
    if rng.random() < 0.5:
        o = max(64, o // 64 * 64)
    n = min(n, 4)
    limit = 2 * 8192 * 11008 * 4096 // (3 if dt == "f32" else 1)
    t = min(_log(rng, 1, 16384), max(1, limit // (n * o * h)))
    return _wgrad("", n, t, o, h, dt, other, ragged, pad)


# ---- work ----------------------------------------------------------------

def _zipf(vocab):
    """Token frequencies of a language: p(id) ~ 1 / (id + 2.7)."""
    p = 1.0 / (torch.arange(vocab, dtype=torch.float64) + 2.7)
    return p / p.sum()


def _lengths(case):
    """Tokens of each worker's batch."""
    n, t = case["n"], case["t"]
    if not case["ragged"]:
        return [t] * n
    # from a full batch down to about a third, one a worker
    return [max(1, t - (i * 2 * t) // (3 * n)) for i in range(n)]


def work(case):
    lens = _lengths(case)
    tok = sum(lens)
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        h, v = case["h"], case["v"]
        p = _zipf(case["vocab"])[:v]
        held = float(p.sum())
        if kind == "embed":
            rows = sum(float((1.0 - (1.0 - p) ** m).sum()) for m in lens)
            b = tok * 4 + rows * h * _esize(case["dtype"]) + tok * h * _esize(case["odtype"])
            return {"bytes": b, "flops": tok * held * h}
        b = (tok * 4 + tok * held * h * _esize(case["dtype"])
             + case["n"] * v * h * _esize(case["gdtype"]))
        return {"bytes": b, "flops": tok * held * h + case["n"] * v * h}
    if kind == "checkpoint":
        h = case["h"]
        groups = (h + GROUP - 1) // GROUP
        b = tok * (h * (_esize(case["dtype"]) + _esize(case["odtype"])) + 2 * (h + groups))
        return {"bytes": b, "flops": 4 * tok * h}
    o, h = case["o"], case["h"]
    b = (tok * (o * _esize(case["dtype"]) + h + (h + GROUP - 1) // GROUP)
         + case["n"] * o * h * _esize(case["gdtype"]))
    return {"bytes": b, "flops": 2 * tok * o * h}


# ---- inputs --------------------------------------------------------------

def _up(x, m):
    return (x + m - 1) // m * m


def _offset(case):
    # a table or weight behind other parameters of the shard; pad moves it
    # off the vector boundaries
    return 256 + case["pad"]


def _tokens(case, g):
    n, t = case["n"], case["t"]
    # the distribution is summed on the host, in order, and inverted in 64
    # bits, so that a seed always gives the same tokens
    cdf = _zipf(case["vocab"]).cumsum(0).to("cuda")
    u = torch.rand(n * t, generator=g, device="cuda", dtype=torch.float64)
    ids = torch.searchsorted(cdf, u).clamp_max(case["vocab"] - 1)
    return ids.to(torch.int32).view(n, t)


def _activations(shape, g):
    """Normal values with a few channels ten times as large."""
    x = torch.randn(shape, generator=g, device="cuda")
    gain = 1.0 + 9.0 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.01).float()
    return x.mul_(gain)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 17)
    n, t, kind = case["n"], case["t"], case["kind"]
    st = {"case": case}
    if own:
        import paper_2507_07114_amd as ll
        st["ll"] = ll
    lens = _lengths(case)
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda") if case["ragged"] else None
    st["valid"] = (torch.arange(t, device="cuda")[None, :]
                   < torch.tensor(lens, device="cuda")[:, None]) if case["ragged"] else None
    if kind == "embed":
        v, h = case["v"], case["h"]
        st["tokens"] = _tokens(case, g)
        ld = _up(_offset(case) + v * h, 256)
        st["replicas"] = torch.empty((n, ld), dtype=_dtype(case["dtype"]), device="cuda")
        st["replicas"].normal_(0.0, 0.02, generator=g)
        st["out"] = torch.zeros((n, t, h), dtype=_dtype(case["odtype"]), device="cuda")
    elif kind == "embed_grad":
        v, h = case["v"], case["h"]
        st["tokens"] = _tokens(case, g)
        st["dy"] = torch.empty((n, t, h), dtype=_dtype(case["dtype"]), device="cuda")
        st["dy"].normal_(0.0, 1e-3, generator=g)
        ld = _up(_offset(case) + v * h, 256)
        st["grads"] = torch.zeros((n, ld), dtype=_dtype(case["gdtype"]), device="cuda")
        if own:
            st["ws"] = torch.empty(ll.ll_embed_grad_workspace_bytes(n, t, h, v),
                                   dtype=torch.uint8, device="cuda")
    elif kind == "checkpoint":
        h = case["h"]
        st["x"] = _activations((n, t, h), g).to(_dtype(case["dtype"]))
        st["out"] = torch.zeros((n, t, h), dtype=_dtype(case["odtype"]), device="cuda")
        if own:
            st["q"] = torch.empty((n, t, _up(h, 16)), dtype=torch.uint8, device="cuda")[:, :, :h]
            st["s"] = torch.empty((n, t, (h + GROUP - 1) // GROUP), dtype=torch.uint8,
                                  device="cuda")
    else:
        o, h = case["o"], case["h"]
        q = torch.zeros((n, t, _up(h, 16)), dtype=torch.uint8, device="cuda")
        s = torch.zeros((n, t, (h + GROUP - 1) // GROUP), dtype=torch.uint8, device="cuda")
        for i in range(n):
            q[i, :, :h], s[i] = _pack(_activations((t, h), g).to(_dtype(case["dtype"])))
        st["q"], st["s"] = q[:, :, :h], s
        st["dy"] = torch.empty((n, t, o), dtype=_dtype(case["dtype"]), device="cuda")
        st["dy"].normal_(0.0, 1e-3, generator=g)
        ld = _up(_offset(case) + o * h, 256)
        st["grads"] = torch.zeros((n, ld), dtype=_dtype(case["gdtype"]), device="cuda")
        if own:
            st["ws"] = torch.empty(ll.ll_act_wgrad_workspace_bytes(n, t, o, h),
                                   dtype=torch.uint8, device="cuda")
    return st


# ---- plain forms -----------------------------------------------------------

def _pack(x):
    """8-bit form of x [..., h]: e4m3 codes and, a group of 32 columns, the
    exponent byte k + 127 of the smallest power of two 2^k that brings the
    group's largest value to 448 or less."""
    h = x.shape[-1]
    groups = (h + GROUP - 1) // GROUP
    f = x.float()
    if groups * GROUP != h:
        f = torch.nn.functional.pad(f, (0, groups * GROUP - h))
    f = f.reshape(*x.shape[:-1], groups, GROUP)
    m, e = torch.frexp(f.abs().amax(-1))
    k = torch.where(m <= 0.875, e - 9, e - 8).clamp_min(MIN_EXP)
    k = torch.where(m == 0, torch.full_like(k, MIN_EXP), k)
    q = torch.ldexp(f, -k.unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8)
    q = q.reshape(*x.shape[:-1], groups * GROUP)[..., :h]
    return q, (k + 127).to(torch.uint8)


def _unpack(q, s):
    """fp32 values of an 8-bit form."""
    f = q.contiguous().view(torch.float8_e4m3fn).float()
    e = s.to(torch.int32).repeat_interleave(GROUP, -1)[..., : f.shape[-1]] - 127
    return torch.ldexp(f, e)


def _keep(valid, new, old):
    """new where the batch has a token, old behind its end."""
    return new if valid is None else torch.where(valid.unsqueeze(-1), new, old)


def _plain_embed(st):
    c = st["case"]
    v, h, off = c["v"], c["h"], _offset(c)
    n = c["n"]
    table = st["replicas"][:, off:off + v * h].unflatten(1, (v, h))
    ids = st["tokens"].long()
    held = (ids >= 0) & (ids < v)
    rows = table[torch.arange(n, device=ids.device)[:, None], ids.clamp(0, v - 1)]
    y = rows.float() * c["scale"]
    y = torch.where(held.unsqueeze(-1), y, torch.zeros((), device=y.device))
    st["out"].copy_(_keep(st["valid"], y.to(st["out"].dtype), st["out"]))
    return st["out"]


def _plain_embed_grad(st):
    c = st["case"]
    v, h, off, n = c["v"], c["h"], _offset(c), c["n"]
    ids = st["tokens"].long()
    held = (ids >= 0) & (ids < v)
    if st["valid"] is not None:
        held = held & st["valid"]
    # tokens that are not held go to a row of their own behind the table
    rows = torch.where(held, ids, torch.full_like(ids, v))
    view = st["grads"][:, off:off + v * h].unflatten(1, (v, h))
    for i in range(n):
        acc = torch.zeros((v + 1, h), dtype=torch.float32, device=ids.device)
        acc.index_add_(0, rows[i], st["dy"][i].float())
        view[i] = (acc[:v] * c["scale"]).to(view.dtype)
    return view


def _plain_checkpoint(st):
    q, s = _pack(st["x"])
    out = st["out"]
    out.copy_(_keep(st["valid"], _unpack(q, s).to(out.dtype), out))
    return out


def _plain_wgrad(st):
    c = st["case"]
    o, h, off = c["o"], c["h"], _offset(c)
    view = st["grads"][:, off:off + o * h].unflatten(1, (o, h))
    for i, m in enumerate(_lengths(c)):
        x = _unpack(st["q"][i, :m], st["s"][i, :m])
        view[i] = (st["dy"][i, :m].float().t() @ x).to(view.dtype)
    return view


def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        return {"embed": _plain_embed, "embed_grad": _plain_embed_grad,
                "checkpoint": _plain_checkpoint, "wgrad": _plain_wgrad}[kind](state)
    ll = state["ll"]
    lens = state["lengths"]
    if kind == "embed":
        ll.ll_embed(state["tokens"], state["replicas"], state["out"], v=c["v"],
                    offset=_offset(c), scale=c["scale"], lengths=lens)
        return state["out"]
    if kind == "embed_grad":
        ll.ll_embed_grad(state["tokens"], state["dy"], state["grads"], v=c["v"],
                         offset=_offset(c), scale=c["scale"], lengths=lens,
                         workspace=state["ws"])
        off = _offset(c)
        return state["grads"][:, off:off + c["v"] * c["h"]].unflatten(1, (c["v"], c["h"]))
    if kind == "checkpoint":
        ll.ll_act_pack(state["x"], state["q"], state["s"], lengths=lens)
        ll.ll_act_unpack(state["q"], state["s"], state["out"], lengths=lens)
        return state["out"]
    ll.ll_act_wgrad(state["dy"], state["q"], state["s"], state["grads"], offset=_offset(c),
                    lengths=lens, workspace=state["ws"])
    off = _offset(c)
    return state["grads"][:, off:off + c["o"] * c["h"]].unflatten(1, (c["o"], c["h"]))


# ---- 64-bit values -----------------------------------------------------------

def _e4m3_values(x):
    """What the 8-bit form of x [t][h] stands for, in 64 bits: per group of
    32 columns values of 4 significant bits (multiples of 2^(k-9) below
    2^(k-6)) for the smallest k >= -117 with max <= 448 * 2^k."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for a in range(0, x.shape[-1], GROUP):
        y = x[..., a:a + GROUP].double()
        top = y.abs().amax(-1, keepdim=True)
        k = torch.ceil(torch.log2(top / E4M3_MAX)).clamp_min(MIN_EXP)
        z = y / torch.exp2(k)
        exponent = torch.floor(torch.log2(z.abs())).clamp_min(-6.0)
        step = torch.exp2(exponent - 3.0)
        out[..., a:a + GROUP] = torch.round(z / step) * step * torch.exp2(k)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    n, t, kind = case["n"], case["t"], case["kind"]
    lens = _lengths(case)
    if kind == "embed":
        v, h, off = case["v"], case["h"], _offset(case)
        out = torch.zeros((n, t, h), dtype=torch.float64, device="cuda")
        for i in range(n):
            ids = st["tokens"][i, : lens[i]].long()
            at = torch.nonzero((ids >= 0) & (ids < v)).flatten()
            table = st["replicas"][i, off:off + v * h].reshape(v, h)
            out[i].index_copy_(0, at, table.index_select(0, ids[at]).double() * case["scale"])
        return out
    if kind == "embed_grad":
        v, h = case["v"], case["h"]
        out = torch.zeros((n, v, h), dtype=torch.float64, device="cuda")
        for i in range(n):
            ids = st["tokens"][i, : lens[i]].long()
            at = torch.nonzero((ids >= 0) & (ids < v)).flatten()
            out[i].index_put_((ids[at],), st["dy"][i].index_select(0, at).double(),
                              accumulate=True)
        return out.mul_(case["scale"])
    if kind == "checkpoint":
        out = torch.zeros((n, t, case["h"]), dtype=torch.float64, device="cuda")
        for i in range(n):
            out[i, : lens[i]] = _e4m3_values(st["x"][i, : lens[i]])
        return out
    o, h = case["o"], case["h"]
    out = torch.zeros((n, o, h), dtype=torch.float64, device="cuda")
    # code -> value of e4m3, by its definition
    code = torch.arange(256, device="cuda")
    man, ex = (code & 7).double(), ((code >> 3) & 15).double()
    val = torch.where(ex > 0, (1.0 + man / 8.0) * torch.exp2(ex - 7.0), man / 8.0 * 2.0 ** -6)
    val = torch.where(code >= 128, -val, val)
    group = torch.arange(h, device="cuda") // GROUP
    for i in range(n):
        x = val[st["q"][i, : lens[i]].long()]
        x = x * torch.exp2(st["s"][i, : lens[i]].double() - 127.0)[:, group]
        out[i] = torch.matmul(st["dy"][i, : lens[i]].double().t(), x)
    return out
