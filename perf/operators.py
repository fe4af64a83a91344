"""Performance cases of the operators of a pre-norm self-attention block: layer norm, multi-head attention with a learned
relative position bias by buckets, and activation checkpoints in 8 bits with their use in the backward pass.

Four kinds of pass, each as a user's program makes it:

  norm    layer norm: forward, and for training also the backward pass with the gradients of weight and bias; the input is
          kept for the backward pass as it is, or as a checkpoint in 8 bits that the forward pass writes on its way
  ckpt    a tensor to its checkpoint and back: a stash slot filled in F and emptied in B
  wgrad   the weight gradient of a projection whose input was kept as a checkpoint: packed in F, read in B
  attn    attention: forward (a prompt, or single tokens against a long cache), or forward and backward with the gradient
          of the bias table

`run` computes them from elementary torch operations in 32 bits, or (own) with the package's entry points.
"""
import math

import torch

own = False

BLOCK = 32          # channels of a row that share a checkpoint's exponent


def listed():
    return [
        # the norm in front of a classifier of a few tokens, evaluation: latency
        dict(name="norm_eval_few_rows", kind="norm", dtype="f32", rows=7, channels=256, train=False, keep8=False),
        # a training micro-batch of a narrow float model with an odd width
        dict(name="norm_train_f32_odd", kind="norm", dtype="f32", rows=10007, channels=515, train=True, keep8=False),
        # an ordinary training micro-batch, input kept as it is
        dict(name="norm_train_bf16", kind="norm", dtype="bf16", rows=8192, channels=1024, train=True, keep8=False),
        # a large one, input kept in 8 bits
        dict(name="norm_train_bf16_kept8", kind="norm", dtype="bf16", rows=65536, channels=2048, train=True, keep8=True),
        # a stash slot of a wide residual stage: out to 8 bits and back
        dict(name="ckpt_bf16", kind="ckpt", dtype="bf16", rows=100352, channels=1000),
        # the projection behind a norm: its input kept in 8 bits
        dict(name="wgrad_bf16_kept8", kind="wgrad", dtype="bf16", rows=16384, channels=1024, outputs=1024),
        # a training micro-batch of an encoder of 512 tokens, some sequences shorter, 32 buckets up to distance 128; packed q | k | v
        dict(name="attn_train_512", kind="attn", dtype="bf16", m=8, heads=12, kv_heads=12, pq=512, pk=512, d=64, causal=False, lengths="ragged",
             buckets=32, reach=128, packed=True, train=True),
        # long sequences, causal, key and value heads shared by four query heads
        dict(name="attn_train_long_causal", kind="attn", dtype="bf16", m=1, heads=16, kv_heads=4, pq=8192, pk=8192, d=128, causal=True, lengths="full",
             buckets=32, reach=128, packed=False, train=True),
        # odd everything: cross-attention, a sample without keys, a head of 40 channels
        dict(name="attn_train_odd", kind="attn", dtype="bf16", m=5, heads=6, kv_heads=3, pq=333, pk=777, d=40, causal=False, lengths="ragged0",
             buckets=16, reach=60, packed=False, train=True),
        # float: the volumetric network's attention size
        dict(name="attn_train_f32", kind="attn", dtype="f32", m=2, heads=4, kv_heads=4, pq=512, pk=512, d=32, causal=False, lengths="full",
             buckets=32, reach=128, packed=True, train=True),
        # evaluation of a prompt
        dict(name="attn_prompt", kind="attn", dtype="bf16", m=4, heads=16, kv_heads=16, pq=2048, pk=2048, d=64, causal=True, lengths="full",
             buckets=32, reach=128, packed=True, train=False),
        # single tokens against caches of up to 16384 positions, shared heads
        dict(name="attn_single_token", kind="attn", dtype="bf16", m=16, heads=32, kv_heads=8, pq=1, pk=16384, d=128, causal=True, lengths="cache",
             buckets=32, reach=128, packed=False, train=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("norm", "ckpt", "wgrad", "attn"), (4, 1, 2, 6))[0]
    dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
    es = 2 if dtype == "bf16" else 4
    if kind == "norm":
        channels = rng.choice((_log(rng, 16, 8192), 8 * _log(rng, 4, 1024)))
        rows = min(_log(rng, 1, 100000), max(1, int(2.6e8 / es / channels)))
        train = rng.random() < 0.7
        return dict(kind=kind, dtype=dtype, rows=rows, channels=channels, train=train, keep8=train and rng.random() < 0.5)
    if kind == "ckpt":
        channels = rng.choice((_log(rng, 16, 8192), 8 * _log(rng, 4, 1024)))
        return dict(kind=kind, dtype=dtype, rows=min(_log(rng, 64, 100000), max(1, int(2e8 / es / channels))), channels=channels)
    if kind == "wgrad":
        channels, outputs = 8 * _log(rng, 4, 192), 8 * _log(rng, 4, 192)
        most = (3.4e10 if dtype == "bf16" else 4e9) / channels / outputs
        return dict(kind=kind, dtype=dtype, rows=min(_log(rng, 64, 65536), max(64, int(most))), channels=channels, outputs=outputs)
    group = rng.choice((1, 1, 2, 4))
    kv_heads = _log(rng, 1, 8)
    heads, d = kv_heads * group, rng.choice((32, 64, 64, 128, 8 * rng.randint(2, 16), rng.randint(16, 128)))
    buckets = rng.choice((8, 16, 32, 64))
    reach = rng.choice((32, 128, 128, 256, _log(rng, 16, 1024)))
    c = dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, d=d, buckets=buckets, reach=reach)
    shape = rng.choices(("self", "cross", "single"), (6, 2, 2))[0]
    if shape == "single":
        pk = _log(rng, 64, 16384)
        return dict(c, m=min(_log(rng, 1, 32), max(1, int(2.5e8 / es / (pk * kv_heads * d)))), pq=rng.choice((1, 1, 2, 4)), pk=pk, causal=True,
                    lengths="cache", packed=False, train=False)
    top = 4.5e11 if dtype == "bf16" else 6e10          # multiply-adds of both directions
    pq = _log(rng, 16, 4096)
    pk = pq if shape == "self" else _log(rng, 16, 4096)
    while 7 * heads * pq * pk * d > top:
        pq, pk = max(16, pq // 2), max(16, pk // 2)
    m = max(1, min(_log(rng, 1, 16), int(top / (7 * heads * pq * pk * d))))
    return dict(c, m=m, pq=pq, pk=pk, causal=shape == "self" and rng.random() < 0.5, lengths=rng.choice(("full", "ragged", "ragged0" if m > 1 else "ragged")),
                packed=shape == "self" and group == 1 and rng.random() < 0.5, train=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------- inputs
def _tdt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _activations(gen, rows, channels, tdt):
    """A residual stream: rows of unequal size and mean, a few channels much larger than the rest."""
    x = torch.randn(rows, channels, generator=gen, device="cuda")
    x *= torch.rand(rows, 1, generator=gen, device="cuda") + 0.5
    x += 0.3 * torch.randn(rows, 1, generator=gen, device="cuda")
    x *= 1 + 7 * (torch.rand(channels, generator=gen, device="cuda") > 0.99).float()
    return x.to(tdt)


def _gradient(gen, shape, tdt):
    return (1e-3 * torch.randn(shape, generator=gen, device="cuda")).to(tdt)


def bucket_map(buckets, reach, causal):
    """Bucket of every offset key - query from -reach to reach: half of a side's buckets for the nearest offsets, one each, the
    others in steps of their logarithm; both sides have half of the buckets each, or the past has all of them."""
    n = buckets if causal else buckets // 2
    exact = max(1, n // 2)
    out = []
    for rel in range(-reach, reach + 1):
        base = 0 if causal or rel <= 0 else n
        r = max(0, -rel) if causal else abs(rel)
        if r >= exact:
            r = min(n - 1, exact + int(math.log(r / exact) / math.log(max(reach, exact + 1) / exact) * (n - exact)))
        out.append(base + r)
    return out


def _lengths(c, gen):
    """Keys of every sample, and the position of its first query."""
    m, pq, pk = c["m"], c["pq"], c["pk"]
    if c["lengths"] == "full":
        n = torch.full((m,), pk, dtype=torch.int32, device="cuda")
    elif c["lengths"] == "cache":
        n = (torch.rand(m, generator=gen, device="cuda") * (pk // 2 + 1)).to(torch.int32) + (pk - pk // 2)
        n.clamp_(pq, pk)
    else:
        n = (torch.rand(m, generator=gen, device="cuda") * (pk - pk // 2 + 1)).to(torch.int32) + pk // 2
        n.clamp_(1, pk)
        if c["lengths"] == "ragged0":
            n[m // 2] = 0
    start = (n - pq) if c["lengths"] == "cache" else torch.zeros(m, dtype=torch.int32, device="cuda")
    return n, start


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c, tdt = case, _tdt(case)
    s = dict(c=c)
    if c["kind"] == "attn":
        m, H, G, pq, pk, d = c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"]
        if c["packed"]:
            x = torch.randn(m, pq, 3 * H * d, generator=gen, device="cuda").to(tdt)
            s["x"], s["q"], s["k"], s["v"] = x, x[:, :, :H * d], x[:, :, H * d:2 * H * d], x[:, :, 2 * H * d:]
        else:
            s["q"] = torch.randn(m, pq, H * d, generator=gen, device="cuda").to(tdt)
            s["k"] = torch.randn(m, pk, G * d, generator=gen, device="cuda").to(tdt)
            s["v"] = torch.randn(m, pk, G * d, generator=gen, device="cuda").to(tdt)
        s["table"] = torch.randn(H, c["buckets"], generator=gen, device="cuda")
        s["map"] = torch.tensor(bucket_map(c["buckets"], c["reach"], c["causal"]), dtype=torch.int32, device="cuda")
        s["len"], s["start"] = _lengths(c, gen)
        if c["train"]:
            s["dy"] = _gradient(gen, (m, pq, H * d), tdt)
            if c["lengths"] != "full" and pq == pk:         # padding takes no part in the loss
                s["dy"] *= (torch.arange(pq, device="cuda")[None, :, None] < s["len"][:, None, None])
    else:
        s["x"] = _activations(gen, c["rows"], c["channels"], tdt)
        if c["kind"] == "norm":
            s["gamma"] = 1 + 0.1 * torch.randn(c["channels"], generator=gen, device="cuda")
            s["beta"] = 0.1 * torch.randn(c["channels"], generator=gen, device="cuda")
            if c["train"]:
                s["dy"] = _gradient(gen, (c["rows"], c["channels"]), tdt)
        if c["kind"] == "wgrad":
            s["dz"] = _gradient(gen, (c["rows"], c["outputs"]), tdt)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The output buffers, stash and scratch that a program keeps beside the inputs."""
    import paper_2207_11019_amd as lpm
    c = s["c"]
    dt = lpm.BF16 if c["dtype"] == "bf16" else lpm.F32
    buf = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")      # noqa: E731
    s["lpm"], s["dt"] = lpm, dt
    if c["kind"] == "attn":
        ld = 3 * c["heads"] * c["d"] if c["packed"] else 0
        s["g"] = lpm.lpm_attn_geom(m=c["m"], heads=c["heads"], kv_heads=c["kv_heads"], pq=c["pq"], pk=c["pk"], d=c["d"], causal=c["causal"],
                                   ldq=ld, ldk=ld, ldv=ld, n_buckets=c["buckets"], reach=c["reach"])
        fwd, bwd = lpm.lpm_attn_ws_bytes(s["g"], dt)
        s["y"] = torch.empty(c["m"], c["pq"], c["heads"] * c["d"], dtype=_tdt(c), device="cuda")
        s["ws"] = buf(max(fwd, bwd if c["train"] else 0))
        s["stats"] = buf(lpm.lpm_attn_stats_bytes(s["g"], dt)) if c["train"] else None
        if c["train"]:
            H = c["heads"] * c["d"]
            if c["packed"]:
                s["dx"] = torch.empty_like(s["x"])
                s["dq"], s["dk"], s["dv"] = s["dx"][:, :, :H], s["dx"][:, :, H:2 * H], s["dx"][:, :, 2 * H:]
            else:
                s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
            s["dtable"] = torch.empty_like(s["table"])
        return
    rows, channels = c["rows"], c["channels"]
    if c["kind"] == "norm":
        s["y"] = torch.empty_like(s["x"])
        if c["train"]:
            s["stats"], s["dx"] = torch.empty(rows, 2, device="cuda"), torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
            s["ws"] = buf(lpm.lpm_norm_ws_bytes(rows, channels, dt))
    if c["kind"] != "norm" or c["keep8"]:
        s["kept"] = buf(lpm.lpm_ckpt8_bytes(rows, channels))
    if c["kind"] == "ckpt":
        s["back"] = torch.empty_like(s["x"])
    if c["kind"] == "wgrad":
        s["geom"] = dict(m=rows, h=1, w=1, cin=channels, cout=c["outputs"], kh=1, kw=1, stride=1, pad=0)
        s["dw"] = torch.empty(c["outputs"], channels, device="cuda")
        s["ws"] = buf(lpm.lpm_conv_wgrad_ckpt8_ws_bytes(s["geom"], dt))


# ---------------------------------------------------------------------------------------------- one pass, the package's operators
def _run_own(s):
    lpm, c, dt, st = s["lpm"], s["c"], s["dt"], torch.cuda.current_stream()
    if c["kind"] == "norm":
        rows, ch = c["rows"], c["channels"]
        if not c["train"]:
            lpm.lpm_norm_forward(rows, ch, dt, s["x"], s["gamma"], s["beta"], 1e-5, s["y"], stream=st)
            return dict(y=s["y"])
        kept = s["kept"] if c["keep8"] else None
        lpm.lpm_norm_forward(rows, ch, dt, s["x"], s["gamma"], s["beta"], 1e-5, s["y"], s["stats"], kept, st)
        lpm.lpm_norm_backward(rows, ch, dt, None if c["keep8"] else s["x"], kept, s["stats"], s["dy"], s["gamma"], s["dx"], s["dgamma"], s["dbeta"],
                              ws=s["ws"], stream=st)
        return dict(y=s["y"], dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    if c["kind"] == "ckpt":
        lpm.lpm_ckpt8_pack(c["rows"], c["channels"], dt, s["x"], s["kept"], st)
        lpm.lpm_ckpt8_unpack(c["rows"], c["channels"], dt, s["kept"], s["back"], st)
        return dict(x=s["back"])
    if c["kind"] == "wgrad":
        lpm.lpm_ckpt8_pack(c["rows"], c["channels"], dt, s["x"], s["kept"], st)
        lpm.lpm_conv_wgrad_ckpt8(s["geom"], dt, s["kept"], s["dz"], s["dw"], False, s["ws"], st)
        return dict(dw=s["dw"])
    lpm.lpm_attn_forward(s["g"], dt, s["q"], s["k"], s["v"], s["len"], s["start"], s["map"], s["table"], s["y"], s["stats"], s["ws"], st)
    if not c["train"]:
        return dict(y=s["y"])
    lpm.lpm_attn_backward(s["g"], dt, s["q"], s["k"], s["v"], s["y"], s["stats"], s["dy"], s["len"], s["start"], s["map"], s["table"],
                          s["dq"], s["dk"], s["dv"], s["dtable"], False, s["ws"], st)
    return dict(y=s["y"], dq=s["dq"], dk=s["dk"], dv=s["dv"], dtable=s["dtable"])


# ---------------------------------------------------------------------------------------------- one pass, elementary operations
def _kept8(x):
    """What the checkpoint of x stands for (float)."""
    rows, ch = x.shape
    full = torch.zeros(rows, (ch + BLOCK - 1) // BLOCK * BLOCK, device=x.device)
    full[:, :ch] = x.float()
    b = full.view(rows, -1, BLOCK)
    top = b.abs().amax(2, keepdim=True)
    mant, ex = torch.frexp(top)                              # top = mant 2^ex, 1/2 <= mant < 1
    k = torch.where(mant * 128 <= 127, ex - 7, ex - 6).clamp_(min=-126)
    power = lambda e: ((e.to(torch.int32) + 127) << 23).view(torch.float32)         # noqa: E731 (exact, which pow is not)
    return (torch.round(b * power(-k)) * power(k)).view(rows, -1)[:, :ch]


def _run_norm(s):
    c, x = s["c"], s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    y = ((x - mean) * rstd * s["gamma"] + s["beta"]).to(_tdt(c))
    if not c["train"]:
        return dict(y=y)
    dy = s["dy"].float()
    xh = ((_kept8(s["x"]) if c["keep8"] else x) - mean) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dict(y=y, dx=dx.to(_tdt(c)), dgamma=(dy * xh).sum(0, dtype=torch.float64).float(), dbeta=dy.sum(0, dtype=torch.float64).float())


def _visible(c, n, start, device):
    j, i = torch.arange(c["pk"], device=device), torch.arange(c["pq"], device=device)
    seen = (j < n)[None, :].expand(c["pq"], -1)
    return seen & (j[None, :] <= i[:, None] + start) if c["causal"] else seen


def _offsets(c, start, device):
    """Index into the bucket map of every pair (query, key)."""
    j, i = torch.arange(c["pk"], device=device), torch.arange(c["pq"], device=device)
    return (j[None, :] - i[:, None] - start).clamp(-c["reach"], c["reach"]) + c["reach"]


def _heads(t, n, heads, d):
    """Sample n as [heads][positions][d] in float."""
    return t[n].float().view(t.shape[1], heads, d).transpose(0, 1).contiguous()


def _run_attn(s):
    c = s["c"]
    m, H, G, pq, pk, d, tdt = c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"], _tdt(c)
    scale = 1 / math.sqrt(d)
    new = lambda like: torch.empty(like.shape, dtype=tdt, device="cuda")            # noqa: E731
    y = torch.empty(m, pq, H * d, dtype=tdt, device="cuda")
    if c["train"]:
        dq, dk, dv = new(s["q"]), new(s["k"]), new(s["v"])
        diag = torch.zeros(H, pq + pk - 1, dtype=torch.float64, device="cuda")      # sums over pairs of one offset, all samples
    for n in range(m):
        q, k, v = _heads(s["q"], n, H, d), _heads(s["k"], n, G, d), _heads(s["v"], n, G, d)
        if G != H:
            k, v = k.repeat_interleave(H // G, 0), v.repeat_interleave(H // G, 0)
        seen = _visible(c, s["len"][n], s["start"][n], "cuda")
        p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale)
        p += s["table"][:, s["map"].long()][:, _offsets(c, s["start"][n], "cuda")]
        p.masked_fill_(~seen, -math.inf)
        top = p.amax(2, keepdim=True)
        p.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
        total = p.sum(2, keepdim=True)
        p /= torch.where(total == 0, torch.ones_like(total), total)
        o = torch.matmul(p, v)
        y[n] = o.transpose(0, 1).reshape(pq, H * d).to(tdt)
        if not c["train"]:
            continue
        g = _heads(s["dy"], n, H, d)
        dv_h = torch.matmul(p.transpose(1, 2).contiguous(), g)
        ds = torch.matmul(g, v.transpose(1, 2).contiguous())
        ds.sub_((g * o).sum(2, keepdim=True)).mul_(p)
        dq[n] = (scale * torch.matmul(ds, k)).transpose(0, 1).reshape(pq, H * d).to(tdt)
        dk_h = scale * torch.matmul(ds.transpose(1, 2).contiguous(), q)
        for out, t in ((dk, dk_h), (dv, dv_h)):
            out[n] = t.view(G, H // G, pk, d).sum(1).transpose(0, 1).reshape(pk, G * d).to(tdt)
        # queries in descending order and rows one element longer than the pitch: the diagonals of ds become columns
        for h in range(H):
            skew = torch.zeros(pq, pk + pq, device="cuda")
            skew[:, :pk] = ds[h].flip(0)
            diag[h] += skew.view(-1)[:pq * (pk + pq - 1)].view(pq, pk + pq - 1).sum(0, dtype=torch.float64)
    if not c["train"]:
        return dict(y=y)
    # column t of the skewed matrix: offset t - (pq - 1), less the position of the first query (zero wherever there is training)
    rel = torch.arange(pq + pk - 1, device="cuda") - (pq - 1)
    bucket = s["map"].long()[rel.clamp(-c["reach"], c["reach"]) + c["reach"]]
    dtable = torch.zeros(H, c["buckets"], dtype=torch.float64, device="cuda").index_add_(1, bucket, diag)
    return dict(y=y, dq=dq, dk=dk, dv=dv, dtable=dtable.float())


def run(s):
    if own:
        return _run_own(s)
    kind = s["c"]["kind"]
    if kind == "norm":
        return _run_norm(s)
    if kind == "attn":
        return _run_attn(s)
    x = _kept8(s["x"])
    if kind == "ckpt":
        return dict(x=x.to(_tdt(s["c"])))
    return dict(dw=torch.matmul(s["dz"].float().t().contiguous(), x))


# ---------------------------------------------------------------------------------------------- work and exact results
def _pairs(c):
    """Visible pairs of a head and sample, on average."""
    pq, pk = c["pq"], c["pk"]
    keys = pk if c["lengths"] == "full" else 0.75 * pk
    if not c["causal"]:
        return pq * keys
    if c["lengths"] == "cache":
        return pq * keys
    return sum(min(i + 1, keys) for i in range(pq))


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "attn":
        keys = (1.0 if c["lengths"] == "full" else 0.75) * c["pk"]
        q, kv = c["m"] * c["heads"] * c["pq"] * c["d"], c["m"] * c["kv_heads"] * keys * c["d"]
        flops = c["m"] * c["heads"] * _pairs(c) * c["d"] * (14 if c["train"] else 4)
        # q, k, v read and y written; for training dy read and dq, dk, dv written
        return {"bytes": int(es * (2 * q + 2 * kv + (2 * q + 2 * kv if c["train"] else 0))), "flops": int(flops)}
    n = c["rows"] * c["channels"]
    kept = n + c["rows"] * ((c["channels"] + BLOCK - 1) // BLOCK)
    if c["kind"] == "norm":
        b, f = 2 * n * es, 8 * n
        if c["train"]:          # dy read and dx written; the input read again, or its checkpoint written and read
            b, f = b + 2 * n * es + (2 * kept if c["keep8"] else n * es), f + 14 * n
        return {"bytes": b, "flops": f}
    if c["kind"] == "ckpt":
        return {"bytes": 2 * n * es + 2 * kept, "flops": 4 * n}
    return {"bytes": n * es + 2 * kept + c["rows"] * c["outputs"] * es + 4 * c["outputs"] * c["channels"],
            "flops": 2 * c["rows"] * c["outputs"] * c["channels"]}


def _exact_kept8(x):
    """The checkpoint's values from its definition: per block the least power of two that leaves no more than 127 steps."""
    x = x.double()
    out = torch.empty_like(x)
    for b in range(0, x.shape[1], BLOCK):
        t = x[:, b:b + BLOCK]
        top = t.abs().amax(1)
        k = torch.full_like(top, -126, dtype=torch.int64)
        step = ((k + 1023) << 52).view(torch.float64)           # 2^k
        for jump in (128, 64, 32, 16, 8, 4, 2, 1):               # the largest k with too large a step count, by halving, and one more
            far = ((k + jump + 1022) << 52).view(torch.float64)
            k = torch.where(top > 127 * far, k + jump, k)
        step = ((k + 1023) << 52).view(torch.float64)
        out[:, b:b + BLOCK] = torch.round(t / step[:, None]) * step[:, None]
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "ckpt":
        return dict(x=_exact_kept8(s["x"]))
    if c["kind"] == "wgrad":
        return dict(dw=s["dz"].double().t().contiguous() @ _exact_kept8(s["x"]))
    if c["kind"] == "norm":
        x, gamma = s["x"].double(), s["gamma"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        rstd = (var + 1e-5) ** -0.5
        out = dict(y=(x - mean) * rstd * gamma + s["beta"].double())
        if c["train"]:
            dy = s["dy"].double()
            xh = ((_exact_kept8(s["x"]) if c["keep8"] else x) - mean) * rstd
            g = dy * gamma
            out["dx"] = rstd * (g - g.sum(1, keepdim=True) / c["channels"] - xh * ((g * xh).sum(1, keepdim=True) / c["channels"]))
            out["dgamma"], out["dbeta"] = (dy * xh).sum(0), dy.sum(0)
        return out
    m, H, G, pq, pk, d = c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"]
    if m * H * pq * pk > 2.2e9:
        return None
    y = torch.zeros(m, pq, H, d, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(y), torch.zeros(m, pk, G, d, dtype=torch.float64, device="cuda"), torch.zeros(m, pk, G, d, dtype=torch.float64, device="cuda")
    dtable = torch.zeros(H, c["buckets"], dtype=torch.float64, device="cuda")
    lens, starts = s["len"].tolist(), s["start"].tolist()
    for n in range(m):
        keys = lens[n]
        if keys == 0:
            continue
        j, i = torch.arange(keys, device="cuda"), torch.arange(pq, device="cuda") + starts[n]
        rel = (j[None, :] - i[:, None]).clamp(-c["reach"], c["reach"]) + c["reach"]
        ids = s["map"].long()[rel]
        for h in range(H):
            q = s["q"][n, :, h * d:(h + 1) * d].double()
            g = h // (H // G)
            k, v = s["k"][n, :keys, g * d:(g + 1) * d].double(), s["v"][n, :keys, g * d:(g + 1) * d].double()
            t = q @ k.t() / math.sqrt(d) + s["table"][h].double()[ids]
            if c["causal"]:
                t = torch.where(j[None, :] <= i[:, None], t, torch.full_like(t, -math.inf))
            p = torch.nan_to_num(torch.softmax(t, 1), nan=0.0)
            y[n, :, h] = p @ v
            if not c["train"]:
                continue
            dy = s["dy"][n, :, h * d:(h + 1) * d].double()
            dp = dy @ v.t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            dq[n, :, h] = ds @ k / math.sqrt(d)
            dk[n, :keys, g] += ds.t() @ q / math.sqrt(d)
            dv[n, :keys, g] += p.t() @ dy
            dtable[h] += torch.bincount(ids.reshape(-1), weights=ds.reshape(-1), minlength=c["buckets"])
    out = dict(y=y.view(m, pq, H * d))
    if c["train"]:
        out.update(dq=dq.view(m, pq, H * d), dk=dk.view(m, pk, G * d), dv=dv.view(m, pk, G * d), dtable=dtable)
    return out
