"""The operators together, as a pre-norm attention block trains with them: norm, projections, attention with its bias, checkpoints in 8 bits for the
weight gradients.  Everything is enqueued at once; afterwards every call is compared with 64-bit arithmetic on the operands that it had, to the
tolerances of its own tests: a contraction's (terms + 8) half steps of float of the sum of magnitudes, and half a step of the stored type."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_gpu_norm as tn          # noqa: E402
import test_gpu_relattn as ta       # noqa: E402

pytestmark = pytest.mark.gpu

U, HALF = tn.U, tn.HALF


@pytest.fixture(scope="module")
def lpm():
    import torch
    assert torch.cuda.is_available()
    import paper_2207_11019_amd as lpm
    return lpm


class Block:
    """x -> x + attention(norm(x) Wqkv) Wo and its gradients, the inputs of the weight gradients kept in 8 bits."""

    def __init__(self, lpm, name, m=2, p=70, heads=4, d=32, causal=1, reach=20, nb=8, lens=None, seed=0):
        import torch
        self.lpm, self.name, self.dt = lpm, name, lpm.BF16 if name == "bf16" else lpm.F32
        self.c = ta.A(m, heads, heads, p, p, d, causal=causal, lens=lens, nb=nb, reach=reach, packed=True)
        self.rows, self.ch = m * p, heads * d
        rng = np.random.default_rng(seed)
        t = lambda *s, k=1.0: tn._torch(k * rng.standard_normal(s), name).cuda()      # noqa: E731
        R, CH = self.rows, self.ch
        self.x, self.dz = t(R, CH), t(R, CH)
        self.wqkv, self.wo = t(3 * CH, CH, k=CH ** -0.5), t(CH, CH, k=CH ** -0.5)
        f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()      # noqa: E731
        self.gamma, self.beta, self.table = 1 + 0.1 * f(CH), 0.1 * f(CH), f(heads, nb)
        self.ids = np.asarray(lpm.lpm_relbias_buckets(nb, reach, not causal))
        self.map = torch.from_numpy(self.ids.astype(np.int32)).cuda()
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
        self.g = lpm.lpm_attn_geom(m=m, heads=heads, kv_heads=heads, pq=p, pk=p, d=d, causal=causal, n_buckets=nb, reach=reach, ldq=3 * CH, ldk=3 * CH, ldv=3 * CH)
        self.proj = dict(m=R, h=1, w=1, cin=CH, cout=3 * CH, kh=1, kw=1, stride=1, pad=0)
        self.out = dict(self.proj, cout=CH)

    def buffers(self):
        import torch
        l, R, CH = self.lpm, self.rows, self.ch
        n = lambda *s: torch.full(s, 5.0).to(self.x.dtype).cuda()      # noqa: E731
        f = lambda *s: torch.full(s, 5.0).cuda()                       # noqa: E731
        o = dict(h=n(R, CH), qkv=n(R, 3 * CH), y=n(R, CH), z=n(R, CH), dy=n(R, CH), dqkv=n(R, 3 * CH), dh=n(R, CH), dx=n(R, CH), stats=f(2 * R), dwo=f(CH, CH),
                 dwqkv=f(3 * CH, CH), dgamma=f(CH), dbeta=f(CH), dtable=f(*self.table.shape))
        for k in ("kx", "kh", "ky"):
            o[k] = tn._bytes(l.lpm_ckpt8_bytes(R, CH))
        o["st"] = tn._bytes(l.lpm_attn_stats_bytes(self.g, self.dt))
        need = list(l.lpm_attn_ws_bytes(self.g, self.dt)) + [l.lpm_norm_ws_bytes(R, CH, self.dt)]
        for g in (self.proj, self.out):
            need += list(l.lpm_conv_ws_bytes(g, self.dt)) + [l.lpm_conv_wgrad_ckpt8_ws_bytes(g, self.dt)]
        o["ws"] = tn._bytes(max(need))
        return o

    def forward(self, o, s=None):
        l, dt, R, CH = self.lpm, self.dt, self.rows, self.ch
        l.lpm_norm_forward(R, CH, dt, self.x, self.gamma, self.beta, 1e-5, o["h"], o["stats"], o["kx"], s)
        l.lpm_ckpt8_pack(R, CH, dt, o["h"], o["kh"], s)
        l.lpm_conv_forward(self.proj, dt, o["h"], self.wqkv, None, None, None, False, o["qkv"], o["ws"], s)
        q, k, v = (o["qkv"][:, i * CH:(i + 1) * CH] for i in range(3))
        l.lpm_attn_forward(self.g, dt, q, k, v, self.lens, None, self.map, self.table, o["y"], o["st"], o["ws"], s)
        l.lpm_ckpt8_pack(R, CH, dt, o["y"], o["ky"], s)
        l.lpm_conv_forward(self.out, dt, o["y"], self.wo, None, None, self.x, False, o["z"], o["ws"], s)

    def backward(self, o, s=None):
        l, dt, R, CH = self.lpm, self.dt, self.rows, self.ch
        l.lpm_conv_wgrad_ckpt8(self.out, dt, o["ky"], self.dz, o["dwo"], False, o["ws"], s)
        l.lpm_conv_dgrad(self.out, dt, self.dz, self.wo, None, o["dy"], False, o["ws"], s)
        (q, k, v), (dq, dk, dv) = ([o[n][:, i * CH:(i + 1) * CH] for i in range(3)] for n in ("qkv", "dqkv"))
        l.lpm_attn_backward(self.g, dt, q, k, v, o["y"], o["st"], o["dy"], self.lens, None, self.map, self.table, dq, dk, dv, o["dtable"], False, o["ws"], s)
        l.lpm_conv_wgrad_ckpt8(self.proj, dt, o["kh"], o["dqkv"], o["dwqkv"], False, o["ws"], s)
        l.lpm_conv_dgrad(self.proj, dt, o["dqkv"], self.wqkv, None, o["dh"], False, o["ws"], s)
        o["dx"].copy_(self.dz)                       # the residual's gradient, to which the norm's is added
        l.lpm_norm_backward(R, CH, dt, None, o["kx"], o["stats"], o["dh"], self.gamma, o["dx"], o["dgamma"], o["dbeta"], True, False, o["ws"], s)

    def check(self, o):
        a, name, R, CH = tn._np, self.name, self.rows, self.ch
        h = HALF[name]

        def near(n, want, tol, stored=h):
            d = np.abs(a(o[n]).reshape(want.shape) - want)
            assert (d <= tol + stored * (np.abs(want) + tol) + 1e-30).all(), (n, float((d / (tol + stored * np.abs(want) + 1e-30)).max()))

        def product(n, x, w, add=0.0, stored=h):
            near(n, x @ w + add, (x.shape[1] + 8) * U * (np.abs(x) @ np.abs(w) + np.abs(add)), stored)
        X, DZ, wqkv, wo, gamma, beta = a(self.x), a(self.dz), a(self.wqkv), a(self.wo), a(self.gamma), a(self.beta)
        mu = X.mean(1, keepdims=True)
        rs = 1 / np.sqrt(((X - mu) ** 2).mean(1, keepdims=True) + np.float64(np.float32(1e-5)))
        big = np.abs(X).max(1, keepdims=True)
        H = (X - mu) * rs
        near("h", gamma * H + beta, np.abs(gamma) * 128 * U * (np.abs(H) + rs * big) + 4 * U * np.abs(beta))
        product("qkv", a(o["h"]), wqkv.T)
        product("z", a(o["y"]), wo.T, X)
        product("dy", DZ, wo)
        product("dh", a(o["dqkv"]), wqkv)
        product("dwo", DZ.T, tn.kept8(a(o["y"]))[2], stored=U)
        product("dwqkv", a(o["dqkv"]).T, tn.kept8(a(o["h"]))[2], stored=U)
        c, hd, d = self.c, self.c["heads"], self.c["d"]
        heads = lambda t: a(t).reshape(c["m"], c["pq"], hd, d)      # noqa: E731
        q, k, v = (heads(o["qkv"][:, i * CH:(i + 1) * CH]) for i in range(3))
        got = dict(y=o["y"], dtable=o["dtable"], **{n: o["dqkv"][:, i * CH:(i + 1) * CH] for i, n in enumerate(("dq", "dk", "dv"))})
        ta.compare(c, name, {n: t if n == "dtable" else t.reshape(c["m"], c["pq"], CH) for n, t in got.items()}, [q, k, v, heads(o["dy"]), a(self.table), self.ids])
        H = (tn.kept8(X)[2] - mu) * rs
        DH = a(o["dh"])
        g = DH * gamma
        dx = rs * (g - g.mean(1, keepdims=True) - H * (g * H).mean(1, keepdims=True)) + DZ
        near("dx", dx, 256 * U * rs * np.abs(g).max(1, keepdims=True) * (1 + np.abs(H).max(1, keepdims=True)) ** 2 * (1 + rs * big) + 4 * U * np.abs(DZ))
        chain, herr = (R / 256 + 128) * U, 128 * U * (np.abs(H) + rs * big)
        near("dgamma", (DH * H).sum(0), chain * np.abs(DH * H).sum(0) + (np.abs(DH) * herr).sum(0), 4 * U)
        near("dbeta", DH.sum(0), chain * np.abs(DH).sum(0), 4 * U)


BLOCKS = [dict(), dict(m=3, p=33, heads=3, d=24, causal=0, reach=5, lens=[33, 1, 0]), dict(m=1, p=1, heads=2, d=64), dict(m=1, p=200, heads=1, d=128, reach=64, nb=32)]


@pytest.mark.parametrize("k", BLOCKS, ids=lambda k: "_".join("%s%s" % i for i in k.items()).replace(" ", "") or "plain")
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_block(lpm, name, k):
    import torch
    b = Block(lpm, name, **k)
    o = b.buffers()
    b.forward(o), b.backward(o)
    torch.cuda.synchronize()
    b.check(o)


RESULTS = ("h", "qkv", "y", "z", "dy", "dqkv", "dh", "dx", "dwo", "dwqkv", "dgamma", "dbeta", "dtable")


def test_two_blocks_on_two_streams(lpm):
    """Calls at once, each with scratch of its own, on streams that are not the current one: the bits of one after the other."""
    import torch
    blocks = [Block(lpm, "bf16", m=4, p=300, heads=6, d=64, seed=1), Block(lpm, "f32", m=2, p=150, seed=2)]
    alone, both = [b.buffers() for b in blocks], [b.buffers() for b in blocks]
    for b, o in zip(blocks, alone):
        b.forward(o), b.backward(o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for turn in range(3):
        for step in ("forward", "backward"):
            for b, o, s in zip(blocks, both, streams):
                with torch.cuda.stream(s):
                    getattr(b, step)(o, s)
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        for n in RESULTS:
            assert torch.equal(x[n], y[n]), n


def test_two_captured_graphs_share_scratch(lpm):
    """Forward and backward captured apart with one scratch buffer, replayed with eager calls between: nothing is kept there from one to the other."""
    import torch
    b = Block(lpm, "bf16", m=2, p=130, heads=2, d=64, seed=3)
    eager, cap = b.buffers(), b.buffers()
    b.forward(eager), b.backward(eager)
    torch.cuda.synchronize()
    graphs = []
    for step in (b.forward, b.backward):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(cap, torch.cuda.current_stream())
    want = {n: eager[n].clone() for n in RESULTS}
    for turn in range(4):
        graphs[0].replay()
        cap["ws"].fill_(255)
        if turn % 2:
            b.forward(eager), b.backward(eager)
            torch.cuda.synchronize()
        graphs[1].replay()
        torch.cuda.synchronize()
        for n in RESULTS:
            assert torch.equal(cap[n], want[n]) and torch.equal(eager[n], want[n]), (turn, n)
            if turn < 3:
                cap[n].fill_(9.0)


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 4.0])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_scales(lpm, name, scale):
    """Scores that are all bias, mostly bias, and steep ones."""
    c = ta.A(1, 2, 1, 40, 70, 32, causal=1, starts=[30], nb=6, reach=9, scale=scale)
    got, operands = ta.run(lpm, c, name)
    if scale < 1e-20:                      # (dq and dk are below the least normal number)
        got = {n: t for n, t in got.items() if n not in ("dq", "dk")}
    ta.compare(c, name, got, operands)


def _differences(f, x, r):
    """f along r by central differences in 64 bits."""
    e = 1e-5
    return (f(x + e * r) - f(x - e * r)) / (2 * e)


def test_attention_gradients_against_differences(lpm):
    c = ta.A(2, 4, 2, 37, 50, 16, causal=1, starts=[13, 5], lens=[50, 30], nb=6, reach=9)
    got, (q, k, v, dy, table, ids) = ta.run(lpm, c, "f32")
    ref, tol = ta.reference(c, "f32", q, k, v, dy, table, ids)
    rng = np.random.default_rng(4)
    loss = lambda **o: (ta.reference(c, "f32", **dict(dict(q=q, k=k, v=v, dy=dy, table=table, ids=ids), **o))[0]["y"] * dy).sum()      # noqa: E731
    for n, x in (("q", q), ("k", k), ("v", v), ("table", table)):
        r = rng.standard_normal(x.shape)
        g = got["d" + n].float().cpu().numpy().astype(np.float64).reshape(x.shape)
        want = _differences(lambda t: loss(**{n: t}), x, r)
        # the gradient's own tolerance along r; the differences err by e^2 times a third derivative and by 2^-53 |loss| / e: 1e-8 of the sizes here
        assert abs((g * r).sum() - want) <= (tol["d" + n] * np.abs(r)).sum() + 1e-8 * (np.abs(g * r).sum() + abs(loss())), n


def test_norm_gradients_against_differences(lpm):
    import torch
    rows, ch = 9, 70
    rng = np.random.default_rng(6)
    x, dy, gamma, beta = (rng.standard_normal(s).astype(np.float32) for s in ((rows, ch), (rows, ch), ch, ch))
    d = lambda a: torch.from_numpy(a).cuda()      # noqa: E731
    y, dx, dg, db, st = torch.zeros(rows, ch).cuda(), torch.zeros(rows, ch).cuda(), torch.zeros(ch).cuda(), torch.zeros(ch).cuda(), torch.zeros(2 * rows).cuda()
    xd, gd = d(x), d(gamma)
    lpm.lpm_norm_forward(rows, ch, lpm.F32, xd, gd, d(beta), 1e-5, y, st)
    lpm.lpm_norm_backward(rows, ch, lpm.F32, xd, None, st, d(dy), gd, dx, dg, db, ws=tn._bytes(lpm.lpm_norm_ws_bytes(rows, ch, lpm.F32)))
    torch.cuda.synchronize()
    x, dy, gamma, beta = (a.astype(np.float64) for a in (x, dy, gamma, beta))

    def loss(x=x, gamma=gamma, beta=beta):
        mu = x.mean(1, keepdims=True)
        return ((gamma * (x - mu) / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + 1e-5) + beta) * dy).sum()
    for n, v, g in (("x", x, dx), ("gamma", gamma, dg), ("beta", beta, db)):
        r = rng.standard_normal(v.shape)
        g = tn._np(g)
        # 256 half steps of float of the terms, as in the norm's own tests, times the largest h squared (16); 1e-8 for the differences
        assert abs((g * r).sum() - _differences(lambda t: loss(**{n: t}), v, r)) <= (256 * 16 * U + 1e-8) * (np.abs(dy).sum() * np.abs(r).max()), n


def test_a_cache_longer_than_offsets_of_32_bits(lpm):
    """Keys and values of one sample over more than 4 GiB: bf16, positions 2^20 elements apart, the last of 4099 beyond 2^32 elements."""
    import torch
    pk, ld, d, H = 4099, 1 << 20, 64, 2
    kv = torch.zeros((pk - 1) * ld + 2 * H * d, dtype=torch.bfloat16, device="cuda")
    k, v = kv, kv[H * d:]
    gen = torch.Generator().manual_seed(3)
    rows = torch.randn(pk, 2 * H * d, generator=gen).to(torch.bfloat16)
    kv.as_strided((pk, 2 * H * d), (ld, 1)).copy_(rows.cuda())
    q, y = torch.randn(1, 3, H * d, generator=gen).to(torch.bfloat16).cuda(), torch.zeros(1, 3, H * d, dtype=torch.bfloat16, device="cuda")
    g = dict(m=1, heads=H, kv_heads=H, pq=3, pk=pk, d=d, causal=0, ldk=ld, ldv=ld)
    lpm.lpm_attn_forward(g, lpm.BF16, q, k, v, None, None, None, None, y, None, tn._bytes(lpm.lpm_attn_ws_bytes(g, lpm.BF16)[0]))
    torch.cuda.synchronize()
    c = ta.A(1, H, H, 3, pk, d, nb=0, reach=0)
    K, V = (rows[:, i * H * d:(i + 1) * H * d].float().numpy().astype(np.float64).reshape(1, pk, H, d) for i in range(2))
    Q = ta._np(q, H, d)
    ta.compare(c, "bf16", dict(y=y), [Q, K, V, Q, np.zeros((H, 1)), np.zeros(1, int)])


def test_host_memory_and_other_devices_are_refused(lpm):
    import torch
    x, y = torch.zeros(4, 8), torch.zeros(4, 8).cuda()
    for a, b in ((x, y), (y, x)):
        with pytest.raises(ValueError):
            lpm.lpm_norm_forward(4, 8, lpm.F32, a, None, None, 1e-5, b)
