"""Multi-head attention with a bias by distance buckets: forward and every gradient against 64-bit arithmetic.

Tolerances are worked out element by element from the roundings that the kernels make (u = 2^-24, h = half a step of the element type):
  scores     (d + 8) u of the sum of |q k| scale and of |bias|, twice that relative to p, and (keys + queries + 64) u for sums over either
  y          p in the element type: h of sum p |v|, and h of the result
  ds         p (relative error of p |dp - delta| + errors of dp and of delta); delta is a row's sum of p dp in dk and dtable, dy . y in dq, with the
             errors of y as it is stored: h of sum |dy| p |v| and h of sum |dy y|
  dq, dk     ds in the element type: h of sum |ds k|, errors of ds, h of the result; dv like y; dtable the errors of ds, summed"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
HALF_P = {"f32": 0.0, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def lpm():
    import torch
    assert torch.cuda.is_available()
    import paper_2207_11019_amd as lpm
    return lpm


def A(m, h, g, pq, pk, d, causal=0, lens=None, starts=None, nb=8, reach=6, packed=False, pad=0, scale=0.0):
    return dict(m=m, heads=h, kv_heads=g, pq=pq, pk=pk, d=d, causal=causal, lens=lens, starts=starts, nb=nb, reach=reach, packed=packed, pad=pad, scale=scale)


def _id(c):
    return "m%d_h%d_%d_%dx%d_d%d%s%s%s" % (c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"], "_causal" if c["causal"] else "",
                                           "_packed" if c["packed"] else "", "_r%d" % c["reach"] if c["nb"] else "_plain")


def reference(c, name, q, k, v, dy, table, ids):
    """Everything in 64 bits, with the tolerance of every output (see above)."""
    m, H, G, pq, pk, d = c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"]
    h, hp = HALF[name], HALF_P[name]
    scale = np.float64(np.float32(c["scale"])) if c["scale"] else 1 / np.sqrt(np.float64(d))
    out = {n: np.zeros(s) for n, s in (("y", (m, pq, H, d)), ("dq", (m, pq, H, d)), ("dk", (m, pk, G, d)), ("dv", (m, pk, G, d)), ("dtable", (H, max(c["nb"], 1))))}
    tol = {n: np.zeros_like(a) for n, a in out.items()}
    for n in range(m):
        keys = pk if c["lens"] is None else min(max(c["lens"][n], 0), pk)
        start = 0 if c["starts"] is None else c["starts"][n]
        if keys == 0 or pq == 0:
            continue
        rel = np.arange(keys)[None, :] - np.arange(pq)[:, None] - start
        seen = (rel <= 0) if c["causal"] else np.ones_like(rel, bool)
        at = np.clip(rel, -c["reach"], c["reach"]) + c["reach"]
        for hh in range(H):
            g = hh // (H // G)
            Q, K, V, DY = q[n, :, hh], k[n, :keys, g], v[n, :keys, g], dy[n, :, hh]
            bias = table[hh][ids[at]] if c["nb"] else np.zeros(rel.shape)
            s = scale * (Q @ K.T) + bias
            s[~seen] = -np.inf
            top = s.max(1, keepdims=True)
            p = np.exp(s - np.where(np.isinf(top), 0, top))
            tot = p.sum(1, keepdims=True)
            p = p / np.where(tot == 0, 1, tot)
            y = p @ V
            es = (d + 8) * U * (scale * (np.abs(Q) @ np.abs(K).T) + np.where(np.isinf(bias) | ~seen, 0, np.minimum(np.abs(bias), 1e4)))
            ep = 2 * np.where(seen, es, 0).max(1, keepdims=True) + (keys + pq + 64) * U
            out["y"][n, :, hh] = y
            ey = (hp + ep) * (p @ np.abs(V))
            tol["y"][n, :, hh] = ey + h * (np.abs(y) + ey)
            dp = DY @ V.T
            delta = (DY * y).sum(1, keepdims=True)
            ds = p * (dp - delta)
            sizes = np.abs(DY) @ np.abs(V).T
            edelta = (p * ((ep + 4 * U) * np.abs(dp - delta) + (d + 8) * U * sizes)).sum(1, keepdims=True) + 8 * U * np.abs(delta)
            edelta_y = (np.abs(DY) * ((hp + ep) * (p @ np.abs(V)) + (h + (d + 4) * U) * np.abs(y))).sum(1, keepdims=True)
            rest = p * (ep * np.abs(dp - delta) + (d + 4) * U * sizes + 4 * U * (np.abs(dp) + np.abs(delta)))
            eds, eds_y = rest + p * (edelta if name == "bf16" else edelta_y), rest + p * edelta_y
            out["dv"][n, :keys, g] += p.T @ DY
            tol["dv"][n, :keys, g] += ((hp + ep) * p).T @ np.abs(DY)
            out["dq"][n, :, hh] = scale * (ds @ K)
            e = scale * (((hp + (keys + 64) * U) * np.abs(ds) + (1 + hp) * eds_y) @ np.abs(K))
            tol["dq"][n, :, hh] = e + h * (np.abs(out["dq"][n, :, hh]) + e)
            out["dk"][n, :keys, g] += scale * (ds.T @ Q)
            tol["dk"][n, :keys, g] += scale * (((hp + (pq * H + 64) * U) * np.abs(ds) + (1 + hp) * eds).T @ np.abs(Q))
            if c["nb"]:
                for b in range(c["nb"]):
                    of = ids[at] == b
                    out["dtable"][hh, b] += ds[of].sum()
                    tol["dtable"][hh, b] += eds[of].sum() + (pq + pk + 64 + 4 * m) * U * np.abs(ds[of]).sum()
    for n in ("dk", "dv"):
        tol[n] += h * (np.abs(out[n]) + tol[n])
    return out, tol


def _operand(rng, name, m, p, ld, parts, width):
    """A buffer [m][p][ld] and views of `parts` operands of `width` elements side by side in it."""
    import torch
    t = torch.from_numpy(rng.standard_normal((m, p, ld)).astype(np.float32))
    t = (t.to(torch.bfloat16) if name == "bf16" else t).cuda()
    return t, [t[:, :, i * width:(i + 1) * width] for i in range(parts)]


def _np(t, heads, d):
    return t.float().cpu().numpy().astype(np.float64).reshape(t.shape[0], t.shape[1], heads, d)


def run(lpm, c, name, table=None, ids=None, change=None, seed=0, train=True, acc=None):
    """Operands, one forward and one backward call; returns the results, and the operands in 64 bits."""
    import torch
    dt = lpm.BF16 if name == "bf16" else lpm.F32
    m, H, G, pq, pk, d = c["m"], c["heads"], c["kv_heads"], c["pq"], c["pk"], c["d"]
    rng = np.random.default_rng(seed + 7 * pq + pk + d)
    wq, wk, pad = H * d, G * d, c["pad"]
    if c["packed"]:
        ldq = ldk = ldv = 3 * wq + pad
        _, (q, k, v) = _operand(rng, name, m, pq, ldq, 3, wq)
        _, (dq, dk, dv) = _operand(rng, name, m, pq, ldq, 3, wq)
    else:
        ldq, ldk, ldv = wq + pad, wk + 2 * pad, wk + 3 * pad
        q, k, v = (_operand(rng, name, m, p, ld, 1, w)[1][0] for p, ld, w in ((pq, ldq, wq), (pk, ldk, wk), (pk, ldv, wk)))
        dq, dk, dv = (_operand(rng, name, m, p, ld, 1, w)[1][0] for p, ld, w in ((pq, ldq, wq), (pk, ldk, wk), (pk, ldv, wk)))
    dy = _operand(rng, name, m, pq, wq, 1, wq)[1][0]
    if change:
        change(q, k, v, dy)
    y = torch.full((m, pq, wq), 3.0).to(q.dtype).cuda()
    if table is None:
        table = rng.standard_normal((H, max(c["nb"], 1)))
        table = table.astype(np.float32).astype(np.float64)
    if ids is None:
        ids = rng.integers(0, max(c["nb"], 1), 2 * c["reach"] + 1)
    g = lpm.lpm_attn_geom(m=m, heads=H, kv_heads=G, pq=pq, pk=pk, d=d, causal=c["causal"], n_buckets=c["nb"], reach=c["reach"], ldq=ldq, ldk=ldk, ldv=ldv,
                          scale=c["scale"])
    i32 = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.int32)).cuda()      # noqa: E731
    lens, starts, tmap = i32(c["lens"]), i32(c["starts"]), i32(ids) if c["nb"] else None
    tt = torch.from_numpy(np.asarray(table, np.float32)).cuda() if c["nb"] else None
    fwd, bwd = lpm.lpm_attn_ws_bytes(g, dt)
    ws = torch.full((max(fwd, bwd, 256),), 255, dtype=torch.uint8).cuda()       # (NaN: what a call reads it has written)
    stats = torch.full((max(lpm.lpm_attn_stats_bytes(g, dt), 256),), 255, dtype=torch.uint8).cuda() if train else None
    lpm.lpm_attn_forward(g, dt, q, k, v, lens, starts, tmap, tt, y, stats, ws)
    got = dict(y=y)
    if train:
        ws.fill_(255)
        dtable = torch.from_numpy(np.asarray(acc if acc is not None else np.full((H, max(c["nb"], 1)), np.nan), np.float32)).cuda() if c["nb"] else None
        lpm.lpm_attn_backward(g, dt, q, k, v, y, stats, dy, lens, starts, tmap, tt, dq, dk, dv, dtable, acc is not None, ws)
        got.update(dq=dq, dk=dk, dv=dv)
        if c["nb"]:
            got["dtable"] = dtable
    torch.cuda.synchronize()
    return got, [_np(t, n, d) for t, n in ((q, H), (k, G), (v, G), (dy, H))] + [np.asarray(table, np.float64), np.asarray(ids)]


def compare(c, name, got, operands, acc=None):
    ref, tol = reference(c, name, *operands)
    for n, t in got.items():
        r = ref[n].reshape(tuple(t.shape)) + (acc if n == "dtable" and acc is not None else 0)
        bound = tol[n].reshape(tuple(t.shape)) + 1e-30 + (4 * U * (np.abs(r) + np.abs(acc)) if n == "dtable" and acc is not None else 0)
        diff = np.abs(t.float().cpu().numpy().astype(np.float64) - r)
        assert np.isfinite(diff).all() and (diff <= bound).all(), (n, float((diff / bound).max()), np.argwhere(~(diff <= bound))[:4].tolist())


def check(lpm, c, name, **k):
    got, operands = run(lpm, c, name, **k)
    compare(c, name, got, operands, k.get("acc"))
    return got


SHAPES = [
    A(1, 1, 1, 1, 1, 8),                                               # one token
    A(2, 2, 1, 1, 70, 16, causal=1, starts=[69, 3], lens=[70, 5]),     # single queries against a cache
    A(2, 3, 3, 17, 17, 24, packed=True),
    A(1, 2, 2, 33, 31, 32, reach=40),                                  # every distance has an entry of its own
    A(2, 2, 1, 65, 64, 40, causal=1),                                  # the first queries see few keys, the last all
    A(2, 4, 2, 64, 130, 33, pad=5, lens=[130, 0]),                     # odd strides, a sample without keys
    A(1, 1, 1, 130, 66, 64, causal=1, starts=[-20]),                   # the first 20 queries see nothing
    A(3, 2, 2, 40, 40, 9, lens=[1, 40, 39], nb=3, reach=0),            # heads of nine channels, one bucket distance
    A(1, 2, 2, 50, 50, 64, nb=0, reach=0),                             # no bias
    A(1, 3, 1, 129, 200, 96, causal=1, starts=[71], reach=17),
    A(1, 2, 1, 70, 260, 128, reach=100, lens=[257]),
    A(1, 1, 1, 140, 300, 72, causal=1, starts=[160], reach=5, scale=0.3),
]
MORE = [
    A(2, 2, 2, 200, 200, 80, packed=True, causal=1, reach=300, nb=33),
    A(1, 2, 1, 300, 310, 128, lens=[301], reach=64, nb=16),
    A(1, 1, 1, 513, 520, 20, reach=128, nb=32),
    A(4, 2, 2, 96, 700, 32, lens=[700, 699, 1, 350], causal=1, starts=[604, 603, 0, 254]),
    A(1, 8, 2, 5, 2000, 64, causal=1, starts=[1995], reach=128, nb=32),          # keys over several blocks
    A(2, 2, 2, 1, 4097, 128, causal=1, starts=[4096, 2500], lens=[4097, 2501], reach=2048, nb=64),
    A(1, 2, 2, 700, 700, 64, causal=1, packed=True, reach=2048, nb=5),
    A(1, 1, 1, 1500, 1500, 64, reach=128, nb=32),
    A(130, 1, 1, 70, 1100, 72, nb=4, reach=30, lens=[1100, 600, 0, 513, 1] * 26),      # no rows shared, keys over two blocks
]


@pytest.mark.parametrize("c", SHAPES, ids=_id)
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_attention(lpm, name, c):
    check(lpm, c, name)


@pytest.mark.parametrize("c", MORE, ids=_id)
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_larger_attention(lpm, name, c):
    check(lpm, c, name)
    check(lpm, c, name, train=False, seed=1)


# as many blocks as two wavefronts share rows in, or none share any; heads that come straight from memory (16, 40, 72, 96, 128) and by way of registers
@pytest.mark.parametrize("d", [16, 33, 40, 72, 96, 121, 128])
@pytest.mark.parametrize("m,causal", [(50, 0), (50, 1), (200, 0), (200, 1)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_many_blocks(lpm, name, m, causal, d):
    r = np.random.default_rng(m + d)
    c = A(m, 2, 2, 100, 70, d, causal=causal, nb=3, reach=11, lens=[int(x) for x in r.integers(0, 71, m)], starts=[int(x) for x in r.integers(-40, 60, m)])
    check(lpm, c, name)


# few queries of heads that share keys, as rows of one block: up to one operand of 32 rows, and two
@pytest.mark.parametrize("m,heads,pq,pk", [(300, 4, 1, 60), (150, 4, 12, 90), (40, 8, 8, 90), (300, 2, 31, 40), (9, 4, 3, 1300)])
@pytest.mark.parametrize("d", [16, 57, 64, 128])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_many_blocks_of_shared_keys(lpm, name, d, m, heads, pq, pk):
    r = np.random.default_rng(m + d)
    lens = r.integers(0, pk + 1, m)
    check(lpm, A(m, heads, 1, pq, pk, d, causal=1, nb=5, reach=20, lens=[int(x) for x in lens], starts=[int(x) - pq for x in lens]), name)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_masks_and_values_in_masked_places(lpm, name):
    """A table of -infinity and of the lowest number in some buckets, rows of nothing else, and NaN and infinities in keys and values behind a
    sample's last one, which nothing reads."""
    c = A(2, 2, 2, 40, 70, 32, lens=[37, 70], reach=3, nb=7)
    table = np.random.default_rng(3).standard_normal((2, 7)).astype(np.float32).astype(np.float64)
    table[0, 2], table[1, 4], table[1, 5] = -np.inf, -3.4e38, -3.4028234663852886e38

    def change(q, k, v, dy):
        k[0, 37:] = float("nan")
        v[0, 37:] = float("inf")
        v[0, 60:] = float("nan")
    got, operands = run(lpm, c, name, table=table, ids=np.arange(7), change=change)
    operands[1][0, 37:], operands[2][0, 37:] = 0, 0
    compare(c, name, got, operands)
    for low in (-np.inf, -3.4028234663852886e38):          # ... everywhere: zeros, or all keys alike
        t = np.full((2, 7), low)
        got, operands = run(lpm, c, name, table=t, ids=np.arange(7))
        if np.isinf(low):
            for n, x in got.items():
                assert (x == 0).all(), n
        else:
            compare(dict(c, scale=1e-30), name, dict(y=got["y"], dv=got["dv"]), operands)


def test_table_gradient_accumulates(lpm):
    acc = np.random.default_rng(1).standard_normal((2, 8)).astype(np.float32).astype(np.float64)
    check(lpm, A(2, 2, 1, 45, 50, 32), "f32", acc=acc)


def test_bucket_ids_and_lengths_out_of_range_are_clamped(lpm):
    """Ids beside the table, lengths beyond the keys, starts far outside: clamped, nothing is read or written out of bounds."""
    c = A(2, 2, 2, 33, 40, 16, lens=[1000, -3], starts=[0, 5], reach=4, nb=4)
    got, operands = run(lpm, c, "f32", ids=np.array([-7, 9, 0, 1, 2, 3, 99, 2, 2 ** 31 - 1]))
    operands[5] = np.clip(operands[5], 0, 3)
    compare(c, "f32", got, operands)
    c = A(2, 1, 1, 33, 40, 16, causal=1, starts=[2 ** 31 - 1, -2 ** 31], reach=4, nb=4)
    got, operands = run(lpm, c, "f32")
    compare(dict(c, starts=[10 ** 6, -10 ** 6]), "f32", got, operands)


def test_nothing_to_do(lpm):
    """No samples, no queries, no keys: gradients of nothing are zeros."""
    for c in (A(0, 2, 1, 5, 6, 16), A(2, 2, 1, 0, 6, 16), A(2, 2, 1, 5, 0, 16)):
        got, _ = run(lpm, c, "f32")
        for n, t in got.items():
            assert (t == 0).all(), (_id(c), n)


def test_neighbours_of_packed_operands_are_left_alone(lpm):
    """What lies between an operand's positions (other parts of a packed row, padding) keeps its bits."""
    import torch
    c = A(2, 2, 2, 37, 37, 20, packed=True)
    x = torch.randn(2, 37, 3 * 40 + 8).cuda()
    before = x.clone()
    g = dict(m=2, heads=2, kv_heads=2, pq=37, pk=37, d=20, ldq=128, ldk=128, ldv=128)
    dt = lpm.F32
    q, k, v = (x[:, :, 40 * i:40 * i + 40] for i in range(3))
    dx = torch.full((2, 37, 128), 7.0).cuda()
    dq, dk, dv = (dx[:, :, 40 * i:40 * i + 40] for i in range(3))
    y, dy = torch.zeros(2, 37, 40).cuda(), torch.randn(2, 37, 40).cuda()
    stats = torch.zeros(lpm.lpm_attn_stats_bytes(g, dt), dtype=torch.uint8, device="cuda")
    ws = torch.zeros(max(lpm.lpm_attn_ws_bytes(g, dt)), dtype=torch.uint8, device="cuda")
    lpm.lpm_attn_forward(g, dt, q, k, v, None, None, None, None, y, stats, ws)
    lpm.lpm_attn_backward(g, dt, q, k, v, y, stats, dy, None, None, None, None, dq, dk, dv, None, False, ws)
    torch.cuda.synchronize()
    assert torch.equal(x, before) and (dx[:, :, 120:] == 7).all() and not (dx[:, :, :120] == 7).any()
    assert c["packed"]


def test_attention_is_repeatable_and_replays_in_a_graph(lpm):
    import torch
    c = dict(m=2, heads=4, kv_heads=2, pq=150, pk=150, d=64, causal=1, n_buckets=16, reach=40)
    gen = torch.Generator().manual_seed(5)
    mk = lambda *s: torch.randn(*s, generator=gen).to(torch.bfloat16).cuda()      # noqa: E731
    q, k, v, dy = mk(2, 150, 256), mk(2, 150, 128), mk(2, 150, 128), mk(2, 150, 256)
    table, tmap = torch.randn(4, 16, generator=gen).cuda(), torch.tensor(lpm.lpm_relbias_buckets(16, 40, False), dtype=torch.int32).cuda()
    sb, wb = lpm.lpm_attn_stats_bytes(c, lpm.BF16), max(lpm.lpm_attn_ws_bytes(c, lpm.BF16) + (256,))
    new = lambda: dict(y=torch.zeros_like(q), dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v), dt=torch.zeros_like(table),      # noqa: E731
                       st=torch.zeros(sb, dtype=torch.uint8, device="cuda"), ws=torch.zeros(wb, dtype=torch.uint8, device="cuda"))
    a, b = new(), new()

    def once(o, s):
        lpm.lpm_attn_forward(c, lpm.BF16, q, k, v, None, None, tmap, table, o["y"], o["st"], o["ws"], s)
        lpm.lpm_attn_backward(c, lpm.BF16, q, k, v, o["y"], o["st"], dy, None, None, tmap, table, o["dq"], o["dk"], o["dv"], o["dt"], False, o["ws"], s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(b, torch.cuda.current_stream())
    for turn in range(3):
        once(a, torch.cuda.current_stream())
        for o in b.values():
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("y", "dq", "dk", "dv", "dt"):
            assert torch.equal(a[n], b[n]), (turn, n)
