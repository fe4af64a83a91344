"""Layer norm (forward, backward, weight and bias gradients) and checkpoints in 8 bits against 64-bit arithmetic.

Tolerances count roundings: a stored value is off by half a step of its type, and float sums of up to 80 terms in a row (64 channels a thread,
six lane exchanges, four wavefronts) by that many half steps of the sum of magnitudes.  Checkpoints are exact: bytes are compared."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24          # half a step of float, relative
HALF = {"f32": U, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def lpm():
    import torch
    assert torch.cuda.is_available()
    import paper_2207_11019_amd as lpm
    return lpm


def _torch(a, name):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return t.to(torch.bfloat16) if name == "bf16" else t


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _bytes(n):
    import torch
    return torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")


def kept8(x):
    """q, exponent bytes and values of a checkpoint, element by element from its definition (x: 64 bits)."""
    rows, ch = x.shape
    nb = -(-ch // 32)
    q, ex, v = np.zeros((rows, ch), np.int8), np.zeros((rows, nb), np.uint8), np.zeros((rows, ch))
    for r in range(rows):
        for b in range(nb):
            t = x[r, 32 * b:32 * b + 32]
            if not np.isfinite(t).all():
                ex[r, b], v[r, 32 * b:32 * b + 32] = 255, np.nan
                continue
            k = -126
            while np.abs(t).max() > 127 * 2.0 ** k:
                k += 1
            ex[r, b] = k + 127
            q[r, 32 * b:32 * b + 32] = np.rint(t / 2.0 ** k)
            v[r, 32 * b:32 * b + 32] = q[r, 32 * b:32 * b + 32] * 2.0 ** k
    return q, ex, v


def kept8_of_many(x):
    """The same for many finite rows at once."""
    rows, ch = x.shape
    nb = -(-ch // 32)
    t = np.zeros((rows, nb * 32))
    t[:, :ch] = x
    t = t.reshape(rows, nb, 32)
    top = np.abs(t).max(2, keepdims=True)
    k = np.maximum(np.frexp(top)[1] - 7, -126)          # top < 2^(k + 7): k, or the next one
    k += top > 127 * 2.0 ** k
    k[top == 0] = -126
    q = np.rint(t / 2.0 ** k)
    flat = lambda a: a.reshape(rows, nb * 32)[:, :ch]      # noqa: E731
    return flat(q).astype(np.int8), (k[:, :, 0] + 127).astype(np.uint8), flat(q * 2.0 ** k)


def _rows(seed, rows, ch, offset=0.0):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, ch)) * (0.5 + r.random((rows, 1))) + 0.3 * r.standard_normal((rows, 1)) + offset
    x[:, r.integers(0, ch)] *= 8
    return x


def check_norm(lpm, name, rows, ch, keep8=False, affine=True, dx_acc=False, acc=False, offset=0.0, eps=1e-5):
    import torch
    dt = lpm.BF16 if name == "bf16" else lpm.F32
    r = np.random.default_rng(rows * 31 + ch)
    xt, dyt = _torch(_rows(rows + ch, rows, ch, offset), name), _torch(r.standard_normal((rows, ch)), name)
    g = (1 + 0.2 * r.standard_normal(ch)).astype(np.float32) if affine else None
    b = (0.2 * r.standard_normal(ch)).astype(np.float32) if affine else None
    dx0 = _torch(r.standard_normal((rows, ch)), name)
    dg0, db0 = (r.standard_normal(ch).astype(np.float32) for _ in range(2))
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()      # noqa: E731
    x, dy, dx, gamma, beta, dg, db = xt.cuda(), dyt.cuda(), dx0.cuda(), dev(g), dev(b), dev(dg0), dev(db0)
    y, stats = torch.full((rows, ch), 7.0).to(xt.dtype).cuda(), torch.zeros(rows * 2, device="cuda")
    kept = _bytes(lpm.lpm_ckpt8_bytes(rows, ch)) if keep8 else None
    ws = _bytes(lpm.lpm_norm_ws_bytes(rows, ch, dt))
    lpm.lpm_norm_forward(rows, ch, dt, x, gamma, beta, eps, y, stats, kept)
    lpm.lpm_norm_backward(rows, ch, dt, None if keep8 else x, kept, stats, dy, gamma, dx, dg, db, dx_acc, acc, ws)
    torch.cuda.synchronize()

    X, DY = _np(xt), _np(dyt)
    G, B = (g.astype(np.float64), b.astype(np.float64)) if affine else (np.ones(ch), np.zeros(ch))
    mu = X.mean(1, keepdims=True)
    rs = 1 / np.sqrt(((X - mu) ** 2).mean(1, keepdims=True) + np.float64(np.float32(eps)))
    big = np.abs(X).max(1, keepdims=True)
    H = (X - mu) * rs
    herr = 128 * U * (np.abs(H) + rs * big)
    y_ref = G * H + B
    assert (np.abs(_np(y) - y_ref) <= HALF[name] * np.abs(y_ref) * 1.01 + np.abs(G) * herr + 4 * U * np.abs(B)).all()
    np.testing.assert_allclose(_np(stats).reshape(rows, 2)[:, :1], mu, rtol=0, atol=(100 * U * big).max())
    np.testing.assert_allclose(_np(stats).reshape(rows, 2)[:, 1:], rs, rtol=200 * U * (1 + (rs * big).max()))
    if keep8:
        q, ex, X = kept8(X) if rows < 600 else kept8_of_many(X)
        n = (rows * ch + 255) // 256 * 256
        got = kept.cpu().numpy()
        assert (got[:rows * ch].view(np.int8) == q.ravel()).all() and (got[n:n + ex.size] == ex.ravel()).all()
        H = (X - mu) * rs
    gg = DY * G
    dx_ref = rs * (gg - gg.mean(1, keepdims=True) - H * (gg * H).mean(1, keepdims=True)) + (_np(dx0) if dx_acc else 0)
    top = np.abs(gg).max(1, keepdims=True) * (1 + np.abs(H).max(1, keepdims=True)) ** 2 * (1 + rs * big)
    assert (np.abs(_np(dx) - dx_ref) <= HALF[name] * np.abs(dx_ref) * 1.01 + 256 * U * rs * top + 4 * U * np.abs(dx_ref)).all()
    chain = (rows / 256 + 128) * U
    herr_max = 128 * U * (np.abs(H) + rs * big)
    for got, ref, start, tol in ((dg, (DY * H).sum(0), dg0, chain * np.abs(DY * H).sum(0) + (np.abs(DY) * herr_max).sum(0)),
                                 (db, DY.sum(0), db0, chain * np.abs(DY).sum(0))):
        ref = ref + (start if acc else 0)
        assert (np.abs(_np(got) - ref) <= tol + 4 * U * (np.abs(ref) + np.abs(start))).all()


# channels: one, less and more than the four to 64 lanes and the block that share a row take, whole chunks of eight and not
@pytest.mark.parametrize("ch", [1, 3, 8, 31, 32, 33, 64, 65, 100, 128, 130, 256, 257, 512, 515, 1000, 1024, 1025, 2048, 2056, 4096, 4099, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_channels(lpm, name, ch):
    rows = 5 if ch > 1024 else 37
    check_norm(lpm, name, rows, ch)
    check_norm(lpm, name, 3, ch, keep8=True, affine=ch % 2 == 0, dx_acc=True, acc=True)


@pytest.mark.parametrize("rows,ch", [(1, 256), (2, 40), (1000, 72), (2500, 96), (513, 520), (129, 2050)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows(lpm, name, rows, ch):
    check_norm(lpm, name, rows, ch, keep8=rows % 2 == 1, acc=True)


def test_many_rows(lpm):
    """More rows than all blocks take in one turn, forward and backward."""
    check_norm(lpm, "bf16", 40000, 24)
    check_norm(lpm, "f32", 9000, 520)


# more rows than all blocks take in one turn, forward (2048 blocks of 256 threads' rows, 64 down to one) and backward (512), for every way to share a row
@pytest.mark.parametrize("rows,ch", [(140000, 8), (66000, 40), (33000, 100), (17000, 130), (9000, 257), (9000, 515), (9000, 1030), (2100, 2056), (2100, 4099), (2060, 8200)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows_of_several_turns(lpm, name, rows, ch):
    check_norm(lpm, name, rows, ch, keep8=(name == "bf16") == (ch % 2 == 0), dx_acc=ch % 3 == 0)


def test_checkpoint_of_many_rows_is_the_definition():
    r = np.random.default_rng(3)
    x = r.standard_normal((40, 70)) * 2.0 ** r.integers(-130, 100, (40, 1))
    x[3], x[4, :32], x[5, 5] = 0, 127 * 2.0 ** -9, 2.0 ** 90
    for a, b in zip(kept8(x), kept8_of_many(x)):
        assert (a == b).all()


def test_rows_far_from_zero(lpm):
    """A mean a thousand times the spread: the variance comes from differences, not from the difference of two squares."""
    check_norm(lpm, "f32", 9, 300, offset=1000.0)


def test_constant_and_zero_rows(lpm):
    import torch
    for name, dt in (("f32", lpm.F32), ("bf16", lpm.BF16)):
        x = torch.zeros(4, 48).to(_torch(np.zeros(1), name).dtype)
        x[1], x[2], x[3, 5] = 3.0, -0.5, 1.0
        x, y, stats = x.cuda(), torch.ones(4, 48).to(x.dtype).cuda(), torch.zeros(8, device="cuda")
        lpm.lpm_norm_forward(4, 48, dt, x, None, None, 1e-5, y, stats)
        torch.cuda.synchronize()
        assert (_np(y)[:3] == 0).all() and np.isfinite(_np(y)).all()


def test_in_place_and_without_gradients(lpm):
    """y may be x, dx may be dy, and neither statistics nor weight gradients have to be asked for."""
    import torch
    x = _torch(_rows(5, 70, 136), "bf16").cuda()
    dy = _torch(_rows(6, 70, 136), "bf16").cuda()
    y, dx, stats = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(140, device="cuda")
    lpm.lpm_norm_forward(70, 136, lpm.BF16, x, None, None, 1e-5, y, stats)
    lpm.lpm_norm_backward(70, 136, lpm.BF16, x, None, stats, dy, None, dx)
    x2, dy2 = x.clone(), dy.clone()
    lpm.lpm_norm_forward(70, 136, lpm.BF16, x2, None, None, 1e-5, x2)
    lpm.lpm_norm_backward(70, 136, lpm.BF16, x, None, stats, dy2, None, dy2)
    torch.cuda.synchronize()
    assert torch.equal(x2, y) and torch.equal(dy2, dx)


def test_no_rows(lpm):
    """No rows: nothing is read, and gradients that are not accumulated become zero."""
    import torch
    e, dg, db = torch.zeros(0, device="cuda"), torch.full((12,), 1.0, device="cuda"), torch.full((12,), 1.0, device="cuda")
    lpm.lpm_norm_forward(0, 12, lpm.F32, e, None, None, 1e-5, e)
    lpm.lpm_norm_backward(0, 12, lpm.F32, e, None, e, e, None, e, dg, db, accumulate=True)
    torch.cuda.synchronize()
    assert (dg == 1).all() and (db == 1).all()
    lpm.lpm_norm_backward(0, 12, lpm.F32, e, None, e, e, None, e, dg, db)
    lpm.lpm_ckpt8_pack(0, 12, lpm.F32, e, e)
    torch.cuda.synchronize()
    assert (dg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("ch", [1, 7, 31, 32, 40, 100, 257, 1000])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_checkpoint(lpm, name, ch):
    """Bytes and values from the definition: ties, zeros, the largest and smallest numbers, borders of the exponent, infinities and NaN."""
    import torch
    dt, rows = (lpm.BF16, 41) if name == "bf16" else (lpm.F32, 41)
    x = _rows(ch, rows, ch)
    x[0], x[1, 0], x[2], x[3], x[4] = 0, 127.0, x[2] * 2.0 ** -120, x[3] * 2.0 ** 100, np.rint(x[4] * 4) / 2
    x[5, 0], x[6, 0], x[7] = 128.0, 127.5, 2.0 ** -133
    x[8, 0], x[9, ch - 1], x[10, ch // 2] = np.inf, np.nan, -np.inf
    x[11, 0] = 3.3e38
    xt = _torch(x, name)
    n = lpm.lpm_ckpt8_bytes(rows, ch)
    kept, back = _bytes(n), xt.clone().cuda()
    lpm.lpm_ckpt8_pack(rows, ch, dt, xt.cuda(), kept)
    lpm.lpm_ckpt8_unpack(rows, ch, dt, kept, back)
    torch.cuda.synchronize()
    q, ex, v = kept8(_np(xt))
    at = (rows * ch + 255) // 256 * 256
    got = kept.cpu().numpy()
    assert n == at + ex.size
    assert (got[:rows * ch].view(np.int8) == q.ravel()).all() and (got[at:at + ex.size] == ex.ravel()).all()
    np.testing.assert_array_equal(_np(back), v)


def test_checkpoint_of_many_rows(lpm):
    """More pieces than one block's, with rows that begin anywhere in them."""
    import torch
    for rows, ch in ((3000, 33), (700, 264), (2, 70000)):
        xt = _torch(_rows(ch, rows, ch), "bf16")
        kept, back = _bytes(lpm.lpm_ckpt8_bytes(rows, ch)), torch.zeros(rows, ch).to(xt.dtype).cuda()
        lpm.lpm_ckpt8_pack(rows, ch, lpm.BF16, xt.cuda(), kept)
        lpm.lpm_ckpt8_unpack(rows, ch, lpm.BF16, kept, back)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(_np(back), kept8(_np(xt))[2])


@pytest.mark.parametrize("name,rows,ch", [("bf16", 70001, 999), ("f32", 40001, 1003), ("bf16", 140000, 512)])
def test_checkpoint_larger_than_half_of_the_cache(lpm, name, rows, ch):
    """Values that go past the caches: the definition's, odd channels and whole chunks."""
    import torch
    dt = lpm.BF16 if name == "bf16" else lpm.F32
    xt = _torch(_rows(ch, rows, ch), name)
    kept, back = _bytes(lpm.lpm_ckpt8_bytes(rows, ch)), torch.full((rows * ch + 8,), 3.0).to(xt.dtype).cuda()
    lpm.lpm_ckpt8_pack(rows, ch, dt, xt.cuda(), kept)
    lpm.lpm_ckpt8_unpack(rows, ch, dt, kept, back)
    torch.cuda.synchronize()
    got = _np(back)
    assert (got[rows * ch:] == 3).all()
    np.testing.assert_array_equal(got[:rows * ch].reshape(rows, ch), kept8_of_many(_np(xt))[2])


# (rows of positions, image sizes) x channels: a projection, odd channels, a filter with padding
@pytest.mark.parametrize("g", [dict(m=300, h=1, w=1, cin=64, cout=96, kh=1, kw=1, stride=1, pad=0), dict(m=50, h=1, w=1, cin=37, cout=10, kh=1, kw=1, stride=1, pad=0),
                               dict(m=2, h=9, w=7, cin=40, cout=24, kh=3, kw=3, stride=1, pad=1)], ids=lambda g: "%dx%d_%d_%d" % (g["m"], g["h"], g["cin"], g["cout"]))
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_weight_gradient_of_a_checkpoint(lpm, name, g):
    """The bits of lpm_conv_wgrad for the unpacked input, and the 64-bit sum for what the checkpoint stands for."""
    import torch
    dt = lpm.BF16 if name == "bf16" else lpm.F32
    rows = g["m"] * g["h"] * g["w"]
    xt, dzt = _torch(_rows(1, rows, g["cin"]), name), _torch(_rows(2, rows, g["cout"]), name)
    kept, x = _bytes(lpm.lpm_ckpt8_bytes(rows, g["cin"])), xt.cuda()
    lpm.lpm_ckpt8_pack(rows, g["cin"], dt, x, kept)
    nw = g["cout"] * g["kh"] * g["kw"] * g["cin"]
    start = torch.randn(nw)
    dw, ref = start.clone().cuda(), start.clone().cuda()
    lpm.lpm_conv_wgrad_ckpt8(g, dt, kept, dzt.cuda(), dw, True, _bytes(lpm.lpm_conv_wgrad_ckpt8_ws_bytes(g, dt)))
    lpm.lpm_ckpt8_unpack(rows, g["cin"], dt, kept, x)
    lpm.lpm_conv_wgrad(g, dt, x, dzt.cuda(), ref, True, _bytes(lpm.lpm_conv_ws_bytes(g, dt)[2]))
    torch.cuda.synchronize()
    if g["kh"] == 1:
        v, dz = kept8(_np(xt))[2], _np(dzt)
        want = (dz.T @ v).ravel() + start.numpy()
        bound = (np.abs(dz).T @ np.abs(v)).ravel()
        assert (np.abs(_np(dw) - want) <= (rows + 8) * U * bound + 4 * U * np.abs(want)).all()
    np.testing.assert_allclose(_np(dw), _np(ref), rtol=0, atol=(rows + 8) * U * float(np.abs(_np(ref)).max()) * 4)


def test_norm_is_repeatable_and_replays_in_a_graph(lpm):
    """The same bits every time, from a captured graph too, with eager work between the replays."""
    import torch
    rows, ch = 700, 520
    x, dy = _torch(_rows(1, rows, ch), "bf16").cuda(), _torch(_rows(2, rows, ch), "bf16").cuda()
    gamma = torch.rand(ch).cuda()
    mk = lambda: dict(y=torch.zeros_like(x), dx=torch.zeros_like(x), st=torch.zeros(rows * 2, device="cuda"), dg=torch.zeros(ch, device="cuda"),      # noqa: E731
                      db=torch.zeros(ch, device="cuda"), kept=_bytes(lpm.lpm_ckpt8_bytes(rows, ch)), ws=_bytes(lpm.lpm_norm_ws_bytes(rows, ch, lpm.BF16)))
    a, b = mk(), mk()

    def once(o, s):
        lpm.lpm_norm_forward(rows, ch, lpm.BF16, x, gamma, None, 1e-5, o["y"], o["st"], o["kept"], s)
        lpm.lpm_norm_backward(rows, ch, lpm.BF16, None, o["kept"], o["st"], dy, gamma, o["dx"], o["dg"], o["db"], ws=o["ws"], stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(b, torch.cuda.current_stream())
    for k in range(3):
        once(a, torch.cuda.current_stream())
        for o in b.values():
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("y", "dx", "st", "dg", "db", "kept"):
            assert torch.equal(a[n], b[n]), (k, n)
