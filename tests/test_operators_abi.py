"""The operators' refusals and host-side functions (no GPU): a call that is refused has launched nothing."""
import ctypes as C

import numpy as np
import pytest

EINVAL, ESHAPE, EALIGN = -1, -2, -3


@pytest.fixture(scope="module")
def lpm():
    import paper_2207_11019_amd as lpm
    return lpm


def test_error_codes_are_the_headers():
    import os
    import re
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lpm.h")).read()
    for name, code in (("LPM_EINVAL", EINVAL), ("LPM_ESHAPE", ESHAPE), ("LPM_EALIGN", EALIGN)):
        assert re.search(r"#define %s\s+\(%d\)" % (name, code), hdr), name


A = 1 << 20          # an address that no call below gets to use


def refused(lpm, code, f, *a):
    with pytest.raises(lpm.LpmError) as e:
        f(*a)
    assert e.value.code == code and str(e.value), (code, str(e.value))


def test_checkpoints(lpm):
    for rows, ch in ((-1, 8), (1, 0), (1, -3), (1, (1 << 24) + 1), (1 << 41, 1), (1 << 38, 64)):
        refused(lpm, ESHAPE, lpm.lpm_ckpt8_bytes, rows, ch)
        refused(lpm, ESHAPE, lpm.lpm_ckpt8_pack, rows, ch, lpm.F32, A, A)
        refused(lpm, ESHAPE, lpm.lpm_ckpt8_unpack, rows, ch, lpm.BF16, A, A)
    for f in (lpm.lpm_ckpt8_pack, lpm.lpm_ckpt8_unpack):
        refused(lpm, EINVAL, f, 4, 8, 2, A, A)
        refused(lpm, EINVAL, f, 4, 8, lpm.F32, None, A)
        refused(lpm, EINVAL, f, 4, 8, lpm.F32, A, None)
        refused(lpm, EALIGN, f, 4, 8, lpm.F32, A + 16, A)
        refused(lpm, EALIGN, f, 4, 8, lpm.F32, A, A + 128)
        f(0, 8, lpm.F32, None, None)                     # nothing to do
    # [rows][channels] bytes to the next 256, and a byte for 32 channels
    for rows, ch in ((0, 5), (1, 1), (7, 100), (1000, 32), (3, 1025)):
        assert lpm.lpm_ckpt8_bytes(rows, ch) == (rows * ch + 255) // 256 * 256 + rows * -(-ch // 32)
    assert lpm.lib.lpm_ckpt8_bytes(1, 8, None) == EINVAL


def test_weight_gradient_of_a_checkpoint(lpm):
    g = dict(m=4, h=1, w=1, cin=8, cout=8, kh=1, kw=1, stride=1, pad=0)
    n = lpm.lpm_conv_wgrad_ckpt8_ws_bytes(g, lpm.BF16)
    assert n == 256 + lpm.lpm_conv_ws_bytes(g, lpm.BF16)[2]
    for args in ((None, A, A, False, A), (A, None, A, False, A), (A, A, None, False, A), (A, A, A, False, None)):
        refused(lpm, EINVAL, lpm.lpm_conv_wgrad_ckpt8, g, lpm.BF16, *args)
    for args in ((A + 2, A, A, False, A), (A, A + 16, A, False, A), (A, A, A + 4, False, A), (A, A, A, False, A + 64)):
        refused(lpm, EALIGN, lpm.lpm_conv_wgrad_ckpt8, g, lpm.BF16, *args)
    for bad in (dict(g, cin=0), dict(g, m=-1), dict(g, stride=0), dict(g, kh=2)):
        with pytest.raises(lpm.LpmError):
            lpm.lpm_conv_wgrad_ckpt8_ws_bytes(bad, lpm.BF16)
    assert lpm.lib.lpm_conv_wgrad_ckpt8_ws_bytes(None, lpm.F32, C.byref(C.c_size_t())) != 0


def test_norm(lpm):
    fwd, bwd = lpm.lpm_norm_forward, lpm.lpm_norm_backward
    for rows, ch in ((-1, 8), (1, 0), (1, 16385), (1 << 40, 2)):
        refused(lpm, ESHAPE, lpm.lpm_norm_ws_bytes, rows, ch, lpm.F32)
        refused(lpm, ESHAPE, fwd, rows, ch, lpm.F32, A, None, None, 1e-5, A)
        refused(lpm, ESHAPE, bwd, rows, ch, lpm.F32, A, None, A, A, None, A)
    refused(lpm, EINVAL, lpm.lpm_norm_ws_bytes, 1, 8, 7)
    refused(lpm, EINVAL, fwd, 4, 8, 2, A, None, None, 1e-5, A)
    for eps in (-1e-9, float("nan")):
        refused(lpm, EINVAL, fwd, 4, 8, lpm.F32, A, None, None, eps, A)
    refused(lpm, EINVAL, fwd, 4, 8, lpm.F32, None, None, None, 1e-5, A)
    refused(lpm, EINVAL, fwd, 4, 8, lpm.F32, A, None, None, 1e-5, None)
    for k in range(6):
        p = [A] * 6
        p[k] += 4
        refused(lpm, EALIGN, fwd, 4, 8, lpm.F32, p[0], p[1], p[2], 1e-5, p[3], p[4], p[5])
    fwd(0, 8, lpm.F32, None, None, None, 1e-5, None)
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, A, A, A, A, None, A)               # the input and its checkpoint
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, None, None, A, A, None, A)         # neither
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, A, None, None, A, None, A)
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, A, None, A, None, None, A)
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, A, None, A, A, None, None)
    refused(lpm, EINVAL, bwd, 4, 8, lpm.F32, A, None, A, A, None, A, A, None)   # a weight gradient without scratch
    refused(lpm, EALIGN, bwd, 4, 8, lpm.F32, A, None, A + 8, A, None, A)
    refused(lpm, EALIGN, bwd, 4, 8, lpm.F32, A, None, A, A, None, A, A + 32, None, False, False, A)


G = dict(m=2, heads=4, kv_heads=2, pq=5, pk=9, d=16, causal=1, n_buckets=8, reach=4)
BAD_SHAPES = [dict(m=-1), dict(pq=-1), dict(pk=-2), dict(pq=(1 << 28) + 1), dict(pk=(1 << 28) + 1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(heads=65540, kv_heads=2),
              dict(d=7), dict(d=129), dict(d=0), dict(n_buckets=-1), dict(n_buckets=65537), dict(reach=-1), dict(reach=2049), dict(ldq=63), dict(ldk=31), dict(ldv=31),
              dict(ldy=60), dict(ldq=(1 << 23) + 1), dict(heads=65535, kv_heads=1, d=128, m=1), dict(m=1 << 20, heads=60000, kv_heads=2)]


@pytest.mark.parametrize("bad", BAD_SHAPES, ids=lambda b: "_".join("%s%d" % i for i in b.items()))
def test_attention_shapes(lpm, bad):
    g = dict(G, **bad)
    for f in (lpm.lpm_attn_ws_bytes, lpm.lpm_attn_stats_bytes):
        code = ESHAPE if bad != dict(heads=65535, kv_heads=1, d=128, m=1) else None
        if code is None:                              # 65535 heads of 128 channels are 2^23 elements, less 128: the widest that is taken
            f(g, lpm.BF16)
        else:
            refused(lpm, code, f, g, lpm.BF16)
            refused(lpm, code, lpm.lpm_attn_forward, g, lpm.BF16, A, A, A, None, None, A, A, A, A, A)


def test_attention_arguments(lpm):
    fwd, bwd = lpm.lpm_attn_forward, lpm.lpm_attn_backward
    args = [A, A, A, None, None, A, A, A, A, A]           # q k v key_len q_start map table y stats ws
    refused(lpm, EINVAL, lpm.lpm_attn_ws_bytes, G, 2)
    for scale in (-1.0, float("nan"), float("inf"), 1e-31, 2e30):
        refused(lpm, EINVAL, lpm.lpm_attn_ws_bytes, dict(G, scale=scale), lpm.F32)
    for k in (0, 1, 2, 5, 6, 7):                           # q, k, v, map, table, y
        refused(lpm, EINVAL, fwd, G, lpm.BF16, *args[:k], None, *args[k + 1:])
    refused(lpm, EINVAL, fwd, dict(G, n_buckets=0), lpm.BF16, *args)            # a table that no bucket count goes with
    for k, off in ((0, 1), (1, 1), (2, 1), (3, 2), (4, 1), (5, 2), (6, 3), (7, 128), (8, 64), (9, 4)):
        refused(lpm, EALIGN, fwd, G, lpm.BF16, *args[:k], A + off, *args[k + 1:])
    refused(lpm, EALIGN, fwd, G, lpm.F32, A + 2, *args[1:])
    for g in (dict(G, m=0), dict(G, pq=0)):
        fwd(g, lpm.BF16, *([None] * 5), A, A, None)        # nothing to do
    back = [A, A, A, A, A, A, None, None, A, A, A, A, A, A, False, A]           # q k v y stats dy key_len q_start map table dq dk dv dtable accumulate ws
    for k in (0, 1, 2, 3, 4, 5, 8, 9, 10, 11, 12, 15):
        refused(lpm, EINVAL, bwd, G, lpm.BF16, *back[:k], None, *back[k + 1:])
    for k, off in ((3, 2), (4, 64), (5, 16), (10, 1), (11, 1), (12, 1), (13, 4), (15, 32)):
        refused(lpm, EALIGN, bwd, G, lpm.BF16, *back[:k], A + off, *back[k + 1:])
    refused(lpm, EINVAL, bwd, dict(G, n_buckets=0), lpm.BF16, A, A, A, A, A, A, None, None, None, None, A, A, A, A, False, A)      # dtable without a table
    few = dict(G, m=1, heads=8, kv_heads=1, pq=1, pk=1 << 16)
    assert lpm.lpm_attn_ws_bytes(few, lpm.BF16)[0] > 0                          # a single query: the keys go over several blocks, joined in scratch
    refused(lpm, EINVAL, fwd, few, lpm.BF16, A, A, A, None, None, A, A, A, A, None)


def test_tensors_are_checked_before_a_call(lpm):
    """Too small, of another type, not dense: refused by the binding (the device is not looked at where there is none)."""
    import torch
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)      # noqa: E731
    b = lambda n: torch.zeros(n, dtype=torch.uint8)               # noqa: E731
    with pytest.raises(ValueError):
        lpm.lpm_ckpt8_pack(4, 8, lpm.F32, z(31), b(300))
    with pytest.raises(ValueError):
        lpm.lpm_ckpt8_pack(4, 8, lpm.F32, z(32), b(259))
    with pytest.raises(ValueError):
        lpm.lpm_ckpt8_pack(4, 8, lpm.BF16, z(32), b(300))
    with pytest.raises(ValueError):
        lpm.lpm_ckpt8_unpack(4, 8, lpm.F32, b(300), z(8, 4).t())
    with pytest.raises(ValueError):
        lpm.lpm_norm_forward(4, 8, lpm.F32, z(32), z(7), z(8), 1e-5, z(32))
    with pytest.raises(ValueError):
        lpm.lpm_norm_forward(4, 8, lpm.F32, z(32), z(8), z(8), 1e-5, z(32), z(7))
    with pytest.raises(ValueError):
        lpm.lpm_norm_backward(4, 8, lpm.F32, z(32), None, z(8), z(32), z(8), z(32), z(8), z(8), ws=b(lpm.lpm_norm_ws_bytes(4, 8, lpm.F32) - 1))
    q, kv, y, tb, mp = z(2, 5, 64), z(2, 9, 32), z(2, 5, 64), z(4, 8), z(9, t=torch.int32)
    st, ws = b(lpm.lpm_attn_stats_bytes(G, lpm.F32)), b(max(256, lpm.lpm_attn_ws_bytes(G, lpm.F32)[1]))
    ok = [q, kv, kv, None, None, mp, tb, y, st, ws]
    for k, t in ((0, z(2, 5, 63)), (0, z(2, 5, 64, t=torch.bfloat16)), (1, z(2, 9, 31)), (2, z(32, 9, 2).transpose(0, 2)), (3, z(1, t=torch.int32)), (3, z(2)), (4, z(2, t=torch.int64)),
                 (5, z(8, t=torch.int32)), (5, z(9)), (6, z(31)), (6, z(4, 8, t=torch.bfloat16)), (7, z(2, 5, 60)), (8, b(8))):
        with pytest.raises(ValueError):
            lpm.lpm_attn_forward(G, lpm.F32, *ok[:k], t, *ok[k + 1:])
    # a part of a packed tensor reaches as far as the geometry says, not as far as the view
    packed = z(2, 5, 192)
    with pytest.raises(ValueError):
        lpm.lpm_attn_forward(dict(G, ldq=192, heads=4), lpm.F32, packed[:, :, 129:], *ok[1:])


def plain_buckets(n_buckets, reach, both):
    """Nearest distances one bucket each, the rest in equal steps of the logarithm (64 bits)."""
    n = n_buckets // 2 if both else n_buckets
    exact, out = max(1, n // 2), []
    for rel in range(-reach, reach + 1):
        r = abs(rel) if both else max(0, -rel)
        if r >= exact:
            r = min(n - 1, exact + int(np.log(r / exact) / np.log(max(reach, exact + 1) / exact) * (n - exact)))
        out.append(r + (n if both and rel > 0 else 0))
    return out


@pytest.mark.parametrize("n,reach,both", [(32, 128, True), (32, 128, False), (8, 20, True), (2, 5, True), (1, 5, False), (64, 2048, False), (6, 0, True), (40, 3, True), (5, 17, False)])
def test_bucket_map(lpm, n, reach, both):
    got = lpm.lpm_relbias_buckets(n, reach, both)
    assert got == plain_buckets(n, reach, both) and min(got) >= 0 and max(got) < n
    near = got[reach::-1]                             # from the query's own position towards older keys
    assert all(a <= b for a, b in zip(near, near[1:])) and near[0] == 0
    if both:
        assert all(b >= n // 2 for b in got[reach + 1:]) and all(b < n // 2 for b in near)
    else:
        assert all(b == 0 for b in got[reach:])


def test_bucket_map_refusals(lpm):
    for n, reach, both in ((0, 4, False), (1, 4, True), (7, 4, True), (8, -1, True), (8, 2049, False), (-2, 3, True)):
        refused(lpm, EINVAL, lpm.lpm_relbias_buckets, n, reach, both)
    assert lpm.lib.lpm_relbias_buckets(8, 4, 1, None) == EINVAL
