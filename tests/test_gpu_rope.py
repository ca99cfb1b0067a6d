"""Rotary positions of several axes on the device against the fp64 oracle."""
import numpy as np
import pytest

from oracle import rope_ref

pytestmark = pytest.mark.gpu


def _t(x, dt):
    import torch
    return torch.tensor(np.ascontiguousarray(x)).to(dt).cuda()


def _bound(want, size, dt, norm):
    """Angles: 2^-25 half turns from fp64 to fp32, sine and cosine two units of the last
    place: below 2^-21 of |a| + |b|.  The norm: up to 256 squares summed in chains of 16
    and 4 exchanges, root, quotient and two products, below 32 roundings of 2^-24.  The
    rotation's own: 3.  Last, half a step of the result."""
    import torch
    c = 2.0 ** -21 + (32 * 2.0 ** -24 if norm else 0) + 3 * 2.0 ** -24
    half = torch.finfo(dt).eps / 2
    return half * np.abs(want) + (1 + half) * c * size + 1e-30


def _check(got, x, pos, sections, theta, g, eps, mixed, dt, name):
    want, size = rope_ref.rope(x, pos, sections, theta, g=g, eps=eps, interleaved=mixed)
    r = (np.abs(got.double().cpu().numpy() - want) / _bound(want, size, dt, g is not None)).max()
    print(f"    {name}: {r:.3f} of the bound", flush=True)
    assert r <= 1


CASES = [
    (1, 32, 8, 128, [64], False), (3, 4, 1, 64, [32], False), (17, 5, 2, 256, [128], False),
    (40, 8, 8, 128, [24, 20, 20], True), (40, 3, 1, 128, [16, 24, 24], False),
    (9, 2, 2, 64, [8, 8, 8, 8], True), (700, 14, 2, 64, [12, 10, 2], False),
    (33, 1, 1, 256, [24], False), (5, 7, 3, 128, [0, 32], False), (4100, 2, 1, 128, [64], False),
    (21, 40, 8, 128, [8], False), (130, 16, 16, 256, [44, 42, 42], True)]


@pytest.mark.parametrize("tokens,nh,nkv,hd,sections,mixed", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
def test_rope(tokens, nh, nkv, hd, sections, mixed, dtype, norm):
    import torch
    from paper_2608_02438_amd.xpress import rope
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(tokens + hd)
    fused = _t(rng.normal(size=(tokens, (nh + 2 * nkv) * hd)) *
               2.0 ** rng.integers(-8, 8, size=(tokens, 1)), dt)
    q = fused[:, :nh * hd].unflatten(1, (nh, hd))
    k = fused[:, nh * hd:(nh + nkv) * hd].unflatten(1, (nkv, hd))
    gq, gk = (_t(1 + 0.2 * rng.normal(size=hd), dt) for _ in range(2)) if norm else (None, None)
    pos = rng.integers(-1000, 1 << 20, size=(len(sections), tokens))
    pos[:, -1] = [0, 2 ** 31 - 1, -2 ** 31, 1][:len(sections)]
    dpos = _t(pos, torch.int32)
    print(f"rope: {tokens} {nh} {nkv} {hd} {sections} {mixed} {dtype} norm={norm}", flush=True)
    kw = dict(theta=1e6, k=k, g_q=gq, g_k=gk, eps=1e-5, interleaved=mixed)
    yq, yk = rope(q, dpos, sections, **kw)
    for name, y, x, g in (("q", yq, q, gq), ("k", yk, k, gk)):
        _check(y, x.double().cpu().numpy(), pos, sections, 1e6,
               None if g is None else g.double().cpu().numpy(), float(np.float32(1e-5)), mixed, dt,
               name)
    # in place, beside what the rows hold besides
    rest = fused[:, (nh + nkv) * hd:].clone()
    rope(q, dpos, sections, q_out=q, k_out=k, **kw)
    assert q.equal(yq) and k.equal(yk) and fused[:, (nh + nkv) * hd:].equal(rest)


def test_queries_alone_row_distances_and_a_view_of_positions():
    import torch
    from paper_2608_02438_amd.xpress import rope
    rng = np.random.default_rng(4)
    q = _t(rng.normal(size=(6, 3, 64)), torch.bfloat16)
    wide = torch.full((6, 3 * 64 + 40), 7.0, dtype=torch.bfloat16, device="cuda")
    pos = _t(rng.integers(0, 99, size=(2, 50)), torch.int32)
    y, none = rope(q, pos[:, 10:16], [20, 12], 1e4, q_out=wide[:, 24:24 + 192].unflatten(1, (3, 64)))
    assert none is None and (wide[:, :24] == 7).all() and (wide[:, 216:] == 7).all()
    _check(y, q.double().cpu().numpy(), pos[:, 10:16].cpu().numpy(), [20, 12], 1e4, None, 0, False,
           torch.bfloat16, "q")
    e, _ = rope(q[:0], pos[:, :0], [20, 12], 1e4)
    assert e.shape == (0, 3, 64)


def test_back_and_on_again():
    """A key rotated for p is, rotated by d more, one for p + d."""
    import torch
    from paper_2608_02438_amd.xpress import rope
    rng = np.random.default_rng(6)
    k = _t(rng.normal(size=(50, 2, 128)), torch.float32)
    p = _t(rng.integers(0, 4000, size=(1, 50)), torch.int32)
    a, _ = rope(k, p, [64], 1e6)
    b, _ = rope(a, -p + 77, [64], 1e6)
    c, _ = rope(k, 0 * p + 77, [64], 1e6)
    # two results of the bound above in turn, and one
    size = rope_ref.rope(k.double().cpu().numpy(), 0 * p.cpu().numpy(), [64], 1e6)[1]
    assert (np.abs((b - c).double().cpu().numpy()) <= 3 * 2.0 ** -20 * 2 * size).all()


def test_captured_replayed_and_on_another_stream():
    import torch
    from paper_2608_02438_amd.xpress import rope
    rng = np.random.default_rng(7)
    q, k = (_t(rng.normal(size=(9, h, 128)), torch.bfloat16) for h in (8, 2))
    pos = _t(np.arange(9)[None], torch.int32)
    eager = rope(q, pos, [64], 1e6, k=k)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = rope(q, pos, [64], 1e6, k=k, stream=s)
    s.synchronize()
    assert other[0].equal(eager[0]) and other[1].equal(eager[1])
    out = [torch.zeros_like(x) for x in (q, k)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope(q, pos, [64], 1e6, k=k, q_out=out[0], k_out=out[1])
    for step in (0, 5, 100000):
        pos.copy_(_t(np.arange(9)[None] + step, torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = rope(q, pos, [64], 1e6, k=k)
        assert out[0].equal(want[0]) and out[1].equal(want[1])


def test_the_binding_refuses():
    import torch
    from paper_2608_02438_amd import xpress as X
    q = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    bad = [lambda: X.rope(q.half(), pos, [64], 1e6), lambda: X.rope(q.cpu(), pos, [64], 1e6),
           lambda: X.rope(q, pos.long(), [64], 1e6), lambda: X.rope(q, pos[:, :3], [64], 1e6),
           lambda: X.rope(q, pos.cpu(), [64], 1e6), lambda: X.rope(q, pos, [32, 32], 1e6),
           lambda: X.rope(q, pos, [64], 1e6, rot_dim=64), lambda: X.rope(q, pos, [], 1e6),
           lambda: X.rope(q, pos, [64], 1e6, g_q=torch.ones(128).cuda()),
           lambda: X.rope(q, pos, [64], 1e6, g_k=q[0, 0]),
           lambda: X.rope(q, pos, [64], 1e6, k=q.float()),
           lambda: X.rope(q, pos, [64], 1e6, k=q[:3]),
           lambda: X.rope(q, pos, [64], 1e6, q_out=q[:, :1]),
           lambda: X.rope(q.transpose(1, 2).contiguous().transpose(1, 2), pos, [64], 1e6)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: X.rope(q, pos, [60], 1e6), lambda: X.rope(q, pos, [72], 1e6),
              lambda: X.rope(q[..., :32].contiguous(), pos, [16], 1e6),
              lambda: X.rope(q, pos, [64], 0.0), lambda: X.rope(q, pos, [64], 1e6, eps=-1.0)):
        with pytest.raises(X.XpError):
            f()
