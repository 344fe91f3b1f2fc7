"""Head norms with the position rotation, forward and backward, against the formulas in 64 bits.

Tolerances, elementwise.  u is the unit roundoff of the storage type, E = 2^-24, D the head dimension.
  - A sum of D squares in binary32 is off by at most D E of itself, its root by half of that; with the division, the
    root and the products a normalised element is off by (D + 8) E of itself.
  - cos and sin are off by 2^-23 = 2 E; with the two products and the sum a rotated element of a pair (a, b) is off by
    another 6 E of |a| + |b|.
  - Backward, S(u x) is off by D E of the sum of magnitudes.  The sums over n rows are off by n E of theirs.
  - A result is rounded once: u of it, or the type's least subnormal."""
import math

import pytest
import torch

import paper_2608_02611_amd as kb
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
E = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def freqs_of(rot, base=10000.0):
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    return (base ** (-2.0 * i / max(rot, 1))).float()


def turn(x, positions, freqs, interleaved, back=False):
    """The rotation in 64 bits; also the sum of magnitudes of each element's pair."""
    r = 0 if freqs is None else 2 * freqs.numel()
    out, mag = x.clone(), x.abs()
    if r:
        order = torch.arange(r, device="cuda")
        ia, ib = (order[0::2], order[1::2]) if interleaved else (order[:r // 2], order[r // 2:])
        a, b = x[..., ia], x[..., ib]
        t = positions.double()[..., None, None] * freqs.double()
        c, s = torch.cos(t), torch.sin(t) * (-1.0 if back else 1.0)
        out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
        mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
    return out, mag


def close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol) & ~(torch.isnan(want) & torch.isnan(got)) & ~(want == got)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of the tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol)[bad].max()))


def check_forward(x, w, eps, positions, freqs, interleaved, y):
    D, u = x.shape[-1], U[x.dtype]
    X = x.double()
    W = torch.ones(D, device="cuda").double() if w is None else w.double()
    g = X / (X.pow(2).mean(-1, keepdim=True) + eps).sqrt() * W
    want, mag = turn(g, positions, freqs, interleaved)
    close(y, want, (D + 14) * E * mag + 1.01 * u * want.abs() + TINY[x.dtype], "y")


def check_backward(dy, x, w, eps, positions, freqs, interleaved, dx, dw):
    D, u = x.shape[-1], U[x.dtype]
    X = x.double()
    W = torch.ones(D, device="cuda").double() if w is None else w.double()
    r = 1.0 / (X.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    z = X * r
    g, mag = turn(dy.double(), positions, freqs, interleaved, back=True)
    eg = 6 * E * mag
    m, mm = (g * W * z).mean(-1, keepdim=True), ((g * W * z).abs() + (eg * W * z).abs()).mean(-1, keepdim=True)
    if dx is not None:
        want = r * (g * W - z * m)
        tol = r * ((eg * W).abs() + (2 * D + 24) * E * ((g * W).abs() + z.abs() * mm) + z.abs() * (eg * W * z).abs().mean(-1, keepdim=True))
        close(dx, want, tol + 1.01 * u * want.abs() + TINY[x.dtype], "dx")
    if dw is not None:
        axes = tuple(range(x.dim() - 1))
        n = x[..., 0].numel()
        want, terms = (g * z).sum(axes), (g * z).abs().sum(axes)
        tol = (eg * z.abs()).sum(axes) + (n + D + 16) * E * terms
        close(dw, want, tol + 1.01 * U[dw.dtype] * want.abs() + TINY[dw.dtype], "dw")


def run(x, wdtype, rot, interleaved, far=5000, seed=0, eps=EPS, weights=True):
    """One forward and one backward call on q and k, checked; returns their results."""
    q, k = x
    d, lead = q.shape[-1], q.shape[:-2]
    wq, wk = ((normal((d,), wdtype, seed + 11 + i, 0.2) + 1.0).to(wdtype) if weights else None for i in range(2))
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    positions = torch.randint(-far, far, lead, generator=g, device="cuda", dtype=torch.int32) if rot else None
    freqs = freqs_of(rot) if rot else None
    args = (eps, positions, freqs, interleaved)
    yq, yk = kb.kb_qk_norm_forward(q, k, wq, wk, *args)
    dyq, dyk = normal(q.shape, q.dtype, seed + 21), normal(k.shape, k.dtype, seed + 22)
    dq, dk, dwq, dwk = kb.kb_qk_norm_backward(dyq, dyk, q, k, wq, wk, *args)
    check_forward(q, wq, *args, yq)
    check_forward(k, wk, *args, yk)
    check_backward(dyq, q, wq, *args, dq, dwq)
    check_backward(dyk, k, wk, *args, dk, dwk)
    return yq, yk, dq, dk, dwq, dwk


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (96, 48), (80, 40), (40, 20), (64, 0), (2, 2), (1, 0), (37, 14),
                                     (34, 34), (256, 256), (255, 254), (200, 8)])
def test_dimensions(dtype, wdtype, interleaved, dim, rot):
    t = DT[dtype]
    run((normal((9, 5, dim), t, 1), normal((9, 2, dim), t, 2)), DT[wdtype], rot, interleaved)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads,kv_heads", [(1, 1, 1), (1, 32, 8), (3, 0, 2), (3, 2, 0), (0, 4, 2), (700, 12, 12), (5000, 3, 1), (70, 130, 1)])
def test_sizes(dtype, tokens, heads, kv_heads):
    """Also no heads of one kind, and no token: then the weights' gradients are zeros."""
    t = DT[dtype]
    got = run((normal((tokens, heads, 64), t, 1), normal((tokens, kv_heads, 64), t, 2)), t, 64, False)
    if tokens == 0 or heads == 0:
        assert torch.all(got[4] == 0)
    if tokens == 0 or kv_heads == 0:
        assert torch.all(got[5] == 0)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_columns_of_one_buffer(dtype):
    """q and k as columns of a projection, at odd addresses, with a leading batch; gradients into columns of one buffer.
    What lies between them stays."""
    t = DT[dtype]
    b, n, h, hk, d = 2, 17, 3, 2, 24
    wide = (h + hk) * d + 5
    x = normal((b * n * wide + 1,), t, 1)[1:].view(b, n, wide)
    q, k = x[..., :h * d].unflatten(-1, (h, d)), x[..., h * d:(h + hk) * d].unflatten(-1, (hk, d))
    positions = torch.arange(n, device="cuda", dtype=torch.int32).repeat(b, 1)
    args = (EPS, positions, freqs_of(16), False)
    want = kb.kb_qk_norm_forward(q.contiguous(), k.contiguous(), None, None, *args)
    got = kb.kb_qk_norm_forward(q, k, None, None, *args)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    check_forward(q, None, *args, got[0])
    dy = normal((b, n, h, d), t, 2), normal((b, n, hk, d), t, 3)
    dx = torch.full_like(x, 7.0)
    dq, dk = dx[..., :h * d].unflatten(-1, (h, d)), dx[..., h * d:(h + hk) * d].unflatten(-1, (hk, d))
    res = kb.kb_qk_norm_backward(*dy, q, k, None, None, *args, dq=dq, dk=dk)
    check_backward(dy[0], q, None, *args, dq, res[2])
    check_backward(dy[1], k, None, *args, dk, res[3])
    assert torch.all(dx[..., (h + hk) * d:] == 7.0)
    other = kb.kb_qk_norm_backward(*dy, q.contiguous(), k.contiguous(), None, None, *args)
    assert torch.equal(dq, other[0]) and torch.equal(dk, other[1]) and torch.equal(res[2], other[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(dtype, interleaved):
    t = DT[dtype]
    q, k, w = normal((300, 6, 80), t, 1), normal((300, 2, 80), t, 2), normal((80,), t, 3)
    positions = torch.arange(300, device="cuda", dtype=torch.int32)
    args = (w, w, EPS, positions, freqs_of(48), interleaved)
    want = kb.kb_qk_norm_forward(q, k, *args)
    q1, k1 = q.clone(), k.clone()
    kb.kb_qk_norm_forward(q1, k1, *args, q_out=q1, k_out=k1)
    assert torch.equal(q1, want[0]) and torch.equal(k1, want[1])


def test_far_positions():
    """cos and sin themselves: rows of sqrt(1/2) ones and zeros are (1, .., 0, ..) after the norm, up to eps, so that the
    output is (cos, .., sin, ..), off by the 2^-23 of these and the (D + 8) E of the norm."""
    n = 64
    g = torch.Generator(device="cuda").manual_seed(1)
    positions = torch.randint(-2 ** 31, 2 ** 31 - 1, (400,), generator=g, device="cuda", dtype=torch.int32)
    positions[:8] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1 << 20, 3], dtype=torch.int32, device="cuda")
    freqs = torch.cat([freqs_of(n // 2), torch.logspace(-6, 5.5, n // 2 - n // 4, device="cuda", dtype=torch.float64).float()])
    assert freqs.numel() == n // 2 and float(freqs.max()) * 2 ** 31 < 2 ** 50
    x = torch.zeros((400, 1, n), device="cuda")
    x[..., :n // 2] = 0.5 ** 0.5
    y, _ = kb.kb_qk_norm_forward(x, x, None, None, 0.0, positions, freqs)
    turns = (positions.double()[:, None] * freqs.double()).cpu().numpy()  # exact below 2^53: 31 and 24 bits, of which few are set
    c, s = torch.from_numpy(__import__("numpy").cos(turns)), torch.from_numpy(__import__("numpy").sin(turns))
    # the product's own rounding in 64 bits, up to 2^-53 of 2^50
    slack = torch.from_numpy(abs(turns)) * 2.0 ** -53
    norm = x[0, 0, 0].double().item() / math.sqrt(x[0, 0, 0].double().item() ** 2 / 2)
    for got, want in ((y[:, 0, :n // 2], c), (y[:, 0, n // 2:], s)):
        off = (got.double().cpu() - norm * want).abs()
        tol = norm * (2.0 ** -23 + slack) + norm * (n + 8) * E * want.abs() + E
        assert torch.all(off <= tol), float((off / tol).max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite(dtype):
    """A NaN or an infinity in a row reaches that row alone, and the weight's gradient."""
    t = DT[dtype]
    q, k = normal((40, 4, 64), t, 1), normal((40, 2, 64), t, 2)
    positions = torch.arange(40, device="cuda", dtype=torch.int32)
    args = (None, None, EPS, positions, freqs_of(64))
    want = kb.kb_qk_norm_forward(q, k, *args)
    dy = normal(q.shape, t, 3), normal(k.shape, t, 4)
    grads = kb.kb_qk_norm_backward(*dy, q, k, *args)
    bad = q.clone()
    bad[7, 1, 3], bad[9, 2, 60] = float("nan"), float("inf")
    got = kb.kb_qk_norm_forward(bad, k, *args)
    other = kb.kb_qk_norm_backward(*dy, bad, k, *args)
    row = torch.zeros((40, 4), dtype=torch.bool, device="cuda")
    row[7, 1] = row[9, 2] = True
    assert torch.equal(got[0][~row], want[0][~row]) and torch.equal(got[1], want[1])
    assert torch.isnan(got[0][7, 1]).all() and torch.isnan(got[0][9, 2, 60])
    assert torch.equal(other[0][~row], grads[0][~row]) and torch.equal(other[1], grads[1])
    assert torch.isnan(other[2]).any() and torch.equal(other[3], grads[3])


def test_zero_rows():
    """Rows of zeros stay zeros; with dy their gradient is that of x / sqrt(eps)."""
    q = torch.zeros((3, 2, 32), device="cuda")
    dy = normal(q.shape, torch.float32, 1)
    y, _ = kb.kb_qk_norm_forward(q, q, None, None, EPS)
    assert torch.all(y == 0)
    dq, _, dwq, _ = kb.kb_qk_norm_backward(dy, dy, q, q, None, None, EPS)
    check_backward(dy, q, None, EPS, None, None, False, dq, dwq)


def test_gradients_against_differences():
    """The gradient of S(dy y) along a direction against a central difference in 64 bits of the formula."""
    q, k = normal((5, 3, 48), torch.float32, 1), normal((5, 2, 48), torch.float32, 2)
    w = normal((48,), torch.float32, 3) + 1.0
    positions, freqs = torch.arange(5, device="cuda", dtype=torch.int32) * 7, freqs_of(32)
    dy = normal(q.shape, torch.float32, 4)
    dq, _, dw, _ = kb.kb_qk_norm_backward(dy, torch.zeros_like(k), q, k, w, w, EPS, positions, freqs, True)

    def loss(x, w):
        g = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
        return float((turn(g, positions, freqs, True)[0] * dy.double()).sum())
    h = 1e-5
    for n in range(3):
        v, vw = normal(q.shape, torch.float32, 10 + n).double(), normal(w.shape, torch.float32, 20 + n).double()
        X, W = q.double(), w.double()
        want = (loss(X + h * v, W) - loss(X - h * v, W)) / (2 * h)
        got = float((dq.double() * v).sum())
        # the difference is off by h^2 / 6 of the third derivative, 64-bit sums by 1e-10; dq by the bound above
        assert abs(got - want) <= 1e-4 * float((dq.double().abs() * v.abs()).sum()), (got, want)
        want = (loss(X, W + h * vw) - loss(X, W - h * vw)) / (2 * h)
        got = float((dw.double() * vw).sum())
        assert abs(got - want) <= 1e-4 * float((dw.double().abs() * vw.abs()).sum()), (got, want)


def test_wanted_gradients_alone():
    """Gradients that are not wanted are left out; the others have the same bits.  (The C interface: None is made.)"""
    L = kb.lib()
    q, k, w = normal((70, 4, 64), torch.float16, 1), normal((70, 2, 64), torch.float16, 2), normal((64,), torch.float32, 3)
    dy = normal(q.shape, torch.float16, 4), normal(k.shape, torch.float16, 5)
    positions, freqs = torch.arange(70, device="cuda", dtype=torch.int32), freqs_of(64)
    want = kb.kb_qk_norm_backward(*dy, q, k, w, w, EPS, positions, freqs)
    opts = kb._qk_opts(q, EPS, positions, freqs, False)
    ws = torch.empty(L.kb_qk_norm_backward_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    views = [kb.pack_view(t) for t in (*dy, q, k, w, w)]
    for mask in range(16):
        outs = [torch.full_like(t, 7.0) for t in want]
        given = [kb.pack_view(t) if mask >> i & 1 else None for i, t in enumerate(outs)]
        sums = mask & 12
        rc = L.kb_qk_norm_backward(*views, opts, *given, ws.data_ptr() if sums else None, ws.numel() if sums else 0,
                                   kb._stream_handle(None))
        assert rc == 0
        for i, (a, c) in enumerate(zip(outs, want)):
            assert torch.equal(a, c) if mask >> i & 1 else torch.all(a == 7.0)


def test_same_bits_on_every_call_and_stream():
    q, k = normal((3000, 8, 128), torch.bfloat16, 1), normal((3000, 2, 128), torch.bfloat16, 2)
    positions, freqs = torch.arange(3000, device="cuda", dtype=torch.int32), freqs_of(128)
    args = (None, None, EPS, positions, freqs)
    first = kb.kb_qk_norm_forward(q, k, *args) + kb.kb_qk_norm_backward(q, k, q, k, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        again = kb.kb_qk_norm_forward(q, k, *args, stream=stream) + kb.kb_qk_norm_backward(q, k, q, k, *args, stream=stream)
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(first, again))


def test_rows_far_apart():
    """Offsets of 2^31 elements and more."""
    step = (1 << 30) + 64
    buf = torch.empty(3 * step + 1000, dtype=torch.float16, device="cuda")
    q = buf.as_strided((4, 2, 64), (step, 128, 1))
    dense = normal((4, 2, 64), torch.float16, 1)
    q.copy_(dense)
    positions, freqs = torch.arange(4, device="cuda", dtype=torch.int32), freqs_of(64)
    want = kb.kb_qk_norm_forward(dense, dense, None, None, EPS, positions, freqs)
    got = kb.kb_qk_norm_forward(q, dense, None, None, EPS, positions, freqs, q_out=q)
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("change", [dict(positions="short"), dict(positions="float"), dict(freqs="half"), dict(q="cpu"),
                                    dict(rot="long"), dict(eps=-1.0), dict(w="size")])
def test_refusals_of_the_binding(change):
    q, k, w = normal((6, 2, 32), torch.float32, 1), normal((6, 1, 32), torch.float32, 2), normal((32,), torch.float32, 3)
    positions, freqs, eps = torch.arange(6, device="cuda", dtype=torch.int32), freqs_of(32), EPS
    if change.get("positions") == "short":
        positions = positions[:5]
    if change.get("positions") == "float":
        positions = positions.float()
    if change.get("freqs"):
        freqs = freqs.half()
    if change.get("q"):
        q = q.cpu()
    if change.get("rot"):
        freqs = freqs_of(34)
    if change.get("w"):
        w = w[:31]
    with pytest.raises((ValueError, kb.KbError)):
        kb.kb_qk_norm_forward(q, k, w, w, change.get("eps", eps), positions, freqs)
