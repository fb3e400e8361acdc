"""The 16-bit layers near the limits of their sizes and values."""
import math

import numpy as np
import pytest
import torch

import paper_2410_13229_amd as Q
from test_gpu_linattn import Call, U, _f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_linear_rows_of_more_than_two_million_elements_with_a_workspace():
    """32 rows of 35 million elements: the last starts past 2^31 bytes.  A few columns hold small whole numbers, so the result is exact."""
    M, N, K = 32, 32, 35000008
    at = torch.tensor([0, 5, 63, 64, 1 << 21, 17000001, (1 << 25) + 3, K - 9, K - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    x, W = (torch.zeros((32, K), dtype=torch.float16, device=DEV) for _ in range(2))
    a, b = (torch.randint(-8, 9, (32, len(at)), generator=g, device=DEV) for _ in range(2))
    x[:, at], W[:, at] = a.half(), b.half()
    ws = torch.empty(2 * 2 * 32 * (K + 64), dtype=torch.uint8, device=DEV)
    for room in (ws, None):
        out = torch.full((M, N), float("nan"), device=DEV)
        Q.quamba_linear(Q.TYPE_F16, x, K, W, K, None, None, 0, M, N, K, Q.ACT_NONE, Q.TYPE_F32, out, N, room)
        assert np.array_equal(out.cpu().numpy(), a.cpu().numpy().astype(np.float32) @ b.cpu().numpy().astype(np.float32).T)


def _closely(c, want):
    """Call.check's bounds without a term for the decays: a weight's exponent is an exact difference and a factor, off by the units of
    its exponentials and products, which the 16 units of 2^-23 hold."""
    out, S, out_size, size = want
    e = torch.finfo(c.dt)
    t_out = ((c.L + c.dk + 64 + 16) * U + 2.0 ** -16) * out_size
    t_out = t_out + e.eps / 2 * (np.abs(out) + t_out) + e.smallest_normal * e.eps
    got = _f64(c.out[..., :c.Hv * c.dv]).reshape(out.shape)
    off = np.abs(got - out) / t_out
    assert off.max() <= 1, "output off by %.2f of what it may be" % off.max()
    off = np.abs(_f64(c.state) - S) / (((c.L + 16 + 64) * U + 2.0 ** -21) * size + 1e-37)
    assert off.max() <= 1, "state off by %.2f of what it may be" % off.max()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 64, 1, 64, 8, 16), (1, 64, 1, 64, 7, 5), (2, 64, 1, 16, 128, 128), (2, 64, 1, 8, 256, 64)])
def test_linattn_weights_behind_steep_decays(shape, dt):
    """One block: 13 tokens that forget nearly everything, then 3 that forget little, whose contributions cancel.  What the sums of the
    log decays have reached by then (about 1600 in a group of 16 tokens) must not show in the weights between the 3.  q, k and v are
    whole numbers that every piece holds, so a weight is off by its two bf16 pieces (each leaves 2^-9 of what it takes: 2^-18), and
    dk + 64 + 16 fp32 operations, then the rounding to the output."""
    B, L, _, Hv, dk, dv = shape
    g = torch.Generator(device=DEV).manual_seed(L)
    for first in (13, 15):  # the 3 at the end of a group of 16 tokens, or across its border
        c = Call(*shape, dt, decay="none", state=False)
        q, k, v = c.parts()
        q.fill_(1.0), k.fill_(1.0)
        v.copy_((torch.arange(L, device=DEV) % 2 * 2.0 - 1.0)[None, :, None].expand_as(v))
        steep = -80 - 7 * torch.rand((B, L, Hv), generator=g, device=DEV)
        weak = -0.02 * torch.rand((B, L, Hv), generator=g, device=DEV)
        c.g = torch.where(((torch.arange(L, device=DEV) - first) % 16 < 3)[None, :, None], weak, steep)
        out, _, size, _ = c.want()
        c.prefill()
        tol = ((dk + 64 + 16) * U / 2 + 2.0 ** -18) * size
        e = torch.finfo(dt)
        tol = tol + e.eps / 2 * (np.abs(out) + tol) + e.smallest_normal * e.eps
        off = np.abs(_f64(c.out[..., :Hv * dv]).reshape(out.shape) - out) / tol
        assert off.max() <= 1, "output off by %.2f of what it may be" % off.max()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("decay", ["token", "strong", "reset"])
@pytest.mark.parametrize("shape", [(2, 150, 1, 2, 64, 64), (1, 700, 2, 4, 128, 64), (1, 300, 1, 1, 40, 130)])
def test_linattn_decays_closely(shape, decay, dt):
    c = Call(*shape, dt, decay=decay)
    want = c.want()
    c.prefill()
    _closely(c, want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape, token, reset", [((1, 64, 1, 2, 64, 64), 20, 24), ((1, 200, 2, 2, 33, 19), 70, 100), ((2, 130, 1, 2, 128, 128), 3, 63),
                                                 ((1, 130, 1, 1, 256, 40), 60, 70)])
def test_linattn_a_reset_does_not_clear_a_bad_token(shape, token, reset, dt):
    """NaN in k or in the decay reaches its head from its token on, also behind a reset in the same block; one in v its column."""
    B, L, Hk, Hv, dk, dv = shape
    for where in ("k", "decay", "v"):
        c = Call(*shape, dt)
        c.g[:, reset] = -float("inf")
        q, k, v = c.parts()
        if where == "k":
            k[0, token, 0] = float("nan")
        elif where == "decay":
            c.g[0, token, 0] = float("nan")
        else:
            v[0, token, dv // 2] = float("inf")
        c.prefill()
        out = c.out.view(B, L, Hv, dv)
        hit = torch.zeros((B, L, Hv, dv), dtype=torch.bool, device=DEV)
        if where == "v":
            hit[0, token:, 0, dv // 2] = True
        else:
            hit[0, token:, :Hv // Hk if where == "k" else 1] = True
        bad = ~torch.isfinite(out)
        assert int((bad != hit).sum()) == 0, where


@pytest.mark.parametrize("form", ["prefill", "step"])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_linattn_forgets_where_the_decay_leaves_the_normal_range(dt, form):
    """exp(g) >= 2^-126 decays, below that nothing of the past remains; both forms draw the line at the same g."""
    B, Hk, Hv, dk, dv = 1, 1, 6, 64, 64
    c = Call(B, 1, Hk, Hv, dk, dv, dt)
    q, k, v = c.parts()
    q.fill_(1.0), k.zero_(), v.zero_()
    c.g = torch.tensor([-86.9, -87.2, -87.33654, -87.33656, -87.5, -100.0], device=DEV).view(1, 1, Hv)
    c.state = torch.full((B, Hv, dk, dv), 2.0 ** 100, device=DEV)
    a = np.exp(_f64(c.g).ravel())
    a[3:] = 0.0
    if form == "prefill":
        c.prefill()
    else:
        c.step(0, c.state, c.out[:, 0])
    want = a[:, None, None] * 2.0 ** 100 * np.ones((dk, dv))
    got = _f64(c.state)[0]
    assert (got[3:] == 0).all() and (_f64(c.out).reshape(Hv, dv)[3:] == 0).all()
    # the exponent, 126 in the worst case, is rounded to fp32 once or twice: 2 * 126 / 2^24, times ln 2
    assert (np.abs(got - want) <= 2 * 126 * 2.0 ** -24 * want).all()
    if dt == torch.bfloat16:  # 64 of them, scaled: about 1e-7, far below fp16
        out = c.scale * dk * want[:, 0]
        assert (np.abs(_f64(c.out).reshape(Hv, dv) - out) <= (2.0 ** -8 + 2.0 ** -15) * out).all()


@pytest.mark.parametrize("act, lowest", [("silu", -104.0), ("gelu", -14.5), ("gelu_tanh", -11.0), ("sigmoid", -88.0)])
@pytest.mark.parametrize("M", [1, 70])
def test_linear_tails_of_the_activations(act, lowest, M):
    """Far negative arguments, whose results are small but normal numbers of fp32 and bf16.  What a result may be off by relative to itself: 16
    units of 2^-23 for the operations, the exponent's rounding (|v|, of GELU v^2, of its tanh form four roundings of 2 u), half a step of the
    output; numbers below the smallest normal one may be 0."""
    N = 4096
    v = torch.linspace(lowest, 8.0, N, device=DEV)
    x, W = torch.zeros((M, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((N, 64), dtype=torch.bfloat16, device=DEV)
    b = v.double().cpu().numpy()
    u2 = 2 * math.sqrt(2 / math.pi) * (b + 0.044715 * b ** 3)
    want = {"silu": lambda: b / (1 + np.exp(-b)), "gelu": lambda: np.array([0.5 * t * math.erfc(-t / math.sqrt(2)) for t in b]),
            "gelu_tanh": lambda: b / (1 + np.exp(-u2)), "sigmoid": lambda: 1 / (1 + np.exp(-b))}[act]()
    exponent = {"silu": np.abs(b), "gelu": b * b, "gelu_tanh": 4 * np.abs(u2), "sigmoid": np.abs(b)}[act]
    for out_type, dt in ((Q.TYPE_F32, torch.float32), (Q.TYPE_BF16, torch.bfloat16)):
        out = torch.full((M, N), float("nan"), dtype=dt, device=DEV)
        Q.quamba_linear(Q.TYPE_BF16, x, 64, W, 64, v, None, 0, M, N, 64, getattr(Q, "ACT_" + act.upper()), out_type, out, N, None)
        off = np.abs(_f64(out) - want)
        tol = (16 + exponent) * U * np.abs(want) + torch.finfo(dt).eps / 2 * np.abs(want) + 2.0 ** -126
        worst = float((off / tol).max())
        assert worst <= 1, "%.2f of what it may be, at %g" % (worst, b[int((off / tol).max(0).argmax())])


@pytest.mark.parametrize("shape", [(1, 700, 1, 2, 128, 64), (3, 333, 1, 1, 33, 19)])
def test_linattn_with_any_workspace(shape):
    """What the query of another shape gave, or nothing: right all the same."""
    need = Q.quamba_linattn_workspace_bytes(*shape)
    assert need > 256
    for room in (None, 256, need // 2, need, 2 * need):
        c = Call(*shape, torch.bfloat16)
        want = c.want()
        q, k, v = c.parts()
        ws = None if room is None else torch.full((room,), 255, dtype=torch.uint8, device=DEV)
        ld = c.rows.stride(1)
        Q.quamba_linattn_prefill(Q.TYPE_BF16, q, ld, k, ld, v, ld, c.g, c.Hv, None, *shape, c.scale, c.out, c.out.stride(1), c.state, ws)
        c.check(want)


def test_linear_copies_of_more_than_four_gigabytes():
    """4200 rows of 524225 elements, none of which starts on 16 bytes: more workgroups of the copy than one dimension of its launch has."""
    M, N, K = 4200, 40, (1 << 19) - 63
    at = torch.tensor([0, 7, 8, 1000, 300001, K - 2, K - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    x, W = (torch.zeros((rows, K), dtype=torch.bfloat16, device=DEV) for rows in (M, N))
    a, b = (torch.randint(-8, 9, (rows, len(at)), generator=g, device=DEV) for rows in (M, N))
    x[:, at], W[:, at] = a.bfloat16(), b.bfloat16()
    ws = torch.full((Q.quamba_linear_workspace_bytes(M, N, K),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((M, N), float("nan"), device=DEV)
    Q.quamba_linear(Q.TYPE_BF16, x, K, W, K, None, None, 0, M, N, K, Q.ACT_NONE, Q.TYPE_F32, out, N, ws)
    assert np.array_equal(out.cpu().numpy(), a.cpu().numpy().astype(np.float32) @ b.cpu().numpy().astype(np.float32).T)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("power", [-80, 100, 112, 116, 120])
@pytest.mark.parametrize("shape", [(1, 130, 1, 2, 64, 64), (1, 70, 1, 1, 128, 100), (2, 66, 1, 2, 33, 19)])
def test_linattn_states_of_any_size(shape, power, dt):
    """The state is fp32, and 2^122 is one of its values also beside fp16 operands."""
    c = Call(*shape, dt)
    c.state *= 2.0 ** power
    c.scale = 2.0 ** -power
    q, k, v = c.parts()
    if power < 0:
        k.zero_()  # their products would be all there is
    want = c.want()
    c.prefill()
    c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("what", ["state", "v"])
def test_linattn_columns_of_a_wide_range(what, dt):
    """Elements of a column that differ by 2^40 and keys that take them apart.  fp16 pieces are relative to the column's largest
    element: 22 bits of those near it, and of what is smaller all that is above 2^-37 of it; bf16 pieces keep theirs anywhere."""
    B, L, dk, dv = 1, 64, 64, 64
    c = Call(B, L, 1, 1, dk, dv, dt, decay="none")
    q, k, v = c.parts()
    eye = torch.eye(64, device=DEV)
    small = torch.exp2(-torch.arange(64, device=DEV).remainder(41).float())
    q.copy_(eye[None].expand_as(q))  # token t asks for row t
    if what == "state":
        k.zero_(), v.zero_()
        c.state = (1 + torch.rand((B, 1, dk, dv), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))) * small[None, None, :, None] * 2.0 ** 20
        most = 2.0 ** 21
    else:
        k.copy_(eye[None].expand_as(k))  # token t writes row t
        v.copy_((v.float() * (small * 2.0 ** 12 + 2.0 ** -14)[None, :, None]).to(dt))
        c.state.zero_()
        most = float(v.abs().max())
    c.scale = 2.0 ** -6  # outputs within fp16
    out, S, out_size, size = c.want()
    c.prefill()
    lost = 2.0 ** -37 * most if dt == torch.float16 else 0.0
    e = torch.finfo(dt)
    t_out = ((64 + dk + 16) * U + 2.0 ** -16) * out_size + c.scale * lost
    t_out = t_out + e.eps / 2 * (np.abs(out) + t_out) + e.smallest_normal * e.eps
    off = np.abs(_f64(c.out).reshape(out.shape) - out) / t_out
    assert off.max() <= 1, "output off by %.2f of what it may be" % off.max()
    off = np.abs(_f64(c.state) - S) / ((16 * U + 2.0 ** -21) * size + lost + 1e-37)
    assert off.max() <= 1, "state off by %.2f of what it may be" % off.max()
