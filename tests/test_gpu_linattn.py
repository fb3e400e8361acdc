"""quamba_linattn_prefill / _step against the recurrence in 64 bits, element by element.

What an element may be off by, relative to the sum of the absolute values it is made of: every fp32 addition and product
one unit of 2^-23 (L tokens into a state, dk terms and at most 64 tokens of a block into an output, 16 for weights and
scale); block weights and the state's copy in front of the matrix unit carry at least 16 bits, two of them in a product
(2^-16), the state's update at least 22 (2^-21); a decay's exponent, the difference of two sums of at most 64 log decays,
is off by two units of the larger.  Then the rounding to the output, half a step."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2410_13229_amd as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KIND = {torch.float16: Q.TYPE_F16, torch.bfloat16: Q.TYPE_BF16}
U = 2.0 ** -23


def _f64(t):
    return t.detach().double().cpu().numpy()


def _tolerances(L, dk, g, dt, out, out_size, S, size):
    finite = 0.0 if g is None else float(np.abs(np.where(np.isfinite(g), np.maximum(np.minimum(g, 0), -88), 0)).max(initial=0.0))
    G = min(L, 64) * finite
    t_state = ((L + 16 + 64) * U + 2.0 ** -21 + 2 * G * U) * size + 1e-37
    t_out = ((L + dk + 64 + 16) * U + 2.0 ** -16 + 2 * G * U) * out_size
    e = torch.finfo(dt)
    return t_out + e.eps / 2 * (np.abs(out) + t_out) + e.smallest_normal * e.eps, t_state


class Call:
    """Inputs of one call: q | k | v as columns of one tensor (`pad` more behind them), decays, state."""

    def __init__(self, B, L, Hk, Hv, dk, dv, dt, decay="token", pad=0, shift=0, state=True, seed=0, gain=1.0):
        g = torch.Generator(device=DEV).manual_seed(seed * 101 + B * 7 + L * 13 + dk * 3 + dv)
        self.B, self.L, self.Hk, self.Hv, self.dk, self.dv, self.dt = B, L, Hk, Hv, dk, dv, dt
        width = 2 * Hk * dk + Hv * dv + pad
        flat = (torch.randn(B * L * width + shift, generator=g, device=DEV) * gain).to(dt)
        self.rows = flat[shift:].view(B, L, width)
        self.g = None
        if decay == "head":
            self.g = -torch.rand(Hv, generator=g, device=DEV) * 0.1
        elif decay != "none":
            self.g = -torch.exp(torch.rand((B, L, Hv), generator=g, device=DEV) * 5 - 6)
            pick = torch.rand((B, L, Hv), generator=g, device=DEV)
            if decay == "strong":  # now and then nearly everything is forgotten
                self.g = torch.where(pick < 0.1, torch.full_like(self.g, -30.0), self.g)
            elif decay == "reset":
                self.g = torch.where(pick < 0.1, torch.full_like(self.g, -float("inf")), self.g)
                self.g = torch.where(pick > 0.95, torch.full_like(self.g, -3.4e38), self.g)
            elif decay == "positive":
                self.g = torch.where(pick < 0.3, -self.g, self.g)
        self.state = torch.randn((B, Hv, dk, dv), generator=g, device=DEV) * 2 if state else None
        self.out = torch.full((B, L, Hv * dv + pad), 7.0, dtype=dt, device=DEV)
        self.scale = dk ** -0.5
        self.lens = None

    def parts(self):
        a, b = self.Hk * self.dk, 2 * self.Hk * self.dk
        r = self.rows
        return r[..., :a], r[..., a:b], r[..., b:b + self.Hv * self.dv]

    def want(self):
        q, k, v = (_f64(t) for t in self.parts())
        s = (self.B, self.L)
        return O.linattn(q.reshape(*s, self.Hk, self.dk), k.reshape(*s, self.Hk, self.dk), v.reshape(*s, self.Hv, self.dv),
                         None if self.g is None else _f64(self.g), None if self.state is None else _f64(self.state),
                         None if self.lens is None else self.lens.tolist(), self.scale)

    def workspace(self):
        return torch.empty(Q.quamba_linattn_workspace_bytes(self.B, self.L, self.Hk, self.Hv, self.dk, self.dv), dtype=torch.uint8, device=DEV)

    def prefill(self, stream=None, ws=None):
        q, k, v = self.parts()
        ld = self.rows.stride(1)
        Q.quamba_linattn_prefill(KIND[self.dt], q, ld, k, ld, v, ld, self.g, 0 if self.g is None or self.g.dim() == 1 else self.Hv, self.lens,
                                 self.B, self.L, self.Hk, self.Hv, self.dk, self.dv, self.scale, self.out, self.out.stride(1), self.state,
                                 self.workspace() if ws is None else ws, stream)

    def step(self, t, state, out, stream=None):
        """Token t of every sequence through the single-token form."""
        q, k, v = (p[:, t] for p in self.parts())
        ld = self.rows.stride(0)
        g = self.g if self.g is None or self.g.dim() == 1 else self.g[:, t]
        Q.quamba_linattn_step(KIND[self.dt], q, ld, k, ld, v, ld, g, 0 if g is None or g.dim() == 1 else g.stride(0), self.B, self.Hk, self.Hv,
                              self.dk, self.dv, self.scale, out, out.stride(0), state, stream)

    def check(self, want):
        out, S, out_size, size = want
        t_out, t_state = _tolerances(self.L, self.dk, None if self.g is None else _f64(self.g), self.dt, out, out_size, S, size)
        w = self.Hv * self.dv
        got = _f64(self.out[..., :w]).reshape(out.shape)
        on = ~np.isnan(out_size)
        assert (got[~on] == 7.0).all(), "rows behind a sequence's end were written"
        assert (self.out[..., w:] == 7.0).all(), "columns beside the output were written"
        off = np.abs(got - out)[on] / t_out[on]
        assert off.max(initial=0.0) <= 1, "output off by %.2f of what it may be" % off.max()
        assert not np.isnan(got[on]).any()
        if self.state is not None:
            off = np.abs(_f64(self.state) - S) / t_state
            assert off.max() <= 1, "state off by %.2f of what it may be" % off.max()


SHAPES = [(1, 1, 1, 1, 1, 1), (2, 2, 1, 2, 16, 16), (1, 63, 1, 2, 16, 16), (1, 64, 2, 2, 64, 64), (2, 65, 1, 2, 64, 64), (3, 130, 1, 3, 96, 80),
          (1, 128, 2, 4, 128, 64), (2, 200, 2, 2, 128, 128), (1, 257, 1, 2, 256, 48), (1, 33, 1, 1, 33, 129), (1, 40, 1, 2, 17, 257),
          (1, 100, 1, 1, 200, 31), (1, 1000, 1, 1, 64, 64), (1, 1500, 1, 2, 128, 40), (5, 17, 3, 3, 8, 24), (1, 70, 1, 1, 128, 1024)]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_prompts(shape, dt):
    for decay in ("token", "none"):
        c = Call(*shape, dt, decay=decay)
        want = c.want()
        c.prefill()
        c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("decay", ["head", "strong", "reset", "positive"])
@pytest.mark.parametrize("shape", [(2, 150, 1, 2, 64, 64), (1, 700, 2, 4, 128, 64), (1, 300, 1, 1, 40, 130)])
def test_decays(shape, decay, dt):
    c = Call(*shape, dt, decay=decay)
    want = c.want()
    c.prefill()
    c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_without_a_state(dt):
    for shape in ((1, 90, 1, 2, 64, 64), (2, 600, 1, 1, 128, 128)):
        c = Call(*shape, dt, state=False)
        want = c.want()
        c.prefill()
        c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("L, lens", [(70, [70, 0, 1, 64, 33]), (600, [0, 600, 65, 129, 512]), (5, [0, 0, 0, 0, 0]), (130, [-3, 1000, 128, 127, 2])])
def test_unequal_lengths(L, lens, dt):
    """What stands behind a sequence's end is NaN and stays out of everything."""
    for shape in ((2, 4, 64, 64), (1, 3, 96, 80), (1, 2, 128, 128)):
        c = Call(5, L, *shape, dt)
        c.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        for b, n in enumerate(lens):
            n = min(max(n, 0), L)
            c.rows[b, n:] = float("nan")
            c.g[b, n:] = float("nan")
        before = c.state.clone()
        want = c.want()
        c.prefill()
        c.check(want)
        for b, n in enumerate(lens):
            assert n > 0 or torch.equal(c.state[b], before[b])


@pytest.mark.parametrize("pad, shift", [(8, 0), (3, 0), (8, 4), (0, 1), (5, 3)])
def test_strides_and_alignments(pad, shift):
    for shape in ((2, 100, 1, 2, 64, 64), (1, 129, 2, 2, 24, 40), (1, 129, 1, 3, 33, 19)):
        c = Call(*shape, torch.bfloat16, pad=pad, shift=shift)
        c.rows[..., c.rows.shape[2] - pad:] = float("nan") if pad else 0
        want = c.want()
        c.prefill()
        c.check(want)


@pytest.mark.parametrize("gain", [1e-3, 30.0, 200.0])
def test_small_and_large_values(gain):
    """fp16 values whose products with each other leave fp16's range (200 * 200), and ones far below it.  Outputs beyond fp16
    are infinite, as in the product's epilogue."""
    for shape in ((1, 150, 1, 2, 64, 64), (1, 90, 1, 1, 128, 100)):
        c = Call(*shape, torch.float16, gain=gain)
        c.scale = 1e-3 if gain > 1 else 1.0
        if gain > 100:
            c.scale = 1e-6
        c.state *= gain * gain
        want = c.want()
        c.prefill()
        c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 5, 1, 1, 1, 1), (2, 6, 12, 12, 64, 64), (64, 2, 1, 8, 128, 64), (3, 4, 2, 10, 96, 80), (2, 3, 1, 1, 256, 129),
                                   (1, 3, 1, 2, 33, 1024), (5, 3, 1, 5, 17, 7)])
def test_single_tokens(shape, dt):
    for decay, pad in (("token", 0), ("head", 3), ("reset", 8), ("none", 1)):
        c = Call(*shape, dt, decay=decay, pad=pad)
        want = c.want()
        for t in range(c.L):
            c.step(t, c.state, c.out[:, t])
        c.check(want)


def test_prefill_then_steps_equals_one_prefill():
    whole = Call(2, 150, 1, 4, 128, 64, torch.bfloat16)
    want = whole.want()
    part = Call(2, 150, 1, 4, 128, 64, torch.bfloat16)
    part.lens = torch.tensor([140, 140], dtype=torch.int32, device=DEV)
    part.prefill()
    for t in range(140, 150):
        part.step(t, part.state, part.out[:, t])
    whole.prefill()
    whole.check(want)
    part.check(want)


@pytest.mark.parametrize("shape", [(1, 2000, 1, 4, 128, 64), (4, 100, 2, 2, 64, 64)])
def test_same_bits_every_time(shape):
    outs = []
    for fill in (0, 255):
        c = Call(*shape, torch.float16)
        ws = c.workspace().fill_(fill)
        c.prefill(ws=ws)
        outs.append((c.out, c.state))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_nan_stays_in_its_sequence_and_head():
    c = Call(2, 100, 2, 2, 64, 64, torch.float16)
    c.rows[0, 50, :64] = float("nan")  # the query of key head 0 at token 50
    c.prefill()
    bad = torch.isnan(c.out.view(2, 100, 2, 64))
    assert bad[0, 50, 0].all() and int(bad.sum()) == 64 and not torch.isnan(c.state).any()


def test_empty_calls_touch_nothing():
    c = Call(1, 4, 1, 1, 16, 16, torch.float16)
    before = c.state.clone()
    Q.quamba_linattn_prefill(Q.TYPE_F16, c.rows, 48, c.rows, 48, c.rows, 48, None, 0, None, 1, 0, 1, 1, 16, 16, 1.0, c.out, 16, c.state, None)
    Q.quamba_linattn_step(Q.TYPE_F16, c.rows, 48, c.rows, 48, c.rows, 48, None, 0, 0, 1, 1, 16, 16, 1.0, c.out, 16, c.state)
    assert torch.equal(c.state, before) and (c.out == 7.0).all()


@pytest.fixture
def segments():
    yield Q.quamba_debug_set_linattn_blocks
    Q.quamba_debug_set_linattn_blocks(0)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("blocks", [1, 2, 3, 100])
def test_any_number_of_segments(blocks, dt, segments):
    segments(blocks)
    for shape in ((2, 150, 1, 2, 64, 64), (1, 700, 2, 4, 128, 64), (3, 300, 1, 1, 40, 130), (1, 260, 1, 1, 200, 72), (2, 190, 1, 1, 33, 19)):
        for decay in ("token", "strong", "reset"):
            c = Call(*shape, dt, decay=decay, state=decay != "strong")
            want = c.want()
            c.prefill()
            c.check(want)
    c = Call(6, 200, 1, 3, 96, 80, dt)
    c.lens = torch.tensor([200, 0, 1, 64, 65, 129], dtype=torch.int32, device=DEV)
    for b, n in enumerate(c.lens.tolist()):
        c.rows[b, n:] = float("nan")
        c.g[b, n:] = float("nan")
    want = c.want()
    c.prefill()
    c.check(want)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape, token", [((2, 150, 1, 2, 64, 64), 40), ((1, 300, 1, 2, 128, 64), 64), ((1, 130, 2, 2, 128, 128), 63),
                                          ((1, 200, 1, 1, 256, 80), 100), ((1, 100, 1, 2, 33, 19), 0), ((1, 90, 1, 1, 24, 130), 89)])
def test_a_bad_token_stays_out_of_earlier_outputs(shape, token, dt):
    """NaN or an infinity in v reaches its own column from its token on, in k or the decay its own head from its token on."""
    clean = Call(*shape, dt)
    clean.prefill()
    B, L, Hk, Hv, dk, dv = shape
    view = lambda c: (c.out.view(B, L, Hv, dv), c.state)
    want, want_state = view(clean)
    for value in (float("nan"), float("inf"), -float("inf")):
        c = Call(*shape, dt)
        c.rows[0, token, 2 * Hk * dk + dv // 2] = value
        c.prefill()
        got, state = view(c)
        hit = torch.zeros((B, L, Hv, dv), dtype=torch.bool, device=DEV)
        hit[0, token:, 0, dv // 2] = True
        assert torch.equal(got[~hit], want[~hit]) and not torch.isfinite(got[hit]).any()
        hit = torch.zeros_like(state, dtype=torch.bool)
        hit[0, 0, :, dv // 2] = True
        assert torch.equal(state[~hit], want_state[~hit]) and not torch.isfinite(state[hit]).any()
    for where in ("k", "decay"):
        c = Call(*shape, dt)
        if where == "k":
            c.rows[0, token, Hk * dk] = float("nan")
        else:
            c.g[0, token, 0] = float("nan")
        c.prefill()
        got, state = view(c)
        heads = Hv // Hk if where == "k" else 1
        hit = torch.zeros((B, L, Hv, dv), dtype=torch.bool, device=DEV)
        hit[0, token:, :heads] = True
        assert torch.equal(got[~hit], want[~hit]) and torch.isnan(got[hit]).all()


@pytest.mark.parametrize("L, ld", [(2100, 1 << 20), (260, (1 << 23) + 8)])
def test_offsets_past_32_bits(L, ld):
    """The last tokens start more than 2^31 elements in; in the second case a block of tokens spans more than 2^31 bytes."""
    c = Call(1, L, 1, 1, 64, 64, torch.bfloat16, pad=ld - 192)
    want = c.want()
    c.prefill()
    c.check(want)
