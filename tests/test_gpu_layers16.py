"""The 16-bit layers together, as a block of a hybrid stack runs them: projection to q | k | v with bias and activation,
fp32 projection of the decays, linear attention over prompts of unequal length, output projection onto the residual
stream; then generation from the carried states.  Against the same block in 64 bits whose 16-bit tensors are rounded
where the library's are."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2410_13229_amd as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KIND = {torch.float16: Q.TYPE_F16, torch.bfloat16: Q.TYPE_BF16}


class Block:
    def __init__(self, dm, Hk, Hv, dk, dv, dt, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.dm, self.Hk, self.Hv, self.dk, self.dv, self.dt = dm, Hk, Hv, dk, dv, dt
        self.wide = 2 * Hk * dk + Hv * dv

        def normal(*s, std):
            return torch.randn(s, generator=g, device=DEV) * std

        self.W, self.b = normal(self.wide, dm, std=dm ** -0.5).to(dt), normal(self.wide, std=0.1)
        self.Wg, self.bg = normal(Hv, dm, std=dm ** -0.5).to(dt), normal(Hv, std=1.0)
        self.Wo = normal(dm, Hv * dv, std=(Hv * dv) ** -0.5).to(dt)

    def buffers(self, B, L):
        M = B * L
        e = lambda w, dt=self.dt: torch.zeros((M, w), dtype=dt, device=DEV)  # noqa: E731
        n = [Q.quamba_linear_workspace_bytes(M, w, k) for w, k in ((self.wide, self.dm), (self.Hv, self.dm), (self.dm, self.Hv * self.dv))]
        n.append(Q.quamba_linattn_workspace_bytes(B, L, self.Hk, self.Hv, self.dk, self.dv))
        return dict(qkv=e(self.wide), gate=e(self.Hv, torch.float32), g=e(self.Hv, torch.float32), o=e(self.Hv * self.dv), ws=torch.empty(max(n), dtype=torch.uint8, device=DEV))

    def run(self, x, B, L, state, lens, buf, stream=None):
        """x [B * L, dm] is updated in place (the residual stream); L = 1 without `lens` is a generation step."""
        M, t, esz = B * L, KIND[self.dt], 2
        Q.quamba_linear(t, x, self.dm, self.W, self.dm, self.b, None, 0, M, self.wide, self.dm, Q.ACT_SILU, t, buf["qkv"], self.wide, buf["ws"], stream)
        Q.quamba_linear(t, x, self.dm, self.Wg, self.dm, self.bg, None, 0, M, self.Hv, self.dm, Q.ACT_SIGMOID, Q.TYPE_F32, buf["gate"], self.Hv, buf["ws"], stream)
        torch.log(buf["gate"], out=buf["g"])
        at = buf["qkv"].data_ptr()
        k, v = at + self.Hk * self.dk * esz, at + 2 * self.Hk * self.dk * esz
        scale = self.dk ** -0.5
        if L == 1 and lens is None:
            Q.quamba_linattn_step(t, at, self.wide, k, self.wide, v, self.wide, buf["g"], self.Hv, B, self.Hk, self.Hv, self.dk, self.dv, scale, buf["o"],
                                  self.Hv * self.dv, state, stream)
        else:
            Q.quamba_linattn_prefill(t, at, self.wide, k, self.wide, v, self.wide, buf["g"], self.Hv, lens, B, L, self.Hk, self.Hv, self.dk, self.dv, scale,
                                     buf["o"], self.Hv * self.dv, state, buf["ws"], stream)
        Q.quamba_linear(t, buf["o"], self.Hv * self.dv, self.Wo, self.Hv * self.dv, None, x, self.dm, M, self.dm, self.Hv * self.dv, Q.ACT_NONE, t, x, self.dm,
                        buf["ws"], stream)

    def want(self, x, B, L, state, lens):
        """64 bits, 16-bit tensors rounded as stored: (x, state); rows behind an end keep whatever `o` was (zero)."""
        f = lambda t: t.double().cpu().numpy()  # noqa: E731

        def rounded(a):
            return torch.from_numpy(a).to(self.dt).double().numpy()

        M = B * L
        qkv = rounded(O.linear(f(x), f(self.W), f(self.b), act="silu")[0])
        g = np.log(O.linear(f(x), f(self.Wg), f(self.bg), act="sigmoid")[0]).reshape(B, L, self.Hv)
        a, b = self.Hk * self.dk, 2 * self.Hk * self.dk
        o, S, _, _ = O.linattn(qkv[:, :a].reshape(B, L, self.Hk, self.dk), qkv[:, a:b].reshape(B, L, self.Hk, self.dk), qkv[:, b:].reshape(B, L, self.Hv, self.dv), g,
                               f(state), lens, self.dk ** -0.5)
        o = rounded(np.nan_to_num(o.reshape(M, -1)))
        return O.linear(o, f(self.Wo), residual=f(x))[0], S


def _close(got, want, dt):
    """One more rounding may fall the other way at each of three 16-bit tensors: 4 half steps of the tensor's largest value."""
    got = got.double().cpu().numpy()
    assert np.abs(got - want).max() <= 4 * torch.finfo(dt).eps / 2 * np.abs(want).max()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_block_prompts_then_generation(dt):
    B, L, blk = 3, 90, Block(192, 1, 4, 64, 48, dt)
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((B * L, 192), generator=g, device=DEV).to(dt)
    state = torch.zeros((B, 4, 64, 48), device=DEV)
    lens = torch.tensor([90, 31, 0], dtype=torch.int32, device=DEV)
    want_x, want_S = blk.want(x, B, L, state, lens.tolist())
    blk.run(x, B, L, state, lens, blk.buffers(B, L))
    _close(x, want_x, dt)
    _close(state, want_S, dt)
    buf = blk.buffers(B, 1)
    for t in range(3):
        y = torch.randn((B, 192), generator=g, device=DEV).to(dt)
        want_y, want_S = blk.want(y, B, 1, state, None)
        blk.run(y, B, 1, state, None, buf)
        _close(y, want_y, dt)
        _close(state, want_S, dt)


@pytest.mark.parametrize("B, L", [(1, 700), (3, 1)])
def test_captured_and_replayed(B, L):
    """The whole block captured into a graph, replayed with other work and synchronizations between, equals the eager run bit for bit."""
    dt, blk = torch.bfloat16, Block(256, 2, 4, 64, 64, torch.bfloat16)
    buf = blk.buffers(B, L)
    x = torch.zeros((B * L, 256), dtype=dt, device=DEV)
    state = torch.zeros((B, 4, 64, 64), device=DEV)
    lens = torch.tensor([L], dtype=torch.int32, device=DEV) if L > 1 else None
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        blk.run(x, B, L, state, lens, buf, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        blk.run(x, B, L, state, lens, buf, torch.cuda.current_stream())
    for i in range(4):
        start = torch.randn((B * L, 256), device=DEV).to(dt)
        eager, S = start.clone(), torch.full_like(state, 0.25 * i)
        blk.run(eager, B, L, S, lens, blk.buffers(B, L), torch.cuda.current_stream())
        x.copy_(start)
        state.fill_(0.25 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, eager) and torch.equal(state, S), i


def test_two_streams_at_once():
    """Two blocks on two streams with their own buffers give what each gives alone."""
    dt = torch.float16
    blocks = [Block(256, 1, 4, 128, 64, dt, seed=i) for i in range(2)]
    xs = [torch.randn((2 * 400, 256), device=DEV).to(dt) for _ in range(2)]
    alone = []
    for blk, x in zip(blocks, xs):
        y, S = x.clone(), torch.zeros((2, 4, 128, 64), device=DEV)
        blk.run(y, 2, 400, S, None, blk.buffers(2, 400), torch.cuda.current_stream())
        alone.append((y, S))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [(blk, x.clone(), torch.zeros((2, 4, 128, 64), device=DEV), blk.buffers(2, 400)) for blk, x in zip(blocks, xs)]
    torch.cuda.synchronize()
    for _ in range(3):  # the last of several rounds
        for s, (blk, y, S, buf), x in zip(streams, work, xs):
            with torch.cuda.stream(s):
                y.copy_(x)
                S.zero_()
                blk.run(y, 2, 400, S, None, buf, s)
    torch.cuda.synchronize()
    for (y, S), (_, y2, S2, _) in zip(alone, work):
        assert torch.equal(y, y2) and torch.equal(S, S2)
