"""Refusals of the 16-bit layers: checked on the host before anything is launched, so no GPU is needed (the addresses
are never touched)."""
import ctypes

import pytest

import paper_2410_13229_amd as Q

P = 1 << 20  # a made-up, aligned address
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3

LINEAR = dict(type=Q.TYPE_F16, x=P, ldx=64, W=P, ldw=64, bias=None, residual=None, ldr=0, M=4, N=32, K=64, act=Q.ACT_NONE,
              out_type=Q.TYPE_F16, out=P, ldo=32, ws=None)
PREFILL = dict(type=Q.TYPE_BF16, q=P, ldq=128, k=P, ldk=128, v=P, ldv=96, log_decay=P, ldg=6, lens=None, Bt=2, L=9, Hk=2, Hv=6, dk=64,
               dv=16, scale=1.0, out=P, ldo=96, state=P, ws=None)
STEP = {k: v for k, v in PREFILL.items() if k not in ("lens", "L", "ws")}


def _refused(call, args, code, word):
    with pytest.raises(Q.QuambaError) as e:
        call(*args.values())
    assert e.value.code == code and word in str(e.value), str(e.value)


@pytest.mark.parametrize("change, code, word", [
    (dict(type=3), UNSUPPORTED, "operand type"), (dict(type=0), UNSUPPORTED, "operand type"),
    (dict(out_type=Q.TYPE_BF16), UNSUPPORTED, "output type"), (dict(act=6), UNSUPPORTED, "activation"),
    (dict(act=-1), UNSUPPORTED, "activation"), (dict(M=-1), INVALID, "M=-1"), (dict(N=0), INVALID, "N=0"), (dict(K=0), INVALID, "K=0"),
    (dict(ldx=63), INVALID, "ldx=63"), (dict(ldw=63), INVALID, "ldw=63"), (dict(ldo=31), INVALID, "ldo=31"),
    (dict(residual=P, ldr=31), INVALID, "ldr=31"), (dict(x=None), INVALID, "NULL"), (dict(W=None), INVALID, "NULL"),
    (dict(out=None), INVALID, "NULL"), (dict(x=P + 1), INVALID, "aligned"), (dict(W=P + 1), INVALID, "aligned"),
    (dict(out=P + 1), INVALID, "aligned"), (dict(out=P + 2, out_type=Q.TYPE_F32), INVALID, "aligned"),
    (dict(bias=P + 2), INVALID, "aligned"), (dict(residual=P + 1, ldr=32), INVALID, "aligned"),
    (dict(residual=P, ldr=40), INVALID, "in place"),
    (dict(M=2 ** 31 - 1, N=2 ** 31 - 1, ldo=2 ** 31 - 1), UNSUPPORTED, "more than one launch"),
])
def test_linear_refuses(change, code, word):
    _refused(Q.quamba_linear, {**LINEAR, **change}, code, word)


def test_linear_refuses_a_misaligned_workspace():
    rc = Q.lib().quamba_linear(Q.TYPE_F16, P, 64, P, 64, None, None, 0, 4, 32, 64, 0, Q.TYPE_F16, P, 32, ctypes.c_void_p(P + 8), 1024, None)
    assert rc == INVALID and "workspace" in Q.quamba_last_error()


ATTENTION = [
    (dict(type=Q.TYPE_F32), UNSUPPORTED, "operand type"), (dict(Bt=-1), INVALID, "Bt=-1"), (dict(Hk=0), INVALID, "Hk=0"),
    (dict(Hv=0), INVALID, "Hv=0"), (dict(dk=0), INVALID, "dk=0"), (dict(dv=0), INVALID, "dv=0"), (dict(Hk=4), UNSUPPORTED, "multiple"),
    (dict(Hk=1, dk=257, ldq=257, ldk=257), UNSUPPORTED, "dk=257"), (dict(Hv=2, dv=1025, ldv=2050, ldo=2050), UNSUPPORTED, "dv=1025"),
    (dict(Bt=65536), UNSUPPORTED, "Bt=65536"), (dict(ldq=127), INVALID, "ldq=127"), (dict(ldk=127), INVALID, "ldk=127"),
    (dict(ldv=95), INVALID, "ldv=95"), (dict(ldo=95), INVALID, "ldo=95"), (dict(ldg=5), INVALID, "ldg=5"), (dict(ldg=-1), INVALID, "ldg=-1"),
    (dict(q=None), INVALID, "NULL"), (dict(k=None), INVALID, "NULL"), (dict(v=None), INVALID, "NULL"), (dict(out=None), INVALID, "NULL"),
    (dict(q=P + 1), INVALID, "aligned"), (dict(k=P + 1), INVALID, "aligned"), (dict(v=P + 1), INVALID, "aligned"),
    (dict(out=P + 1), INVALID, "aligned"), (dict(log_decay=P + 2), INVALID, "aligned"), (dict(state=P + 4), INVALID, "state"),
]


@pytest.mark.parametrize("change, code, word", ATTENTION + [(dict(L=-1), INVALID, "L=-1"), (dict(lens=P + 2), INVALID, "aligned")])
def test_linattn_prefill_refuses(change, code, word):
    _refused(Q.quamba_linattn_prefill, {**PREFILL, **change}, code, word)


@pytest.mark.parametrize("change, code, word", ATTENTION + [(dict(state=None), INVALID, "state is required")])
def test_linattn_step_refuses(change, code, word):
    _refused(Q.quamba_linattn_step, {**STEP, **change}, code, word)


def test_nothing_to_do_is_no_error():
    """No rows: returns before pointers or the device are looked at."""
    Q.quamba_linear(*{**LINEAR, "M": 0, "x": None, "W": None, "out": None}.values())
    Q.quamba_linattn_prefill(*{**PREFILL, "Bt": 0, "q": None}.values())
    Q.quamba_linattn_prefill(*{**PREFILL, "L": 0, "k": None}.values())
    Q.quamba_linattn_step(*{**STEP, "Bt": 0, "v": None}.values())


def test_workspace_queries():
    assert Q.quamba_linear_workspace_bytes(64, 2560, 5120) > 0 and Q.quamba_linear_workspace_bytes(0, 1, 1) > 0
    assert Q.quamba_linattn_workspace_bytes(1, 2048, 1, 80, 128, 64) > 0 and Q.quamba_linattn_workspace_bytes(0, 0, 1, 1, 1, 1) > 0
    assert Q.quamba_linear_workspace_bytes(1, 0, 1) == 0 and "N=0" in Q.quamba_last_error()
    assert Q.quamba_linattn_workspace_bytes(1, 1, 1, 1, 0, 1) == 0 and "dk=0" in Q.quamba_last_error()


def test_linattn_prefill_refuses_prompts_past_its_counters_and_a_short_workspace():
    _refused(Q.quamba_linattn_prefill, {**PREFILL, "L": 2 ** 30 + 1}, UNSUPPORTED, "at most 2^30")
    Q.quamba_debug_set_linattn_blocks(1)  # two segments: their sums need room
    try:
        assert Q.quamba_linattn_workspace_bytes(1, 100, 1, 1, 16, 16) >= 2 * 16 * 16 * 4
        _refused(Q.quamba_linattn_prefill, {**PREFILL, "Bt": 1, "L": 100, "ws": None}, WORKSPACE, "workspace of 0 bytes")
    finally:
        Q.quamba_debug_set_linattn_blocks(0)


def test_linattn_prefill_refuses_more_heads_than_a_launch_takes():
    n = 65535
    _refused(Q.quamba_linattn_prefill, {**PREFILL, "Bt": n, "L": 1, "Hk": n, "Hv": n, "dk": 1, "dv": 1, "ldq": n, "ldk": n, "ldv": n, "ldg": n, "ldo": n},
             UNSUPPORTED, "more than one launch")


@pytest.mark.parametrize("change", [dict(M=2 ** 30 + 1), dict(N=2 ** 30 + 1, ldo=2 ** 31 - 1), dict(K=2 ** 30 + 1, ldx=2 ** 31 - 1, ldw=2 ** 31 - 1)])
def test_linear_refuses_sizes_past_its_counters(change):
    _refused(Q.quamba_linear, {**LINEAR, **change}, UNSUPPORTED, "at most 2^30")
