"""The operators around the attention (norm, dropout, rotary positions), checked without a GPU: the oracle's
definitions against closed forms, known answers and differences, the rotary plan against exact arithmetic, and
the refusals of the C entry points and of the binding."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2510_18692_b200 import build as moga_build
from paper_2510_18692_b200.inputs import MogaConfig


@pytest.fixture(scope="module")
def mb():
    moga_build.build()
    from paper_2510_18692_b200 import binding
    return binding


def _cfg(**kw):
    base = dict(name="t", B=2, H=2, N=10, C=64, D=64, M=4, k=1, dtype="f32", gate_mode=0, seed=0)
    base.update(kw)
    return MogaConfig(**base)


# ---------------------------------------------------------------- the oracle itself
def test_philox_known_answers():
    """The published answers of Philox4x32-10 for all-zero and all-one counter and key."""
    assert ob.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert ob.philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_dropout_rate_and_expectation():
    n, p = 1 << 15, 0.3
    keep = ob.dropout_keep(n, p, 12345, 7)
    words = np.array([ob.philox((g, 0, 7, 0), (12345, 0)) for g in range(n // 8)])
    bits = np.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)
    assert np.array_equal(keep, bits >= round(p * 65536))
    # binomial: five standard deviations
    assert abs(keep.mean() - (1 - p)) < 5 * math.sqrt(p * (1 - p) / n)
    assert ob.dropout_scale(p) * (65536 - ob.dropout_threshold(p)) == 65536
    other = ob.dropout_keep(n, p, 12345, 8)
    assert abs((keep & other).mean() - (1 - p) ** 2) < 5 / math.sqrt(n)
    assert ob.dropout_keep(64, 0.0, 1, 2).all()


@pytest.mark.parametrize("per_batch", [False, True])
def test_layernorm_gradient_against_differences(per_batch):
    rng = np.random.default_rng(0)
    B, N, C, eps = 2, 3, 6, 1e-5
    X, dY = rng.standard_normal((B, N, C)), rng.standard_normal((B, N, C))
    shape = (B, C) if per_batch else (C,)
    W, b = 1 + 0.2 * rng.standard_normal(shape), rng.standard_normal(shape)
    _, mean, rstd = ob.layernorm(X, W, b, eps)
    got = ob.layernorm_backward(X, W, mean, rstd, dY, per_batch)

    def loss(X, W, b):
        return float((ob.layernorm(X, W, b, eps)[0] * dY).sum())

    h = 1e-6
    for which, grad in zip(range(3), got):
        args = [X, W, b]
        for at in np.ndindex(args[which].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[which][at] += h
            down[which][at] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[at]) < 1e-7


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rope_is_relative_and_orthogonal(layout):
    """Scores depend on the distance of positions only, and the transpose undoes the rotation."""
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((1, 1, 1, 64)), rng.standard_normal((1, 1, 1, 64))
    kw = dict(axis_dims=[24, 16], layout=layout)
    score = [float((ob.rope(q, [[p + 5, 40 + p]], **kw) * ob.rope(k, [[p, p + 3]], **kw)).sum()) for p in (0, 17, 100000)]
    assert np.ptp(score) < 1e-9
    back = ob.rope(ob.rope(q, [[7, 9]], **kw), [[7, 9]], transpose=True, **kw)
    assert np.abs(back - q).max() < 1e-14
    assert np.array_equal(ob.rope(q, [[7, 9]], **kw)[..., 40:], q[..., 40:])


# ---------------------------------------------------------------- the rotary plan
ROPES = [
    dict(axis_dims=[64]),
    dict(axis_dims=[44, 42, 42], grid=(30, 52)),
    dict(axis_dims=[6], layout="half", scaling="linear", factor=3.5),
    dict(axis_dims=[32, 32], scaling="base", factor=[4.0, 1.0], grid=(1, 7), start=(-3, 2)),
    dict(axis_dims=[48], layout="half", scaling="by_parts", factor=16.0, original_length=8192, beta_slow=1.0, beta_fast=32.0),
    dict(axis_dims=[2], base=500000.0),
]


@pytest.mark.parametrize("kw", ROPES, ids=lambda k: f"{k['axis_dims']}-{k.get('scaling', 'none')}")
def test_rope_plan(mb, kw):
    """Each pair's turn per step, as a fraction of 2^64, against exact rational arithmetic on the oracle's theta
    (fp64: its relative error of a few 2^-53, with powers up to 2^-48, is what separates the two)."""
    plan = mb.make_rope(**kw)
    theta, axis = ob.rope_thetas(kw["axis_dims"], **{k: v for k, v in kw.items() if k in (
        "scaling", "base", "factor", "original_length", "beta_slow", "beta_fast")})
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    assert plan.pairs == len(theta) and plan.n_axes == len(kw["axis_dims"])
    for j, t in enumerate(theta):
        exact = Fraction(float(t)) / (2 * pi) * 2 ** 64
        assert abs(Fraction(plan.turns[j]) - exact) <= exact * Fraction(1, 2 ** 48) + 1
    got_axis = np.repeat(np.arange(3), list(plan.axis_pairs))
    assert np.array_equal(got_axis, axis)
    assert list(plan.start) == list(kw.get("start", (0, 0, 0))) + [0] * (3 - len(kw.get("start", (0, 0, 0))))


def test_rope_plan_refusals(mb):
    for kw in (dict(axis_dims=[7]), dict(axis_dims=[0]), dict(axis_dims=[]), dict(axis_dims=[8] * 4), dict(axis_dims=[-2]),
               dict(axis_dims=[8], base=0.5), dict(axis_dims=[8], base=float("nan")), dict(axis_dims=[8], layout="spiral"),
               dict(axis_dims=[8], scaling="linear", factor=0.0), dict(axis_dims=[8], scaling="linear", factor=float("inf")),
               dict(axis_dims=[8], scaling="by_parts", factor=2.0), dict(axis_dims=[8], amplitude=float("nan")),
               dict(axis_dims=[8], scaling="by_parts", factor=2.0, original_length=100, beta_slow=3.0, beta_fast=3.0)):
        with pytest.raises(mb.MogaError) as e:
            mb.make_rope(**kw)
        assert e.value.code == 1, kw
    with pytest.raises(mb.MogaError) as e:
        mb.make_rope([100, 100])
    assert e.value.code == 2


def test_rope_plan_refuses_what_it_would_cut(mb):
    """Numbers past 32 bits, and lists that are not one number for each axis."""
    for kw in (dict(axis_dims=[64], start=(2 ** 31,)), dict(axis_dims=[64], start=(-2 ** 31 - 1,)), dict(axis_dims=[64], start=(2 ** 32 + 5,)),
               dict(axis_dims=[2 ** 32 + 64]), dict(axis_dims=[32, 32], grid=(1, 2 ** 32 + 7)), dict(axis_dims=[32, 32], grid=(7,)),
               dict(axis_dims=[32, 32], scaling="linear", factor=[4.0]), dict(axis_dims=[32], scaling="linear", factor=[4.0, 2.0]),
               dict(axis_dims=[16, 16, 16], start=(5, 1)), dict(axis_dims=[64], start=(5, 1))):
        with pytest.raises(mb.MogaError) as e:
            mb.make_rope(**kw)
        assert e.value.code == 1, kw
    assert list(mb.make_rope([64], start=(-2 ** 31,)).start) == [-2 ** 31, 0, 0]
    assert list(mb.make_rope([32, 32], start=(2 ** 31 - 1, 3)).start) == [2 ** 31 - 1, 3, 0]


# ---------------------------------------------------------------- refusals of the entry points: nothing is launched
def _p(addr):
    return ctypes.c_void_p(addr)


A, Bp, Cp, Dp, Ep, Fp, Gp, Hp, Ip = (0x10000000 * (i + 1) for i in range(9))   # far apart, 16-byte aligned
Z, SZ = ctypes.c_void_p(0), ctypes.c_size_t(1 << 30)


def test_layernorm_refusals(mb):
    sh, lib = mb.make_shape(_cfg()), mb.lib
    r = ctypes.byref

    def call(shape=sh, norm=mb.make_norm(), X=A, W=Bp, b=Cp, Y=Dp, m=Ep, v=Fp):
        return lib.moga_layernorm(None if shape is None else r(shape), None if norm is None else r(norm), _p(X), _p(W), _p(b), _p(Y), _p(m), _p(v), Z)

    for kw in (dict(shape=None), dict(norm=None), dict(norm=mb.make_norm(eps=0.0)), dict(norm=mb.make_norm(eps=float("nan"))),
               dict(norm=mb.make_norm(eps=-1.0)), dict(X=0), dict(Y=0), dict(X=A + 4), dict(W=Bp + 8), dict(Y=A + 16), dict(Y=Bp),
               dict(m=Ep + 2), dict(v=Ep), dict(m=A)):
        assert call(**kw) == 1, kw
    n = mb.make_norm()
    n.per_batch = 2
    assert call(norm=n) == 1
    assert call(shape=mb.make_shape(_cfg(C=8196))) == 2           # rows of more than 32,768 bytes
    assert call(shape=mb.make_shape(_cfg(C=16392, dtype="bf16"))) == 2
    assert call(shape=mb.make_shape(_cfg(B=4, N=2 ** 30))) == 2   # 2^32 tokens
    assert call(shape=mb.make_shape(_cfg(C=66))) == 2             # not whole 16-byte vectors
    assert call(shape=mb.make_shape(_cfg(N=0)), X=0, Y=0) == 0


def test_residual_norm_refusals(mb):
    sh, lib, r = mb.make_shape(_cfg()), mb.lib, ctypes.byref

    def call(drop=mb.make_dropout(0.1, 1), X=A, R=Bp, W=Cp, b=Dp, H=Ep, Y=Fp):
        return lib.moga_residual_norm(r(sh), r(mb.make_norm()), None if drop is None else r(drop), _p(X), _p(R), _p(W), _p(b), _p(H), _p(Y), Z, Z, Z)

    step = mb.make_dropout(0.1, 1)
    step.step = 0x1004
    for kw in (dict(drop=mb.make_dropout(1.0, 1)), dict(drop=mb.make_dropout(-0.1, 1)), dict(drop=mb.make_dropout(float("nan"), 1)),
               dict(drop=step), dict(R=0), dict(H=0), dict(Y=Ep), dict(H=A + 32), dict(Y=Bp + 32), dict(H=Cp), dict(drop=None, X=0)):
        assert call(**kw) == 1, kw


def test_norm_backward_refusals(mb):
    sh, lib, r, n = mb.make_shape(_cfg()), mb.lib, ctypes.byref, mb.make_norm()
    need = mb.moga_layernorm_backward_workspace_bytes(sh, n)
    assert need > 0

    def call(X=A, W=Bp, m=Cp, v=Cp + 4096, dY=Dp, dX=Ep, dW=Fp, db=Gp, ws=Hp, size=need):
        return lib.moga_layernorm_backward(r(sh), r(n), _p(X), _p(W), _p(m), _p(v), _p(dY), _p(dX), _p(dW), _p(db), _p(ws), ctypes.c_size_t(size), Z)

    for kw in (dict(X=0), dict(m=0), dict(v=0), dict(dY=0), dict(dX=0), dict(dX=Dp + 16), dict(dW=Fp + 2), dict(dW=Gp), dict(dX=Fp), dict(db=A),
               dict(ws=A), dict(dW=Bp)):
        assert call(**kw) == 1, kw
    for kw in (dict(ws=0), dict(ws=Hp + 64), dict(size=need - 1)):
        assert call(**kw) == 3, kw

    def residual(dH=0, dX=Ep, dR=Ip, drop=None):
        return lib.moga_residual_norm_backward(r(sh), r(n), drop, _p(A), _p(Bp), _p(Cp), _p(Cp + 4096), _p(Dp), _p(dH), _p(dX), _p(dR), _p(Fp), _p(Gp), _p(Hp), ctypes.c_size_t(need), Z)

    for kw in (dict(dR=0), dict(dR=Ep), dict(dH=Ep + 16), dict(drop=r(mb.make_dropout(2.0, 0)))):
        assert residual(**kw) == 1, kw
    assert mb.moga_layernorm_backward_workspace_bytes(mb.make_shape(_cfg(C=66)), n) == 0


def test_workspace_grows_with_the_problem(mb):
    """Partial rows: at least one for each item, and at most 512 rows of a thread behind each."""
    n, per = mb.make_norm(), mb.make_norm(per_batch=True)
    for cfg in (_cfg(B=1, N=1), _cfg(B=700, N=3), _cfg(B=1, N=126360, C=5120, dtype="bf16"), _cfg(B=1, N=561600, C=5120, dtype="bf16")):
        sh = mb.make_shape(cfg)
        for norm, items in ((n, 1), (per, cfg.B)):
            partials = (mb.moga_layernorm_backward_workspace_bytes(sh, norm) - 256) // (8 * cfg.C)
            assert partials >= items
            assert partials <= 148 * 8 * math.ceil(cfg.B * cfg.N / (148 * 512)) + items


def test_partial_sums_of_the_longest_problems(mb):
    """A thread adds at most 512 rows in fp32, so a partial row stands for at most 512 rows of each of a block's groups: one of
    them for rows of 5,120 channels, 16 for 1,000, 32 for 8."""
    n, per = mb.make_norm(), mb.make_norm(per_batch=True)
    for norm, cfg, groups in ((per, _cfg(B=300, N=126360, C=5120, dtype="bf16"), 1), (n, _cfg(B=1, N=2 ** 31 - 1, C=8, dtype="bf16"), 32),
                              (per, _cfg(B=160, N=561600, C=1000, dtype="bf16"), 16), (n, _cfg(B=40, N=561600, C=5120), 1)):
        items, rows = (cfg.B, cfg.N) if norm is per else (1, cfg.B * cfg.N)
        partials = (mb.moga_layernorm_backward_workspace_bytes(mb.make_shape(cfg), norm) - 256) // (8 * cfg.C)
        assert partials >= items * math.ceil(rows / (512 * groups)), cfg
        assert partials <= 2 * items * math.ceil(rows / (512 * groups)) + 148 * 8


def test_dropout_refusals(mb):
    sh, lib, r = mb.make_shape(_cfg()), mb.lib, ctypes.byref

    def call(drop=mb.make_dropout(0.5, 3), X=A, R=0, Y=Bp):
        return lib.moga_dropout_add(r(sh), None if drop is None else r(drop), _p(X), _p(R), _p(Y), Z)

    for kw in (dict(drop=None), dict(drop=mb.make_dropout(1.0, 3)), dict(X=0), dict(Y=0), dict(Y=A + 16), dict(R=Cp + 4), dict(R=Bp + 16)):
        assert call(**kw) == 1, kw


def test_rope_refusals(mb):
    lib, r = mb.lib, ctypes.byref
    sh, plan = mb.make_shape(_cfg()), mb.make_rope([64])

    def call(shape=sh, plan=plan, pos=0, per=0, Q=A, K=Bp, Qo=Cp, Ko=Dp):
        return lib.moga_rope(r(shape), None if plan is None else r(plan), _p(pos), ctypes.c_int32(per), _p(Q), _p(K), _p(Qo), _p(Ko), ctypes.c_int32(0), Z)

    s = lambda *st: mb.make_shape(_cfg(), strides=st)
    for kw in (dict(plan=None), dict(plan=mb.MogaRopePlan()), dict(pos=2), dict(per=2), dict(Q=0), dict(Qo=0), dict(Ko=0), dict(K=0),
               dict(Qo=A + 16), dict(Qo=Bp), dict(Ko=Cp), dict(Ko=A), dict(pos=Cp), dict(Q=A + 8), dict(plan=mb.make_rope([8, 8])),
               dict(plan=mb.make_rope([8, 8, 8], grid=(0, 5))),
               dict(shape=s(1280, 0, 64)), dict(shape=s(1280, 640, 64 - 4)), dict(shape=s(640, 640, 64)), dict(shape=s(1280, 320, 64))):
        assert call(**kw) == 1, kw
    # one projection's [B, N, 3, H, D] output: the rows of Q and K alternate, but they may not meet
    packed = s(10 * 384, 64, 384)
    e = 4
    for kw in (dict(Q=A, Qo=A, K=A + 64 * e, Ko=A + 64 * e), dict(Q=A, Qo=A, K=A + 120 * e, Ko=A + 120 * e), dict(Q=A, Qo=A + 384 * e), dict(Q=A, Qo=A + 100 * e),
               dict(Q=A, Qo=A, K=A + 9 * 384 * e, Ko=A + 9 * 384 * e), dict(Q=A + 19 * 384 * e, Qo=A + 19 * 384 * e, K=A, Ko=A)):
        assert call(**{**dict(shape=packed, K=0, Ko=0), **kw}) == 1, kw
    assert call(plan=mb.make_rope([128])) == 2                    # more rotated channels than the head has
    assert call(shape=mb.make_shape(_cfg(N=0)), Q=0, Qo=0) == 0


def test_permute_rope_refusals(mb):
    lib, r = mb.lib, ctypes.byref
    sh, plan = mb.make_shape(_cfg()), mb.make_rope([64])
    need = mb.moga_scratch_bytes(sh)

    def call(plan=plan, gid=A, Q=Bp, K=Cp, V=Dp, Qp=Ep, Kp=Fp, Vp=Gp, size=need):
        return lib.moga_permute_rope(r(sh), None if plan is None else r(plan), Z, ctypes.c_int32(0), _p(gid), _p(Q), _p(K), _p(V), _p(Hp), _p(Hp + (1 << 20)),
                                     _p(Hp + (2 << 20)), _p(Qp), _p(Kp), _p(Vp), _p(Ip), ctypes.c_size_t(size), Z)

    for kw in (dict(plan=None), dict(gid=0), dict(Qp=0), dict(Vp=0), dict(Qp=Bp), dict(Qp=Fp), dict(Vp=Dp), dict(Q=0)):
        assert call(**kw) == 1, kw
    assert call(size=need - 1) == 3

    def back(a=A, b=Bp, c=Cp, inv=Dp, x=Ep, y=Fp, z=Gp):
        return lib.moga_permute_rope_backward(r(sh), r(plan), Z, ctypes.c_int32(0), _p(a), _p(b), _p(c), _p(inv), _p(x), _p(y), _p(z), Z)

    for kw in (dict(a=0), dict(inv=0), dict(x=A), dict(y=Ep), dict(z=0), dict(x=Dp)):
        assert back(**kw) == 1, kw


def test_forward_and_backward_rope_refusals(mb):
    lib, r = mb.lib, ctypes.byref
    sh, plan = mb.make_shape(_cfg()), mb.make_rope([128])
    args = [r(sh), r(plan), Z, ctypes.c_int32(0)]
    assert lib.moga_forward_rope(*args, *[_p(A)] * 7, *[Z] * 4, _p(Bp), SZ, Z) == 2
    assert lib.moga_backward_rope(*args, *[_p(A)] * 14, _p(Bp), SZ, Z) == 2
    none = mb.make_shape(_cfg(N=0))                                # no tokens: nothing to do, as moga_forward
    ok = [r(none), r(mb.make_rope([64])), Z, ctypes.c_int32(0)]
    assert lib.moga_forward_rope(*ok, *[Z] * 11, Z, SZ, Z) == 0
    assert lib.moga_backward_rope(*ok, *[Z] * 14, Z, SZ, Z) == 0
    assert lib.moga_rope(*ok, *[Z] * 4, ctypes.c_int32(0), Z) == 0
    assert lib.moga_permute_rope_backward(*ok, *[Z] * 7, Z) == 0
    over = [r(mb.make_shape(_cfg(), strides=(1280, 0, 64))), r(mb.make_rope([64])), Z, ctypes.c_int32(0)]
    assert lib.moga_forward_rope(*over, *[_p(A)] * 7, *[Z] * 4, _p(Bp), SZ, Z) == 1
    args[1] = None
    assert lib.moga_forward_rope(*args, *[_p(A)] * 7, *[Z] * 4, _p(Bp), SZ, Z) == 1
    assert lib.moga_backward_rope(*args, *[_p(A)] * 14, _p(Bp), SZ, Z) == 1


def _refuses_overlaps(call, inputs, outputs, size):
    """call(**addresses) refuses every output over an input or another output: at the same address, and over its last
    bytes (size: the bytes of each)."""
    at = {name: 0x10000000 * (i + 1) for i, name in enumerate([*inputs, *outputs])}
    for i, out in enumerate(outputs):
        for other in [*inputs, *outputs[:i], *outputs[i + 1:]]:
            assert call(**{**at, out: at[other]}) == 1, (out, other)
            assert call(**{**at, out: at[other] + (size[other] - 1) // 16 * 16}) == 1, (out, other, "end")


def test_permute_rope_refuses_overlaps(mb):
    sh, plan = mb.make_shape(_cfg(k=2)), mb.make_rope([32, 32], grid=(2, 5))
    need = mb.moga_scratch_bytes(sh)
    names = ("gid", "Q", "K", "V", "perm", "inv", "offsets", "Qp", "Kp", "Vp", "ws")

    def call(pos, per=0, **at):
        return mb.lib.moga_permute_rope(ctypes.byref(sh), ctypes.byref(plan), _p(pos), ctypes.c_int32(per), *[_p(at[n]) for n in names], ctypes.c_size_t(need), Z)

    ints, rows = 4 * 2 * 10 * 2, 4 * 2 * 2 * 10 * 64
    size = dict(pos=4 * 10 * 2, gid=ints, Q=rows, K=rows, V=rows, perm=ints, inv=ints, offsets=4 * 2 * 5, Qp=2 * rows, Kp=2 * rows, Vp=2 * rows, ws=need)
    _refuses_overlaps(call, ("pos",) + names[:4], names[4:], size)
    at = {n: 0x10000000 * (i + 1) for i, n in enumerate(names)}
    assert call(pos=at["Qp"] - 80, per=1, **at) == 1              # positions of each batch item: twice as long


def test_forward_rope_refuses_overlaps(mb):
    plan = mb.make_rope([32, 32], grid=(2, 5))
    names = ("X", "Wr", "bias", "Q", "K", "V", "O", "gid", "gate", "perm", "offsets", "ws")

    def call(pos, shape=mb.make_shape(_cfg(k=2)), **at):
        return mb.lib.moga_forward_rope(ctypes.byref(shape), ctypes.byref(plan), _p(pos), ctypes.c_int32(0), *[_p(at[n]) for n in names], SZ, Z)

    words, rows = 4 * 2 * 10 * 2, 4 * 2 * 2 * 10 * 64
    size = dict(pos=4 * 10 * 2, X=4 * 2 * 10 * 64, Wr=4 * 64 * 4, bias=4 * 4, Q=rows, K=rows, V=rows, O=rows, gid=words, gate=words, perm=words,
                offsets=4 * 2 * 5, ws=mb.moga_workspace_bytes(mb.make_shape(_cfg(k=2))))
    _refuses_overlaps(call, ("pos",) + names[:6], names[6:], size)
    # the rows of Q, K, V and O alternate in one [B, N, 4, H, D] tensor: they may, up to the row
    packed = mb.make_shape(_cfg(k=2), strides=(10 * 512, 64, 512))
    at = {n: 0x10000000 * (i + 1) for i, n in enumerate(("pos",) + names)}
    at.update(shape=packed, Q=A, K=A + 512, V=A + 1024, pos=0, ws=0)
    assert call(**{**at, "O": A + 1536}) == 3                     # only the workspace is missing
    assert call(**{**at, "O": A + 1536 - 16}) == 1 and call(**{**at, "O": A + 1024}) == 1 and call(**{**at, "O": A + 512 + 2048}) == 1


def test_backward_rope_refuses_overlaps(mb):
    plan, sh = mb.make_rope([32, 32], grid=(2, 5)), mb.make_shape(_cfg(k=2))
    names = ("Qp", "Kp", "Vp", "Op", "lse", "gate", "perm", "inv", "offsets", "dO", "dQ", "dK", "dV", "dgate", "ws")

    def call(pos, shape=sh, **at):
        return mb.lib.moga_backward_rope(ctypes.byref(shape), ctypes.byref(plan), _p(pos), ctypes.c_int32(0), *[_p(at[n]) for n in names], SZ, Z)

    words, rows = 4 * 2 * 10 * 2, 4 * 2 * 2 * 10 * 64
    size = dict(pos=4 * 10 * 2, lse=2 * words, gate=words, perm=words, inv=words, offsets=4 * 2 * 5, dO=rows, dQ=rows, dK=rows, dV=rows,
                dgate=words, ws=mb.moga_backward_workspace_bytes(sh), **{n: 2 * rows for n in names[:4]})
    _refuses_overlaps(call, ("pos",) + names[:10], names[10:], size)
    packed = mb.make_shape(_cfg(k=2), strides=(10 * 512, 64, 512))
    at = {n: 0x10000000 * (i + 1) for i, n in enumerate(names)}
    at.update(shape=packed, dQ=A + (9 << 32), dK=A + (9 << 32) + 512, dV=A + (9 << 32) + 1024, pos=0, ws=0)
    last = A + (9 << 32) + 1536
    assert call(**{**at, "dO": last}) == 3                        # only the workspace is missing
    assert call(**{**at, "dO": last - 16}) == 1 and call(**{**at, "dO": at["dV"]}) == 1 and call(**{**at, "dO": at["dK"] + 2048}) == 1


def test_overlaps_are_told_row_by_row(mb):
    """Strided rows and contiguous tensors around and between them, placed at random: refused (1) if and only if any two share
    a byte; otherwise only the workspace is missing (3)."""
    rng, lib, r = np.random.default_rng(5), mb.lib, ctypes.byref
    plan, base, seen = mb.make_rope([64]), 0x100000000, {1: 0, 3: 0}
    for _ in range(4000):
        B, H, N, D, k = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 5)), 64, 1
        axes, strides, reach = [("b", B), ("h", H), ("n", N)], {}, D
        for i in rng.permutation(3):                               # strides whose rows are apart, in any order of the axes
            name, size = axes[i]
            strides[name] = reach + 4 * int(rng.choice([0, 0, 4, 16, 40, 200]))
            reach = (size - 1) * strides[name] + reach if size > 1 else reach
        cfg = _cfg(B=B, H=H, N=N, k=k)
        sh = mb.make_shape(cfg, strides=(strides["b"], strides["h"], strides["n"]))
        extent = 4 * reach
        at = {"O": base}
        for t in ("Q", "K", "V"):                                  # far away, or near O
            at[t] = base + (int(rng.integers(-extent // 16, extent // 16 + 1)) * 16 if rng.random() < 0.4 else (1 << 24) * (1 + "QKV".index(t)))
        size = dict(gid=4 * B * N, gate=4 * B * N, perm=4 * B * N, offsets=4 * B * 5, X=4 * B * N * 64, Wr=4 * 64 * 4, bias=16, pos=4 * N)
        for i, t in enumerate(size):
            at[t] = base + (int(rng.integers(-20, extent // 16 + 4)) * 16 if t in ("gid", "offsets", "pos", "bias") and rng.random() < 0.3 else (1 << 25) * (2 + i))
        names = ("X", "Wr", "bias", "Q", "K", "V", "O", "gid", "gate", "perm", "offsets")
        got = lib.moga_forward_rope(r(sh), r(plan), _p(at["pos"]), ctypes.c_int32(0), *[_p(at[n]) for n in names], Z, SZ, Z)
        rows = np.array([4 * (b * strides["b"] + h * strides["h"] + n * strides["n"]) for b in range(B) for h in range(H) for n in range(N)])
        spans = {t: [(at[t] + int(o), at[t] + int(o) + 4 * D) for o in rows] for t in "QKVO"} | {t: [(at[t], at[t] + size[t])] for t in size}
        outs = ("O", "gid", "gate", "perm", "offsets")
        meet = any(x[0] < y[1] and y[0] < x[1] for o in outs for t in spans if t != o for x in spans[o] for y in spans[t])
        assert got == (1 if meet else 3), (at, strides, B, H, N)
        seen[got] += 1
    assert min(seen.values()) > 500


def test_tensors_in_the_gaps_of_padded_rows(mb):
    """Batch items of up to 64 tokens, of which 10 are used: indexes and sorted rows may lie behind an item's tokens."""
    lib, r, plan = mb.lib, ctypes.byref, mb.make_rope([64])
    sh = mb.make_shape(_cfg(), strides=(2 * 64 * 64, 64 * 64, 64))                 # [2, 2, 64, 64], N = 10
    behind = A + 4 * 10 * 64                                                       # of head 0 of item 0
    names = ("gid", "Q", "K", "V", "perm", "inv", "offsets", "Qp", "Kp", "Vp")
    at = {n: 0x10000000 * (i + 1) for i, n in enumerate(names)}
    at["Q"], need = A, mb.moga_scratch_bytes(sh)

    def call(**kw):
        return lib.moga_permute_rope(r(sh), r(plan), Z, ctypes.c_int32(0), *[_p({**at, "gid": Bp << 8, **kw}[n]) for n in names], Z, ctypes.c_size_t(need), Z)

    assert call(perm=behind, inv=behind + 256, offsets=behind + 512) == 3
    assert call(perm=behind - 16) == 1 and call(inv=A + 4 * 64 * 64 - 64) == 1
    assert call(Qp=behind) == 3 and call(Qp=behind + 8192) == 1                    # 10,240 of the 13,824 bytes before head 1


def test_permute_rope_backward_refuses_overlaps(mb):
    plan, sh = mb.make_rope([32, 32], grid=(2, 5)), mb.make_shape(_cfg(k=2))
    names = ("dQp", "dKp", "dVp", "inv", "dQ", "dK", "dV")

    def call(pos, per=0, **at):
        return mb.lib.moga_permute_rope_backward(ctypes.byref(sh), ctypes.byref(plan), _p(pos), ctypes.c_int32(per), *[_p(at[n]) for n in names], Z)

    rows = 4 * 2 * 2 * 10 * 64
    size = dict(pos=4 * 10 * 2, inv=4 * 2 * 10 * 2, dQ=rows, dK=rows, dV=rows, dQp=2 * rows, dKp=2 * rows, dVp=2 * rows)
    _refuses_overlaps(call, ("pos",) + names[:4], names[4:], size)
    at = {n: 0x10000000 * (i + 1) for i, n in enumerate(names)}
    assert call(pos=at["dV"] - 80, per=1, **at) == 1


def test_dropout_step_word_over_an_output(mb):
    """The device word that is added to the offset may lie in no output: some blocks would read what others have written."""
    sh, lib, r, n = mb.make_shape(_cfg()), mb.lib, ctypes.byref, mb.make_norm()
    drop, need = mb.make_dropout(0.1, 1), mb.moga_layernorm_backward_workspace_bytes(sh, n)
    t, rows = 4 * 2 * 10 * 64, 4 * 2 * 10
    for last in (0, 1):
        for out, size in ((Cp, t), (Dp, t), (Ep, rows), (Fp, rows)):
            drop.step = out + (size - 8) * last
            assert lib.moga_residual_norm(r(sh), r(n), r(drop), _p(A), _p(Bp), Z, Z, _p(Cp), _p(Dp), _p(Ep), _p(Fp), Z) == 1, (out, last)
        for out, size in ((Ep, t), (Fp, t), (Gp, 256), (Hp, 256), (Ip, need)):
            drop.step = out + (size - 8) * last
            assert lib.moga_residual_norm_backward(r(sh), r(n), r(drop), _p(A), Z, _p(Bp), _p(Bp + 4096), _p(Cp), _p(Dp), _p(Ep), _p(Fp), _p(Gp), _p(Hp), _p(Ip),
                                                   ctypes.c_size_t(need), Z) == 1, (out, last)
        drop.step = Bp + (t - 8) * last
        assert lib.moga_dropout_add(r(sh), r(drop), _p(A), Z, _p(Bp), Z) == 1


def test_binding_refuses_tensors_of_the_cpu(mb):
    sh = mb.make_shape(_cfg())
    x = torch.zeros(2, 10, 64)
    with pytest.raises(mb.MogaError):
        mb.moga_layernorm(sh, mb.make_norm(), x, None, None, x)
    with pytest.raises(mb.MogaError):
        mb.moga_dropout_add(sh, mb.make_dropout(0.1, 0), x, None, x)
    q = torch.zeros(2, 2, 10, 64)
    with pytest.raises(mb.MogaError):
        mb.moga_rope(sh, mb.make_rope([64]), None, q, None, q, None)
    with pytest.raises(mb.MogaError):
        mb.moga_rope(sh, mb.make_rope([64]), torch.zeros(9, 1, dtype=torch.int32), q, None, q, None)
    with pytest.raises(mb.MogaError):
        mb.make_dropout(0.1, 0, step=torch.zeros(1, dtype=torch.int64))


class _OnDevice:
    """Stands for a contiguous tensor of a CUDA device."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0, at=A):
        self.shape, self.dtype, self.index, self.at = shape, dtype, device, at
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.index

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return True

    def stride(self):
        return ()

    def data_ptr(self):
        return self.at

    def element_size(self):
        return self.dtype.itemsize


def test_binding_refuses_a_step_word_of_another_device(mb, monkeypatch):
    monkeypatch.setattr(mb, "_current_device", lambda: 0)
    sh, norm = mb.make_shape(_cfg()), mb.make_norm()
    drop = mb.make_dropout(0.1, 0, step=_OnDevice(1, dtype=torch.int64, device=1, at=Ip))
    x, r, h, y = (_OnDevice(2, 10, 64, at=at) for at in (A, Bp, Cp, Dp))
    m, v, ws = _OnDevice(2, 10, at=Ep), _OnDevice(2, 10, at=Fp), _OnDevice(1 << 20, dtype=torch.uint8, at=Gp)
    for call in (lambda: mb.moga_dropout_add(sh, drop, x, r, y), lambda: mb.moga_residual_norm(sh, norm, drop, x, r, None, None, h, y),
                 lambda: mb.moga_residual_norm_backward(sh, norm, drop, x, None, m, v, r, None, h, y, None, None, ws)):
        with pytest.raises(mb.MogaError) as e:
            call()
        assert e.value.code == 1 and "step word" in str(e.value)
